"""Cases that measure a paged cache in 8 bits and rotary positions: rotating queries and keys, appending tokens to the pages with the
rotation applied on the way, and attention over the pages.

A page holds e4m3 codes of `page` tokens for every KV head; 16 neighbouring slots of a head share a scale, a power of two that is
the smallest with which the largest of them stays within 448.  A block of slots that has tokens already keeps its scale or takes a
larger one, to which its codes are rounded again.  Keys are noise around heavy hitters that the queries attend to strongly, as
those are that were kept of a long prompt.  Where `own` is false the operators are computed from elementary torch operations.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"

# query heads, KV heads, head dim
SHAPES = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 2, 64)}
LIFT, SINK = 5.0, 7.0                  # logit lift of heavy hitters and of the first token
BLOCK = 16                             # slots that share a scale
TOP, LOW = 448.0, -40                  # largest code, smallest exponent of a scale


def _case(name, kind, shape, dtype="bf16", heads=0, tokens=0, batch=1, lengths=(), new=1, page=64, kept=0, ragged=False, rope="plain",
          dim=0, interleaved=False, inverse=False, far=0, queries=False, softcap=0.0):
    c = {"kind": kind, "shape": shape, "dtype": dtype, "heads": heads, "tokens": tokens, "batch": batch,
         "lengths": ",".join(map(str, lengths)), "new": new, "page": page, "kept": kept, "ragged": ragged, "rope": rope, "dim": dim,
         "interleaved": interleaved, "inverse": inverse, "far": far, "queries": queries, "softcap": softcap}
    return {"name": name, **c} if name else c


def listed():
    ragged = [411, 1024, 5003, 733, 2048, 300, 4096, 1500, 1, 2777, 640, 3500, 129, 4999, 900, 1777]
    return [
        # the observation window's queries of one layer, before they are scored: latency
        _case("rotate window llama 64", "rotate", "llama", heads=32, tokens=64, far=32704),
        # all keys of one layer of a 128K prompt, frequencies scaled by their wavelengths
        _case("rotate keys llama 131072", "rotate", "llama", heads=8, tokens=131072, rope="bands"),
        # the gradient's way back: part of the head, neighbouring elements paired, fp32, an odd length
        _case("rotate gradient small fp32", "rotate", "small", "fp32", heads=8, tokens=2047, batch=4, dim=32, interleaved=True,
              inverse=True, rope="linear"),
        # a decoding step of a serving batch: one token's keys, values and queries each
        _case("append llama 16 ragged", "append", "llama", lengths=ragged, queries=True, rope="bands"),
        # what a selection kept of one layer of a 128K prompt goes to pages
        _case("append 16384 of 131072 llama", "append", "llama", lengths=[0], new=131072, kept=16384),
        # prompts of different lengths behind what their sequences hold, far positions
        _case("append prompts qwen 4 ragged", "append", "qwen", lengths=[0, 1001, 77, 4000], new=8191, ragged=True, page=16,
              rope="ramp", far=900000),
        # one sequence over the smallest budget kept of a 128K prompt: latency
        _case("attend llama 1 x 1024", "attend", "llama", lengths=[1024]),
        # a serving batch whose sequences have all lengths, down to one token
        _case("attend llama 16 ragged", "attend", "llama", lengths=ragged),
        # sequences that keep the largest budget of a 128K prompt
        _case("attend llama 16 x 16384", "attend", "llama", lengths=[16384] * 16, page=128),
        # a few drafted tokens of a model that caps its scores; not every sequence has as many
        _case("verify 4 qwen 8 ragged", "attend", "qwen", lengths=[4096, 1001, 2500, 333, 4095, 64, 3777, 2049], new=4, ragged=True,
              softcap=30.0, page=32),
        # a longer piece of text over long caches: as much arithmetic as reading
        _case("verify 16 llama 4 x 8192", "attend", "llama", lengths=[8192] * 4, new=16),
        # a step of one layer: keys, values and queries are rotated, appended and attend
        _case("step llama 32 x 2048", "step", "llama", lengths=[2048 + 7 * i for i in range(32)], queries=True, rope="bands"),
    ]


def _size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, n | 1) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "step"])
    shape = rng.choice(["llama", "llama", "qwen", "small"])
    dtype = "fp32" if shape == "small" and rng.random() < 0.5 else "bf16"
    rope = rng.choice(["plain", "linear", "base", "bands", "ramp"])
    pairs = {"rope": rope, "dim": rng.choice([0, 0, 32, 48]), "interleaved": rng.random() < 0.4, "far": rng.choice([0, 5000, 1000000])}
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "rotate":
        batch = rng.randint(1, 8)
        return _case(None, kind, shape, dtype, rng.choice([1, 4, 8, 32]), _size(rng, 1, 16384 // batch), batch,
                     inverse=rng.random() < 0.3, **pairs)
    batch = _size(rng, 1, 32)
    if kind == "append":
        new = _size(rng, 1, 32768 // batch)
        lengths = [rng.choice([0, rng.randint(1, 3000)]) for _ in range(batch)]
        kept = _size(rng, 1, new) if new > 64 and rng.random() < 0.4 else 0
        return _case(None, kind, shape, dtype, lengths=lengths, new=new, page=page, kept=kept,
                     ragged=not kept and rng.random() < 0.5, queries=new <= 64 and rng.random() < 0.5, **pairs)
    longest = _size(rng, 16, 131072 // batch)
    lengths = [rng.randint(longest // 8, longest) for _ in range(batch)]
    new = rng.choice([1, 1, rng.randint(2, 4), rng.randint(2, 64 if longest * batch < 40000 else 16)])
    if kind == "attend":
        return _case(None, kind, shape, dtype, lengths=lengths, new=new, page=page, ragged=new > 1 and rng.random() < 0.5,
                     softcap=rng.choice([0.0, 0.0, 20.0, 50.0]))
    return _case(None, kind, shape, dtype, lengths=lengths, new=new, page=page, queries=True, **pairs)


# ---- inputs ------------------------------------------------------------------------------------
ROPES = {"plain": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
         "bands": {"factor": 8.0, "original": 8192, "slow": 1.0, "fast": 4.0},
         "ramp": {"factor": 32.0, "original": 32768, "slow": 1.0, "fast": 32.0}}
BASE = 500000.0


def _frequencies(case, d):
    """(angles per position of every pair, what cosine and sine are multiplied by)."""
    dim, kind, o = case["dim"] or d, case["rope"], ROPES[case["rope"]]
    base = BASE * o["factor"] ** (dim / (dim - 2)) if kind == "base" else BASE
    plain = [base ** (-2.0 * c / dim) for c in range(dim // 2)]
    if kind == "linear":
        return [f / o["factor"] for f in plain], 1.0
    if kind == "bands":                # short wavelengths stay, long ones are stretched, those between go over smoothly
        def of(f):
            part = (o["original"] * f / (2 * math.pi) - o["slow"]) / (o["fast"] - o["slow"])
            part = min(1.0, max(0.0, part))
            return part * f + (1 - part) * f / o["factor"]
        return [of(f) for f in plain], 1.0
    if kind == "ramp":                 # the same by the pair's number
        def pair(turns):
            return dim * math.log(o["original"] / (2 * math.pi * turns)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(pair(o["fast"]))), min(dim - 1, math.ceil(pair(o["slow"])))
        part = [1 - min(1.0, max(0.0, (c - lo) / max(hi - lo, 1e-3))) for c in range(dim // 2)]
        return [p * f + (1 - p) * f / o["factor"] for p, f in zip(part, plain)], 0.1 * math.log(o["factor"]) + 1
    return plain, 1.0


def _exponents(top):
    """Of the smallest power of two with which `top` stays within 448."""
    mantissa, exponent = torch.frexp(top)                   # top = mantissa 2^exponent, 0.5 <= mantissa < 1
    e = exponent - 9 + (mantissa > TOP / 512).to(exponent.dtype)
    return torch.where(top > 0, e, LOW).clamp_min(LOW)


def _codes(x):
    """[..., slots, d] as e4m3 codes and the exponents of the scales of 16 slots each."""
    y = x.unflatten(-2, (-1, BLOCK))
    e = _exponents(y.abs().amax(dim=(-2, -1)))
    return (y * torch.exp2(-e.to(y.dtype))[..., None, None]).flatten(-3, -2).to(torch.float8_e4m3fn), e


def prepare(case, seed):
    h, g, d = SHAPES[case["shape"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    steps, amplitude = _frequencies(case, d)

    def noise(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=dt)

    state = {"kind": case["kind"], "dim": case["dim"] or d, "interleaved": case["interleaved"], "inverse": case["inverse"],
             "steps": torch.tensor(steps, device=DEV, dtype=torch.float64), "amplitude": amplitude, "rope": case["rope"],
             "shape": (h, g, d), "dtype": dt, "page": case["page"]}
    if case["kind"] == "rotate":
        b, n = case["batch"], case["tokens"]
        first = torch.randint(0, 1000, (b, 1), generator=gen, device=DEV) + case["far"]
        # (heads before tokens, as the scorer takes them)
        x = noise(b, case["heads"], n, d).transpose(1, 2)
        return {**state, "x": x, "positions": (first + torch.arange(n, device=DEV)).to(torch.int32), "out": torch.empty_like(x)}
    lengths = [int(x) for x in case["lengths"].split(",")]
    b, t, page = len(lengths), case["new"], case["page"]
    most = case["kept"] or t
    columns = (max(lengths) + most + page - 1) // page
    pool = b * columns + 3
    # what the pages hold of earlier tokens; the others' slots hold what earlier sequences left
    common = torch.randn((b, g, 1, d), generator=gen, device=DEV)
    common *= math.sqrt(d) / common.norm(dim=-1, keepdim=True)
    rows = columns * page
    k, v = (torch.randn((b, g, rows, d), generator=gen, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    hitters = torch.rand((b, g, rows), generator=gen, device=DEV) < 0.02
    hitters[:, :, 0] = False
    k += (common * (hitters.unsqueeze(-1) * (LIFT / math.sqrt(d)))).to(k.dtype)
    k[:, :, :1] += (common * (SINK / math.sqrt(d))).to(k.dtype)
    v[:, :, :1] *= 0.05                                     # the first token's values are small
    places = torch.randperm(pool, generator=gen, device=DEV)
    table, state["spare"] = places[:b * columns].view(b, columns), places[-1]
    for name, x in (("k", k), ("v", v)):
        codes, e = _codes(x)
        to = torch.zeros((pool, g, page, d), device=DEV, dtype=torch.uint8)
        to[table] = codes.view(torch.uint8).view(b, g, columns, page, d).transpose(1, 2)
        scales = torch.full((pool, g, page // BLOCK), 127 + LOW, device=DEV, dtype=torch.uint8)
        scales[table] = (e + 127).to(torch.uint8).view(b, g, columns, -1).transpose(1, 2)
        state[name], state[name + "_scales"] = to.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)
    counts = [rng.randint(1, t) for _ in range(b)] if case["ragged"] else None
    state |= {
        "table": table.to(torch.int32), "lengths": torch.tensor(lengths, device=DEV, dtype=torch.int32), "new": t,
        "counts": torch.tensor(counts, device=DEV, dtype=torch.int32) if counts else None, "index": None, "queries": None,
        "scale": 1.0 / math.sqrt(d), "softcap": case["softcap"],
    }
    if case["kind"] in ("append", "step"):
        state |= {"k_new": noise(b, g, t, d).transpose(1, 2), "v_new": noise(b, g, t, d).transpose(1, 2),
                  "positions": ((state["lengths"][:, None] + case["far"]) + torch.arange(t, device=DEV, dtype=torch.int32)).contiguous()}
        if case["kept"]:
            state["index"] = torch.rand((b, t), generator=gen, device=DEV).argsort(-1)[:, :case["kept"]].sort(-1).values.to(torch.int32)
        if case["queries"]:
            state["queries"], state["q"] = noise(b, t, h, d), torch.empty((b, t, h, d), device=DEV, dtype=dt)
    if case["kind"] == "attend":
        group = common.view(b, 1, g, 1, d).expand(b, t, g, h // g, d).reshape(b, t, h, d)
        state["q"] = (noise(b, t, h, d).float() + group).to(dt)
    if case["kind"] != "append":
        state |= {"out": torch.empty((b, t, h, d), device=DEV, dtype=dt), "lse": torch.empty((b, t, h), device=DEV)}
    return state


# ---- the plain forms -----------------------------------------------------------------------------
def _rotated(s, x, positions):
    """x [batch, tokens, heads, d] at `positions` [batch, tokens], in 32 bits."""
    angle = positions.double()[:, :, None, None] * s["steps"]
    cos, sin = (torch.cos(angle) * s["amplitude"]).float(), (torch.sin(angle) * s["amplitude"]).float()
    if s["inverse"]:
        sin = -sin
    x, half = x.float(), s["dim"] // 2
    y = x.clone()
    first = slice(0, s["dim"], 2) if s["interleaved"] else slice(0, half)
    second = slice(1, s["dim"], 2) if s["interleaved"] else slice(half, s["dim"])
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def _store(s, name, x, there):
    """Rows x [batch, heads, tokens, d] go behind the first lengths[b] (those that are not `there` [batch, tokens] nowhere)."""
    g, d = s["shape"][1:]
    page, (b, columns), t, n = s["page"], s["table"].shape, x.shape[2], s["lengths"].long()[:, None]
    # the blocks that the rows may fall into, [batch, blocks]; those behind the table are of a page that nobody has
    blocks = (t + 2 * BLOCK - 2) // BLOCK
    first = (n // BLOCK + torch.arange(blocks, device=DEV)) * BLOCK
    inside = first < columns * page
    at = torch.where(inside, s["table"].long().gather(1, (first // page).clamp_max(columns - 1)), s["spare"])
    part = torch.where(inside, first % page // BLOCK, 0)
    codes, scales = s[name].view(-1, g, page // BLOCK, BLOCK, d).view(torch.uint8), s[name + "_scales"].view(torch.uint8)
    old, e_old = codes[at, :, part].view(s[name].dtype).float(), scales[at, :, part].int() - 127      # [batch, blocks, heads, ...]
    # the largest of a block's new values
    slot = n % BLOCK + torch.arange(t, device=DEV)
    rows = torch.zeros((b, g, blocks * BLOCK, d), device=DEV)
    rows.scatter_(2, slot[:, None, :, None].expand(x.shape), x * there[:, None, :, None])
    rows = rows.view(b, g, blocks, BLOCK, d).transpose(1, 2)
    fills = torch.zeros((b, blocks * BLOCK), device=DEV, dtype=torch.bool).scatter_(1, slot, there).view(b, blocks, 1, BLOCK)
    e, gets, live = _exponents(rows.abs().amax(dim=(-2, -1))), fills.any(-1), (first < n)[..., None]
    e = torch.where(gets, torch.where(live, torch.maximum(e, e_old), e), e_old)
    before = (first[..., None] + torch.arange(BLOCK, device=DEV) < n[..., None])[:, :, None]
    lower = torch.where(before, (e_old - e)[..., None], 0)
    new = torch.where(fills[..., None], rows * torch.exp2(-e.float())[..., None, None], old * torch.exp2(lower.float())[..., None])
    codes[at, :, part] = new.to(s[name].dtype).view(torch.uint8)
    scales[at, :, part] = (e + 127).to(torch.uint8)


def _append(s):
    k, v, positions = s["k_new"], s["v_new"], s["positions"]
    if s["index"] is not None:
        at = s["index"].long()
        rows = at[:, :, None, None].expand(-1, -1, *k.shape[2:])
        k, v, positions = k.gather(1, rows), v.gather(1, rows), positions.gather(1, at)
    i = torch.arange(k.shape[1], device=DEV)
    counts = s["counts"] if s["counts"] is not None else torch.full_like(s["lengths"], k.shape[1])
    there = i < counts[:, None]
    _store(s, "k", _rotated(s, k, positions).transpose(1, 2), there)
    _store(s, "v", v.float().transpose(1, 2), there)
    if s["queries"] is not None:
        s["q"].copy_(_rotated(s, s["queries"], s["positions"]))


def _dense(s, name):
    """Values of the pages, [batch, KV head, slot, d] in 32 bits."""
    table = s["table"].long()
    b, columns = table.shape
    g, d = s["shape"][1:]
    x = s[name][table].float().view(b, columns, g, -1, BLOCK, d)
    x = x * s[name + "_scales"][table].float()[..., None, None]
    return x.flatten(3, 4).transpose(1, 2).reshape(b, g, columns * s["page"], d)


def _attend(s):
    b, t, h, d = s["q"].shape
    g = s["shape"][1]
    k, v = _dense(s, "k"), _dense(s, "v")
    q = s["q"].float().view(b, t, g, h // g, d).permute(0, 2, 1, 3, 4).reshape(b, g, -1, d)
    x = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(b, g, t, h // g, -1)
    if s["softcap"]:
        x = s["softcap"] * torch.tanh(x / s["softcap"])
    slot, i = torch.arange(x.shape[-1], device=DEV), torch.arange(t, device=DEV)[None]
    last = s["lengths"].long()[:, None] + i                # the token's own slot
    if s["counts"] is not None:
        last = torch.where(i < s["counts"][:, None], last, -1)
    x = x.masked_fill((slot > last[..., None])[:, None, :, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul((p / total.clamp_min(1e-30)).view(b, g, -1, x.shape[-1]), v).view(b, g, t, -1, d)
    s["out"].copy_(o.transpose(1, 2).reshape(b, t, h, d))
    s["lse"].copy_((top + total.log()).squeeze(-1).transpose(1, 2).reshape(b, t, h))


# ---- the framework's calls -------------------------------------------------------------------------
_contexts = {}                         # one per model shape, as a program keeps them


def _handle(s):
    """What a program keeps beside its cache: a context of the model's shape, the pages' description, frequencies, a workspace."""
    if "context" not in s:
        from paper_2604_06746_b200 import binding
        key = (*s["shape"], s["dtype"])
        if key not in _contexts:
            _contexts[key] = binding.Context(*key[:3], 8, 8, key[3], DEV)
        ctx, scaling = _contexts[key], None if s["rope"] == "plain" else s["rope"]
        s["turns"] = binding.Rope(s["dim"], BASE, interleaved=s["interleaved"], scaling=scaling, **ROPES[s["rope"]])
        if s["kind"] != "rotate":
            s["pages"] = binding.Pages(s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"], s["lengths"])
        if s["kind"] in ("attend", "step"):
            s["workspace"] = ctx.attend_pages_workspace(s["pages"], s["new"])
        s["context"] = ctx
    return s["context"]


def run(s):
    kind = s["kind"]
    if own:
        ctx = _handle(s)
        if kind == "rotate":
            ctx.rotate(s["x"], s["positions"], s["turns"], out=s["out"], inverse=s["inverse"])
        if kind in ("append", "step"):
            ctx.append_pages(s["pages"], s["k_new"], s["v_new"], positions=s["positions"], rope=s["turns"], counts=s["counts"],
                             index=s["index"], q=s["queries"], q_out=s["q"] if s["queries"] is not None else None)
        if kind in ("attend", "step"):
            ctx.attend_pages(s["pages"], s["q"], s["scale"], s["out"], s["workspace"], counts=s["counts"], softcap=s["softcap"],
                             lse=s["lse"])
    else:
        if kind == "rotate":
            s["out"].copy_(_rotated(s, s["x"], s["positions"]))
        if kind in ("append", "step"):
            _append(s)
        if kind in ("attend", "step"):
            _attend(s)
    if kind == "rotate":
        return s["out"]
    pages = {name: s[name] for name in ("k", "k_scales", "v", "v_scales")} if kind != "attend" else {}
    if s["queries"] is not None:
        pages["q"] = s["q"]
    return pages if kind == "append" else {**pages, "out": s["out"], "lse": s["lse"]}


def work(case):
    h, g, d = SHAPES[case["shape"]]
    es = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "rotate":
        rows = case["batch"] * case["tokens"]
        return {"bytes": rows * (case["heads"] * 2 * d * es + 4), "flops": 3 * rows * case["heads"] * (case["dim"] or d)}
    lengths = [int(x) for x in case["lengths"].split(",")]
    b, most = len(lengths), case["kept"] or case["new"]
    tokens = b * (most + 1) // 2 if case["ragged"] else b * most       # (on average)
    row = 2 * d + 2 / BLOCK                                            # codes and scales of a token's K and V
    queries = b * case["new"] * h
    append = tokens * (g * (2 * d * es + row) + 4) + (2 * queries * d * es if case["queries"] else 0)
    slots = g * (sum(lengths) + tokens)
    attend = slots * row + 2 * queries * d * es + queries * 4
    flops = {"append": 6 * tokens * g * d, "attend": 4 * d * (h // g) * case["new"] * slots}
    if case["kind"] == "step":
        return {"bytes": append + attend, "flops": flops["append"] + flops["attend"]}
    return {"bytes": append if case["kind"] == "append" else attend, "flops": flops[case["kind"]]}


# ---- the definition in 64 bits ------------------------------------------------------------------------
def _turned(case, x, positions, d):
    """x [tokens, heads, d] in 64 bits, as products with complex numbers."""
    steps, amplitude = _frequencies(case, d)
    dim = case["dim"] or d
    angle = positions.double()[:, None, None] * torch.tensor(steps, device=DEV, dtype=torch.float64)
    by = torch.polar(torch.full_like(angle, amplitude), -angle if case["inverse"] else angle)
    part = x[..., :dim]
    part = part.unflatten(-1, (-1, 2)) if case["interleaved"] else part.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * by)
    z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., dim:]], dim=-1)


def _kept(codes, scales, table, n, x, page):
    """Writes rows x [tokens, heads, d] (64 bits) behind the first n of one sequence, a block of slots after another."""
    e = scales.view(torch.uint8)
    for lo in range(n // BLOCK * BLOCK, n + x.shape[0], BLOCK):
        at, slot = int(table[lo // page]), lo % page
        j = slot // BLOCK
        a, z = max(lo, n), min(lo + BLOCK, n + x.shape[0])
        new = x[a - n:z - n].transpose(0, 1)                # [heads, tokens, d]
        top = new.abs().amax(dim=(1, 2))
        exp = torch.where(top > 0, torch.ceil(torch.log2(top / TOP)), LOW).clamp_min(LOW)
        if a > lo:
            before = e[at, :, j].double() - 127
            exp = torch.maximum(exp, before)
            part = codes[at, :, slot:slot + a - lo]
            codes[at, :, slot:slot + a - lo] = (part.double() * torch.exp2(before - exp)[:, None, None]).to(codes.dtype)
        codes[at, :, slot + a - lo:slot + z - lo] = (new * torch.exp2(-exp)[:, None, None]).to(codes.dtype)
        e[at, :, j] = (exp + 127).to(torch.uint8)


def exact(case, seed):
    s = prepare(case, seed)
    h, g, d = SHAPES[case["shape"]]
    f64 = torch.float64
    if case["kind"] == "rotate":
        return torch.stack([_turned(case, x.to(f64), p, d) for x, p in zip(s["x"], s["positions"])])
    n_of, table = s["lengths"].tolist(), s["table"]
    b, t, page = len(n_of), case["new"], case["page"]
    counts = s["counts"].tolist() if s["counts"] is not None else [case["kept"] or t] * b
    if sum(counts) > 20000 and case["kind"] == "append":
        return None                                         # (a block after another takes too long)
    got = {}
    if case["kind"] in ("append", "step"):
        queries = []
        for i in range(b):
            at = s["index"][i].long() if s["index"] is not None else torch.arange(counts[i], device=DEV)
            k = _turned(case, s["k_new"][i, at].to(f64), s["positions"][i, at], d)
            _kept(s["k"], s["k_scales"], table[i], n_of[i], k, page)
            _kept(s["v"], s["v_scales"], table[i], n_of[i], s["v_new"][i, at].to(f64), page)
            if s["queries"] is not None:
                queries.append(_turned(case, s["queries"][i].to(f64), s["positions"][i], d))
        got = {name: s[name] for name in ("k", "k_scales", "v", "v_scales")}
        if queries:
            got["q"] = torch.stack(queries)
        if case["kind"] == "append":
            return got
    out = torch.zeros((b, t, h, d), dtype=f64, device=DEV)
    lse = torch.full((b, t, h), -math.inf, dtype=f64, device=DEV)
    rows = got["q"].to(s["dtype"]) if case["kind"] == "step" else s["q"]
    for i in range(b):
        n, c = n_of[i], counts[i] if case["ragged"] else t
        for j in range(g):
            k, v = ((s[name][table[i].long(), j].to(f64).unflatten(1, (-1, BLOCK)) *
                     s[name + "_scales"][table[i].long(), j].to(f64)[..., None, None]).reshape(-1, d)[:n + c] for name in "kv")
            heads = slice(j * (h // g), (j + 1) * (h // g))
            x = torch.einsum("thd,nd->thn", rows[i, :c, heads].to(f64), k) * s["scale"]
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            sees = torch.ones((c, n + c), dtype=torch.bool, device=DEV).tril(n)
            x = x.masked_fill(~sees[:, None], -math.inf)
            out[i, :c, heads] = torch.einsum("thn,nd->thd", torch.softmax(x, dim=-1), v)
            lse[i, :c, heads] = torch.logsumexp(x, dim=-1)
    return {**got, "out": out, "lse": lse}
