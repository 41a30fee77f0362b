"""Cases that measure decoding over a compacted cache: attention of new tokens (one, or a tree of drafted ones), the weight
that accepted tokens gave, eviction by accumulated weight, and the steps between them.

A cache holds, for every sequence (or layer and sequence) and KV head, `length` tokens in slots of its own, in any order, each
with the position it has in its prompt and the attention weight it has gathered.  Keys are noise around heavy hitters that the
queries attend to strongly, as they are in prompts that were compacted for them.  Where `own` is false the operators are
computed from elementary torch operations.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"

# query heads, KV heads, head dim
SHAPES = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 2, 64)}
LIFT, SINK = 5.0, 7.0                  # logit lift of heavy hitters and of the first token
SLACK = 32                             # slots of a cache beyond what a case fills


def _case(name, kind, shape, lengths, new, dtype="bf16", softcap=0.0, distance=False, head_step=0, accepted=0, budget=0,
          recent=0):
    c = {"kind": kind, "shape": shape, "lengths": ",".join(map(str, lengths)), "new": new, "dtype": dtype, "softcap": softcap,
         "distance": distance, "head_step": head_step, "accepted": accepted, "budget": budget, "recent": recent}
    return {"name": name, **c} if name else c


def listed():
    ragged = [411, 1024, 5003, 733, 2048, 300, 4096, 1500, 1, 2777, 640, 3500, 129, 4999, 900, 1777]
    return [
        # one sequence over the smallest budget kept of a 128K prompt, one token at a time: latency
        _case("decode llama 1 x 1024", "decode", "llama", [1024], 1),
        # a serving batch whose sequences have all lengths, down to one token
        _case("decode llama 16 ragged", "decode", "llama", ragged, 1),
        # sequences that keep the largest budget of a 128K prompt
        _case("decode llama 16 x 16384", "decode", "llama", [16384] * 16, 1),
        # a small model in fp32 whose scores fall with distance, heads that kept different numbers of tokens
        _case("decode small fp32 distance", "decode", "small", [2048, 777, 1301, 2000], 1, "fp32", distance=True, head_step=9),
        # a draft model's tree for one sequence
        _case("tree of 8 llama 1 x 2048", "tree", "llama", [2048], 8),
        # trees for a batch of a model that caps its scores
        _case("tree of 16 qwen 8 ragged", "tree", "qwen", [4096, 1001, 2500, 333, 4095, 64, 3777, 2049], 16, softcap=30.0),
        # large trees over long caches: as much arithmetic as reading
        _case("tree of 64 llama 4 x 16384", "tree", "llama", [16384] * 4, 64),
        # the weight that the accepted path of a tree gave, for the next eviction
        _case("weigh 3 of 8 llama 1 x 2048", "weigh", "llama", [2048], 8, accepted=3),
        _case("weigh 7 of 64 llama 4 x 16384", "weigh", "llama", [16384] * 4, 64, accepted=7),
        # every step one token comes and one goes, in all 32 layers at once
        _case("evict 1 of 2049, 32 layers", "evict", "llama", [2048] * 32, 1, budget=2048, recent=64),
        # a block of tokens goes at a time
        _case("evict 128 of 8320, 16 layers", "evict", "llama", [8192] * 16, 128, budget=8192, recent=256),
        # a whole speculative step of one layer: attention over the tree, weights of the accepted path, commit, eviction
        _case("speculative step llama 4 x 4096", "step", "llama", [4096] * 4, 8, accepted=4, budget=4096, recent=4),
    ]


def _size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, n | 1) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["decode", "decode", "tree", "tree", "weigh", "evict", "step"])
    shape = rng.choice(["llama", "llama", "qwen", "small"])
    dtype = "fp32" if shape == "small" and rng.random() < 0.5 else "bf16"
    batch = _size(rng, 1, 16)
    longest = _size(rng, 16, (16384 if kind == "decode" else 65536 // max(4, batch)) // (2 if dtype == "fp32" else 1))
    softcap, distance = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3
    step = rng.choice([0, 0, 1, 5]) if longest > 100 else 0
    if kind in ("decode", "tree", "weigh"):
        lengths = [rng.randint(max(1, longest // 8), longest) for _ in range(batch)]
        new = 1 if kind == "decode" else rng.randint(2, 64 if dtype == "bf16" else 12)
        return _case(None, kind, shape, lengths, new, dtype, softcap, distance, step if min(lengths) > 64 else 0,
                     rng.randint(1, min(new, 8)) if kind == "weigh" else 0)
    if kind == "evict":
        budget, layers = _size(rng, 64, 8192), rng.randint(1, 16)
        new = min(_size(rng, 1, 256), budget // 2)
        return _case(None, kind, shape, [budget] * layers, new, dtype, budget=budget, recent=rng.randint(0, budget // 4))
    budget, new = max(128, longest), rng.randint(2, 16)
    accepted = rng.randint(1, min(new, 5))
    return _case(None, kind, shape, [budget] * batch, new, dtype, softcap, distance, 0, accepted, budget, accepted)


# ---- inputs ------------------------------------------------------------------------------------
def _dims(case):
    h, g, d = SHAPES[case["shape"]]
    lengths = [int(x) for x in case["lengths"].split(",")]
    return h, g, d, lengths, [[max(0, n - i * case["head_step"]) for i in range(g)] for n in lengths]


def _tree(rng, new, path):
    """Parents of a tree whose first nodes are not all on the path that will be accepted: (masks, depths, accepted nodes)."""
    spine = sorted(rng.sample(range(new), path)) if path else []
    masks, depths, below = [], [], -1
    for i in range(new):
        if i in spine:
            parent, below = below, i
        else:
            parent = rng.randint(-1, i - 1)
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
        depths.append(depths[parent] + 1 if parent >= 0 else 0)
    return masks, depths, spine


def _signed(mask):
    return mask - (1 << 64) if mask >= 1 << 63 else mask


def prepare(case, seed):
    h, g, d, lengths, per_head = _dims(case)
    b, t, group = len(lengths), case["new"], h // g
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    cap = (max(lengths) + t + SLACK + 7) // 8 * 8

    def noise(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=dt)

    common = torch.randn((b, g, 1, d), generator=gen, device=DEV)
    common *= math.sqrt(d) / common.norm(dim=-1, keepdim=True)
    k, v = noise(b, g, cap, d), noise(b, g, cap, d)
    hitters = torch.rand((b, g, cap), generator=gen, device=DEV) < 0.02
    hitters[:, :, 0] = False
    k += (common * (hitters.unsqueeze(-1) * (LIFT / math.sqrt(d)))).to(dt)
    k[:, :, :1] += (common * (SINK / math.sqrt(d))).to(dt)
    q = (noise(b, t, h, d).float() + common.view(b, 1, g, 1, d).expand(b, t, g, group, d).reshape(b, t, h, d)).to(dt)
    # tokens that were kept of a prompt eight times as long, in order
    positions = torch.arange(cap, device=DEV, dtype=torch.int32) * 8
    positions = positions + torch.randint(0, 8, (b, g, cap), generator=gen, device=DEV, dtype=torch.int32)
    weights = 1 + torch.rand((b, g, cap), generator=gen, device=DEV)
    if case["kind"] == "evict":
        weights = torch.rand((b, g, cap), generator=gen, device=DEV) ** 4
    elif case["kind"] == "step":       # as many light tokens as will go
        light = torch.rand((b, g, cap), generator=gen, device=DEV) - 2.0 * hitters
        light[:, :, max(lengths):] = -2.0
        light = light.topk(case["accepted"], dim=-1).indices
        weights.scatter_(2, light, 1e-3)
    masks, depths, paths = zip(*(_tree(rng, t, case["accepted"]) for _ in range(b)))
    if case["kind"] in ("decode", "evict"):
        masks, depths = [[(2 << i) - 1 if i < 63 else -1 for i in range(t)]] * b, [list(range(t))] * b
    first = torch.tensor(lengths, device=DEV, dtype=torch.int32) * 8 + 8
    state = {
        "kind": case["kind"], "k": k, "v": v, "positions": positions.contiguous(), "weights": weights,
        "lengths": torch.tensor(per_head, device=DEV, dtype=torch.int32), "q": q, "k_new": noise(b, t, g, d),
        "v_new": noise(b, t, g, d),
        "new_positions": (first[:, None] + torch.tensor(depths, device=DEV, dtype=torch.int32)).contiguous(),
        "scale": 1.0 / math.sqrt(d), "softcap": case["softcap"], "budget": case["budget"], "recent": case["recent"],
        "slopes": torch.exp2(-8.0 * (torch.arange(h, device=DEV, dtype=torch.float32) + 1) / h) if case["distance"] else None,
        "tree": None, "accepted": None, "path": None, "counts": None, "new": t, "moved": case["accepted"] or t,
        "out": torch.empty((b, t, h, d), device=DEV, dtype=dt), "lse": torch.empty((b, t, h), device=DEV),
    }
    if case["kind"] in ("tree", "weigh", "step"):
        state["tree"] = torch.tensor([[_signed(m) for m in row] for row in masks], device=DEV, dtype=torch.int64)
    if case["accepted"]:
        state["accepted"] = torch.tensor([_signed(sum(1 << i for i in p)) for p in paths], device=DEV, dtype=torch.int64)
        state["path"] = torch.tensor([p + [-1] * (t - len(p)) for p in paths], device=DEV, dtype=torch.int32)
        state["counts"] = torch.tensor([len(p) for p in paths], device=DEV, dtype=torch.int32)
    if case["kind"] == "weigh":        # the drafts are in the cache, their attention was computed
        _append(state)
        logits = _logits(state)
        state["lse"] = torch.logsumexp(logits, dim=-1).transpose(1, 2).reshape(b, t, h).contiguous()
    return state


# ---- the plain forms -----------------------------------------------------------------------------
def _append(s):
    t = s["new"]
    at = s["lengths"].long()[:, :, None] + torch.arange(t, device=DEV)
    rows = at.unsqueeze(-1).expand(-1, -1, -1, s["k"].shape[-1])
    s["k"].scatter_(2, rows, s["k_new"].transpose(1, 2))
    s["v"].scatter_(2, rows, s["v_new"].transpose(1, 2))
    s["positions"].scatter_(2, at, s["new_positions"][:, None].expand(-1, at.shape[1], -1))
    s["weights"].scatter_(2, at, 0.0)


def _logits(s):
    """[batch, KV head, new token, head of the group, slot], minus infinity where a token is not seen."""
    b, g, cap, d = s["k"].shape
    t, n = s["new"], s["lengths"].long()[:, :, None, None]
    q = s["q"].float().view(b, t, g, -1, d).permute(0, 2, 1, 3, 4)
    group = q.shape[3]
    x = torch.matmul(q.reshape(b, g, t * group, d), s["k"].float().transpose(2, 3)).view(b, g, t, group, cap) * s["scale"]
    if s["softcap"]:
        x = s["softcap"] * torch.tanh(x / s["softcap"])
    slot = torch.arange(cap, device=DEV)
    if s["slopes"] is not None:
        far = s["new_positions"][:, None, :, None] - s["positions"][:, :, None, :]
        x = x - s["slopes"].view(1, g, 1, group, 1) * far.unsqueeze(3)
    draft = slot - n                                        # [batch, KV head, 1, slot]
    bits = s["tree"][:, None, :, None] if s["tree"] is not None else (2 << torch.arange(t, device=DEV))[:, None] - 1
    seen = (draft < 0) | ((draft < t) & ((bits >> draft.clamp(0, 63)) & 1).bool())
    return x.masked_fill(~seen.unsqueeze(3), -math.inf)


def _attend(s, accumulate):
    b, g, cap, d = s["k"].shape
    t = s["new"]
    x = _logits(s)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(dim=-1, keepdim=True)
    p = p / total
    o = torch.matmul(p.reshape(b, g, -1, cap), s["v"].float()).view(b, g, t, -1, d)
    s["out"].copy_(o.transpose(1, 2).reshape(b, t, -1, d))
    s["lse"].copy_((top + total.log()).squeeze(-1).transpose(1, 2).reshape(b, t, -1))
    if accumulate:
        s["weights"].add_(p.sum(dim=(2, 3)))


def _weigh(s):
    b, g, cap, d = s["k"].shape
    t = s["new"]
    p = torch.exp(_logits(s) - s["lse"].view(b, t, g, -1).transpose(1, 2).unsqueeze(-1))
    taken = (s["accepted"][:, None] >> torch.arange(t, device=DEV)) & 1
    s["weights"].add_((p * taken.view(b, 1, t, 1, 1)).sum(dim=(2, 3)))


def _commit(s):
    t, n = s["new"], s["lengths"].long()[:, :, None]
    i = torch.arange(t, device=DEV)
    if s["path"] is None:
        s["lengths"] += t
        return
    of = torch.where(i < s["counts"][:, None], s["path"].long(), i)[:, None] + n
    to = (n + i).expand_as(of)
    for x in (s["positions"], s["weights"]):
        x.scatter_(2, to, x.gather(2, of))
    rows = (-1, -1, -1, s["k"].shape[-1])
    for x in (s["k"], s["v"]):
        x.scatter_(2, to.unsqueeze(-1).expand(rows), x.gather(2, of.unsqueeze(-1).expand(rows)))
    s["lengths"] += s["counts"][:, None]


def _evict(s):
    """The tokens kept beyond the budget move, in order, into the slots below it whose tokens go."""
    budget, n = s["budget"], s["lengths"].long()[:, :, None]
    slot = torch.arange(s["k"].shape[2], device=DEV)
    live = slot < n
    newest = s["positions"].masked_fill(~live, -1).amax(dim=-1, keepdim=True)
    rank = s["weights"].masked_fill(s["positions"] > newest - s["recent"], math.inf).masked_fill(~live, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(live).scatter_(2, order[:, :, :budget], True) & live
    free, moves = ~kept & (slot < budget) & live, kept & (slot >= budget)
    most = min(s["k"].shape[2] - budget, budget)
    of = torch.sort((~moves).to(torch.int8), dim=-1, stable=True).indices[:, :, :most]
    to = torch.sort((~free).to(torch.int8), dim=-1, stable=True).indices[:, :, :most]
    of = torch.where(torch.arange(most, device=DEV) < moves.sum(dim=-1, keepdim=True), of, to)
    for x in (s["positions"], s["weights"]):
        x.scatter_(2, to, x.gather(2, of))
    rows = (-1, -1, -1, s["k"].shape[-1])
    for x in (s["k"], s["v"]):
        x.scatter_(2, to.unsqueeze(-1).expand(rows), x.gather(2, of.unsqueeze(-1).expand(rows)))
    s["lengths"].clamp_(max=budget)


# ---- the framework's calls -------------------------------------------------------------------------
_contexts = {}                         # one per model shape and workspace, as a program keeps them


def _handle(s):
    """What a program keeps beside its cache: a context of the model's shape, the cache's description, a workspace."""
    if "cache" not in s:
        from paper_2604_06746_b200 import binding
        b, g, cap, d = s["k"].shape
        key = (s["q"].shape[2], g, d, s["k"].dtype)
        if key not in _contexts:
            _contexts[key] = binding.Context(*key[:3], 8, 8, key[3], DEV)
        s["cache"] = binding.Cache(s["k"], s["v"], s["positions"], s["weights"], s["lengths"])
        s["workspace"] = _contexts[key].attend_workspace(s["cache"], s["new"]) if s["kind"] in ("decode", "tree", "step") else None
        s["context"] = _contexts[key]
    return s["context"], s["cache"], s["workspace"]


def run(s):
    kind = s["kind"]
    if own:
        ctx, cache, ws = _handle(s)
        if kind in ("decode", "tree", "step"):
            ctx.attend(cache, s["q"], s["scale"], s["out"], ws, k_new=s["k_new"], v_new=s["v_new"],
                       positions=s["new_positions"], tree=s["tree"], softcap=s["softcap"], slopes=s["slopes"], lse=s["lse"],
                       accumulate=kind == "decode")
        if kind in ("weigh", "step"):
            ctx.weigh(cache, s["q"], s["scale"], s["lse"], s["accepted"], tree=s["tree"], softcap=s["softcap"],
                      slopes=s["slopes"])
        if kind == "evict":
            ctx.append(cache, s["k_new"], s["v_new"], s["new_positions"])
        if kind in ("evict", "step"):
            ctx.commit(cache, s["new"], counts=s["counts"], path=s["path"])
            ctx.evict(cache, s["budget"], s["recent"])
    else:
        if kind in ("decode", "tree", "step"):
            _append(s)
            _attend(s, kind == "decode")
        if kind in ("weigh", "step"):
            _weigh(s)
        if kind == "evict":
            _append(s)
        if kind in ("evict", "step"):
            _commit(s)
            _evict(s)
    if kind in ("evict", "step"):
        s["new_positions"] += s["moved"]                    # the next tokens' places
    whole = {"k": s["k"], "v": s["v"], "positions": s["positions"], "weights": s["weights"], "lengths": s["lengths"]}
    if kind in ("decode", "tree", "step"):
        return {"out": s["out"], "lse": s["lse"], **whole}
    return {"weights": s["weights"]} if kind == "weigh" else whole


def work(case):
    h, g, d, lengths, per_head = _dims(case)
    es = 4 if case["dtype"] == "fp32" else 2
    t, b = case["new"], len(lengths)
    slots = sum(n + t for row in per_head for n in row)     # of all heads
    new = b * t * g
    queries = b * t * h
    row = 2 * d * es                                        # K and V of a token
    words = 4 if case["distance"] else 0                    # a position
    attend = {"bytes": slots * (row + words) + new * (row + 8) + 2 * queries * d * es + queries * 4,
              "flops": 4 * d * (h // g) * t * slots}
    rows = b * case["accepted"] * h
    weigh = {"bytes": slots * (row // 2 + 8 + words) + rows * (d * es + 4), "flops": 2 * d * (h // g) * case["accepted"] * slots}
    moved = b * g * (case["accepted"] or t)
    evict = {"bytes": slots * 8 + 2 * moved * (row + 8), "flops": 0}
    if case["kind"] == "decode":
        return {"bytes": attend["bytes"] + 8 * slots, "flops": attend["flops"]}
    if case["kind"] == "tree":
        return attend
    if case["kind"] == "weigh":
        return weigh
    if case["kind"] == "evict":
        return {"bytes": evict["bytes"] + 2 * new * (row + 8), "flops": 0}
    return {"bytes": attend["bytes"] + weigh["bytes"] + evict["bytes"], "flops": attend["flops"] + weigh["flops"]}


# ---- the definition in 64 bits, one KV head of one sequence at a time -----------------------------------
def exact(case, seed):
    if case["kind"] == "evict":
        return None                                         # nothing is computed: rows move
    s = prepare(case, seed)
    h, g, d, lengths, per_head = _dims(case)
    t, group, f64 = case["new"], h // g, torch.float64
    out = torch.zeros((len(lengths), t, h, d), dtype=f64, device=DEV)
    lse = torch.zeros((len(lengths), t, h), dtype=f64, device=DEV)
    weights = s["weights"].to(f64)
    for b in range(len(lengths)):
        for i in range(g):
            n = per_head[b][i]
            k = torch.cat([s["k"][b, i, :n], s["k_new"][b, :, i]]).to(f64)
            v = torch.cat([s["v"][b, i, :n], s["v_new"][b, :, i]]).to(f64)
            places = torch.cat([s["positions"][b, i, :n], s["new_positions"][b]]).to(f64)
            sees = torch.ones((t, n + t), dtype=torch.bool, device=DEV)
            if s["tree"] is None:
                sees[:, n:] = torch.ones((t, t), device=DEV).tril().bool()
            else:
                bits = torch.tensor([[m >> j & 1 for j in range(t)] for m in s["tree"][b].tolist()], device=DEV)
                sees[:, n:] = bits.bool()
            heads = slice(i * group, (i + 1) * group)
            x = torch.einsum("thd,nd->thn", s["q"][b, :, heads].to(f64), k) * s["scale"]
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            if case["distance"]:
                x = x - s["slopes"][heads].to(f64)[None, :, None] * (places[n:, None] - places)[:, None]
            x = x.masked_fill(~sees[:, None], -math.inf)
            p = torch.softmax(x, dim=-1)
            out[b, :, heads] = torch.einsum("thn,nd->thd", p, v)
            lse[b, :, heads] = torch.logsumexp(x, dim=-1)
            if case["kind"] == "decode":
                weights[b, i, n:n + t] = 0
                weights[b, i, :n + t] += p.sum(dim=(0, 1))
            if case["kind"] == "weigh":
                taken = [j for j in range(t) if s["accepted"][b].item() >> j & 1]
                weights[b, i, :n + t] += p[taken].sum(dim=(0, 1))
    if case["kind"] == "weigh":
        return {"weights": weights}
    if case["kind"] == "step":         # (which of the moved tokens' weights lie where is the selection's answer)
        return {"out": out, "lse": lse, "k": None, "v": None, "positions": None, "weights": None, "lengths": None}
    if case["kind"] == "tree":
        weights = None
    return {"out": out, "lse": lse, "k": None, "v": None, "positions": None, "weights": weights, "lengths": None}
