"""GPU tests of the decoding operators together, as pipeline.Decode uses them behind a Prefill: every step is compared with the
statement in oracle/decode_oracle.py on the state that the step found.  Also: graphs that share a workspace, another stream, views
far apart, the smallest capacities."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from paper_2604_06746_b200 import synth
from tests.decode_cases import Problem, random_tree, signed

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LAYERS, BUDGET = 3, 150


def prompt(device, seq, shift):
    from paper_2604_06746_b200 import pipeline
    wl = synth.WORKLOADS["llama32k"].scaled(seq, n_layers=LAYERS, n_hubs=4, budgets=(BUDGET,))
    pl = synth.plan(wl)
    layers = [synth.make_layer(wl, pl, (l + shift) % LAYERS, device=device) for l in range(LAYERS)]
    pf = pipeline.Prefill(wl.n_layers, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, wl.window, wl.seq, BUDGET,
                          wl.struct_budget(), BF, device=device)
    pf.run(layers)
    return wl, layers, pf


class Mirror:
    """The cache on the host: read from the device before a step, moved on by the statement."""

    def __init__(self, cache):
        torch.cuda.synchronize()
        self.k, self.v = cache.k.double().cpu().numpy(), cache.v.double().cpu().numpy()
        self.pos, self.w, self.n = (t.cpu().numpy().copy() for t in (cache.positions, cache.weights, cache.lengths))

    def commit(self, b, g, t, count=None, path=None):
        n = int(self.n[b, g])
        slots = D.commit_slots(n, t, count, path)
        for a in (self.k, self.v, self.pos, self.w):
            a[b, g, n:n + len(slots)] = a[b, g, slots].copy()
        self.n[b, g] = n + len(slots)

    def evict(self, b, g, budget, recent):
        moves = D.evict_moves(self.w[b, g], self.pos[b, g], int(self.n[b, g]), budget, recent)
        for a in (self.k, self.v, self.pos, self.w):
            rows = [a[b, g, f].copy() for f, _ in moves]
            for (_, to), r in zip(moves, rows):
                a[b, g, to] = r
        self.n[b, g] = min(int(self.n[b, g]), budget)

    def same(self, other):
        assert np.array_equal(self.n, other.n)
        for b in range(self.n.shape[0]):
            for g in range(self.n.shape[1]):
                n = int(self.n[b, g])
                for x, y in ((self.k, other.k), (self.v, other.v), (self.pos, other.pos), (self.w, other.w)):
                    assert np.array_equal(x[b, g, :n], y[b, g, :n]), (b, g)


class Tokens:
    """New tokens of a layer."""

    def __init__(self, gen, wl, batch, t, positions, device):
        def noise(heads):
            return torch.randn((batch, t, heads, wl.head_dim), generator=gen).to(BF).to(device)
        self.q, self.k, self.v = noise(wl.n_q_heads), noise(wl.n_kv_heads), noise(wl.n_kv_heads)
        self.positions = positions
        self.out = torch.full_like(self.q, 7.0)


def check_layer(m, x, layer, batch, scale, out, masks=None):
    """out against the statement over mirror m (bounds as in decode_cases.Problem.check_attention); returns the probabilities
    [batch][KV head] and twice a logit's error."""
    half, result = torch.finfo(BF).eps / 2, []
    q, k, v = (t.double().cpu().numpy() for t in (x.q, x.k, x.v))
    got, groups, d = out.double().cpu().numpy(), k.shape[2], q.shape[3]
    G = q.shape[2] // groups
    for b in range(batch):
        result.append([])
        for g in range(groups):
            i, n = layer * batch + b, int(m.n[layer * batch + b, g])
            keys, vals = np.concatenate([m.k[i, g, :n], k[b, :, g]]), np.concatenate([m.v[i, g, :n], v[b, :, g]])
            pos = np.concatenate([m.pos[i, g, :n], x.positions[b].cpu().numpy()])
            qs = q[b, :, g * G:(g + 1) * G]
            o, _, p = D.attend(qs, keys, vals, pos, n, scale, masks=None if masks is None else masks[b])
            e = 2.0 ** -24 * (d + 8) * scale * float((np.abs(qs).max(axis=(0, 1)) @ np.abs(keys).T).max())
            mass = np.einsum("tgn,nd->tgd", p, np.abs(vals))
            tol = half * (mass + np.abs(o)) + (2 * e + 2.0 ** -20) * mass + 1e-30
            assert (np.abs(got[b, :, g * G:(g + 1) * G] - o) <= tol).all(), (layer, b, g)
            result[-1].append((p, 2 * e))
    return result


def check_weights(before, after, layer, batch, taken, probs, t, decay):
    """A weight: each added probability off by twice a logit's error and 2^-20, relative; decay and sums rounded in fp32."""
    for b in range(batch):
        for g, (p, e) in enumerate(probs[b]):
            i, n = layer * batch + b, int(before.n[layer * batch + b, g])
            add = p[taken[b]].sum(axis=(0, 1))
            old = np.concatenate([before.w[i, g, :n].astype(np.float64), np.zeros(t)])
            tol = (e + 2.0 ** -20) * add + 2.0 ** -22 * (old + add) + 1e-30
            assert (np.abs(after.w[i, g, :n + t] - (decay * old + add)) <= tol).all(), (layer, b, g)


@pytest.mark.parametrize("decay", [1.0, 0.75])
def test_decoding_behind_a_prefill(cuda_device, decay):
    """Two prompts are compacted, three single tokens follow, then a tree of drafted tokens of which some are accepted, then a
    single token again; the budget holds all along."""
    from paper_2604_06746_b200 import binding, pipeline
    dev, batch, t = cuda_device, 2, 6
    gen, rng = torch.Generator().manual_seed(3), np.random.default_rng(3)
    made = [prompt(dev, 1201, s) for s in range(batch)]
    wl = made[0][0]
    dec = pipeline.Decode(LAYERS, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, BUDGET + 2 + t, BF, batch=batch, budget=BUDGET + 2,
                          recent=16, max_new=t, decay=decay, device=dev)
    for b, (_, layers, pf) in enumerate(made):
        dec.take(pf, b)
    m = Mirror(dec.cache)
    assert (m.n == BUDGET).all()
    for b, (_, layers, pf) in enumerate(made):
        idx = pf.i_kv.cpu().numpy()
        for l in range(LAYERS):
            i = l * batch + b
            assert np.array_equal(m.k[i, :, :BUDGET], layers[l]["k"].double().cpu().numpy()[:, idx[l]])
            assert np.array_equal(m.v[i, :, :BUDGET], layers[l]["v"].double().cpu().numpy()[:, idx[l]])
            assert (m.pos[i, :, :BUDGET] == idx[l]).all()
            assert (m.w[i, :, :BUDGET] == pf.s_hist[l].cpu().numpy()[idx[l]]).all()
    scale, at = layers[0]["scale"], 1201

    def single():
        nonlocal at
        positions = torch.full((batch, 1), at, dtype=torch.int32, device=dev)
        xs = [Tokens(gen, wl, batch, 1, positions, dev) for _ in range(LAYERS)]
        before = Mirror(dec.cache)
        for l, x in enumerate(xs):
            dec.step(l, x.q, x.k, x.v, x.positions, scale, x.out)
        after = Mirror(dec.cache)
        for l, x in enumerate(xs):
            probs = check_layer(before, x, l, batch, scale, x.out)
            check_weights(before, after, l, batch, [[0]] * batch, probs, 1, decay)
        dec.advance()
        for i in range(LAYERS * batch):
            for g in range(wl.n_kv_heads):
                assert after.pos[i, g, after.n[i, g]] == at
                after.commit(i, g, 1)
                after.evict(i, g, dec.budget, dec.recent)
        Mirror(dec.cache).same(after)
        at += 1

    for _ in range(3):
        single()
    assert (Mirror(dec.cache).n == BUDGET + 2).all()
    masks = [random_tree(rng, t) for _ in range(batch)]
    depth = torch.tensor([[bin(x).count("1") - 1 for x in row] for row in masks], dtype=torch.int32, device=dev)
    tree = torch.tensor([[signed(x) for x in row] for row in masks], dtype=torch.int64, device=dev)
    leaf = [max(range(t), key=lambda i: bin(row[i]).count("1")) for row in masks]
    paths = [[u for u in range(t) if row[i] >> u & 1] for row, i in zip(masks, leaf)]
    xs = [Tokens(gen, wl, batch, t, depth + at, dev) for _ in range(LAYERS)]
    before = Mirror(dec.cache)
    for l, x in enumerate(xs):
        dec.verify(l, x.q, x.k, x.v, x.positions, scale, x.out, tree)
    probs = [check_layer(before, x, l, batch, scale, x.out, masks) for l, x in enumerate(xs)]
    counts = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=dev)
    path = torch.tensor([p + [0] * (t - len(p)) for p in paths], dtype=torch.int32, device=dev)
    keep, dec.budget = dec.budget, 0                       # (the weights are looked at before anything goes)
    dec.accept(counts, path)
    after = Mirror(dec.cache)
    want = Mirror(dec.cache)
    want.n = before.n.copy()
    for l, x in enumerate(xs):
        k, v = x.k.double().cpu().numpy(), x.v.double().cpu().numpy()
        for b in range(batch):
            for g in range(wl.n_kv_heads):
                i, n, c = l * batch + b, int(before.n[l * batch + b, g]), len(paths[b])
                assert after.n[i, g] == n + c
                assert np.array_equal(after.k[i, g, n:n + c], k[b, paths[b], g]) and np.array_equal(after.v[i, g, n:n + c], v[b, paths[b], g])
                assert np.array_equal(after.pos[i, g, n:n + c], x.positions[b].cpu().numpy()[paths[b]])
                p, e = probs[l][b][g]
                add = p[paths[b]].sum(axis=(0, 1))[list(range(n)) + [n + u for u in paths[b]]]
                old = np.concatenate([before.w[i, g, :n].astype(np.float64), np.zeros(c)])
                tol = (e + 2.0 ** -20) * add + 2.0 ** -22 * (old + add) + 1e-30
                assert (np.abs(after.w[i, g, :n + c] - (decay * old + add)) <= tol).all(), (l, b, g)
    dec.budget = keep
    single()
    assert (Mirror(dec.cache).n == dec.budget).all()
    torch.cuda.synchronize()
    assert dec.ctx.poll_device_status() == binding.OK


def test_refusals_of_the_run(cuda_device):
    from paper_2604_06746_b200 import pipeline
    wl, layers, pf = prompt(cuda_device, 1201, 0)
    make = lambda cap, **more: pipeline.Decode(LAYERS, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, cap, BF, device=cuda_device, **more)
    for cap, more in ((8, dict(max_new=65)), (8, dict(max_new=0)), (8, dict(budget=8)), (8, dict(budget=-1)), (8, dict(recent=-1))):
        with pytest.raises(ValueError):
            make(cap, **more)
    with pytest.raises(ValueError):
        make(BUDGET).take(pf)                              # no room behind it
    dec = make(BUDGET + 4, max_new=2)
    with pytest.raises(ValueError):
        dec.take(pf, 1)
    with pytest.raises(ValueError):
        pipeline.Decode(LAYERS + 1, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, BUDGET + 4, BF, device=cuda_device).take(pf)
    dec.take(pf)
    counts, path = torch.ones(1, dtype=torch.int32, device=cuda_device), torch.zeros((1, 2), dtype=torch.int32, device=cuda_device)
    with pytest.raises(ValueError):
        dec.accept(counts, path)                           # nothing was verified
    gen = torch.Generator().manual_seed(1)
    x = Tokens(gen, wl, 1, 3, torch.zeros((1, 3), dtype=torch.int32, device=cuda_device), cuda_device)
    with pytest.raises(ValueError):
        dec.verify(0, x.q, x.k, x.v, x.positions, 0.1, x.out)
    x = Tokens(gen, wl, 1, 2, torch.zeros((1, 2), dtype=torch.int32, device=cuda_device), cuda_device)
    dec.verify(0, x.q, x.k, x.v, x.positions, 0.1, x.out)
    with pytest.raises(ValueError):
        dec.accept(counts, path)                           # one layer of three


def far_apart(p):
    """The same cache in views whose sequences lie 2^31 bytes and more apart, heads 2^28."""
    b, g, cap, d = p.dk.shape
    s_head, s_batch = 2 ** 28 // p.dk.element_size(), 2 ** 31 // p.dk.element_size() * max(1, -(-g // 8)) + 64

    def view(x):
        buf = torch.empty((b - 1) * s_batch + (g - 1) * s_head + cap * d, dtype=x.dtype, device=x.device)
        y = buf.as_strided((b, g, cap, d), (s_batch, s_head, d, 1))
        y.copy_(x)
        return y
    p.dk, p.dv = view(p.dk), view(p.dv)


@pytest.mark.parametrize("shape,lengths,t,dtype,more", [
    ("small", [100, 65, 5], 1, BF, {}), ("llama", [70, 300, 1], 6, BF, dict(tree="random")), ("small", [40, 129, 0], 3, F32, {})])
def test_caches_beyond_32_bits(cuda_device, shape, lengths, t, dtype, more):
    p = Problem(cuda_device, shape, lengths, t, dtype, seed=6, **more)
    near_k = p.dk.clone()
    far_apart(p)
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, t)
    p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
    torch.cuda.synchronize()
    p.check_attention()
    for b in range(p.b):
        for g in range(p.g):
            n = int(p.n[b, g])
            assert torch.equal(p.dk[b, g, :n], near_k[b, g, :n]) and torch.equal(p.dk[b, g, n:n + t], p.dk_new[b, :, g])
            assert torch.equal(p.dv[b, g, n:n + t], p.dv_new[b, :, g])
    ctx.commit(cache, t)
    p.dw.nan_to_num_(0.0)
    ctx.evict(cache, 30, 4)
    torch.cuda.synchronize()
    for b in range(p.b):
        for g in range(p.g):
            n = int(p.n[b, g]) + t
            weights = np.concatenate([p.w[b, g, :n - t].numpy(), np.zeros(t, dtype=np.float32)])
            pos = np.concatenate([p.pos[b, g, :n - t].numpy(), p.new_pos[b].numpy()])
            k = torch.cat([near_k[b, g, :n - t], p.dk_new[b, :, g]])
            for f, to in D.evict_moves(weights, pos, n, 30, 4):
                assert torch.equal(p.dk[b, g, to], k[f]), (b, g, f, to)


@pytest.mark.parametrize("t,dtype", [(1, BF), (1, F32), (20, BF)])
def test_graphs_that_share_a_workspace(cuda_device, t, dtype):
    """Two problems, one workspace, a graph each, replayed in turn on one stream other than the current one."""
    ps = [Problem(cuda_device, "llama", lengths, t, dtype, seed=s, spare=30) for s, lengths in ((1, [300, 20]), (2, [5, 900]))]
    made = [(p, p.context(), p.cache()) for p in ps]
    ws = max((ctx.attend_workspace(c, t) for _, ctx, c in made), key=lambda w: w.numel())
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for p, ctx, cache in made:
            p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
            graphs.append(g)
        for p in ps:
            p.out.fill_(7)
            p.lse.fill_(7)
        for _ in range(4):
            for g in graphs:
                g.replay()
    torch.cuda.synchronize()
    for p in ps:
        p.check_attention()


def test_a_stream_that_is_named(cuda_device):
    p = Problem(cuda_device, "qwen", [500], 3, BF, seed=9)
    ctx, cache = p.context(), p.cache()
    ws, side = ctx.attend_workspace(cache, 3), torch.cuda.Stream()
    torch.cuda.synchronize()
    p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos, stream=side)
    side.synchronize()
    p.check_attention()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_cache_of_one_slot(cuda_device, dtype):
    """Capacity 1, length 0: the new token sees itself."""
    p = Problem(cuda_device, "small", [0, 0], 1, dtype, seed=4, spare=0)
    assert p.cap == 1
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, 1)
    p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos, accumulate=True)
    ctx.commit(cache, 1)
    ctx.evict(cache, 1, 0)
    torch.cuda.synchronize()
    p.check_attention()
    assert torch.equal(p.out, p.dv_new.repeat_interleave(p.group, dim=2)) and (p.dlen == 1).all()
    assert (p.dw - p.group).abs().max() <= p.group * 2.0 ** -20


@pytest.mark.parametrize("t,dtype", [(1, BF), (3, F32), (12, BF), (4, BF), (64, BF)])
def test_a_negative_scale_and_no_scale(cuda_device, t, dtype):
    for scale in (-0.125, 0.0):
        p = Problem(cuda_device, "llama", [200, 3], t, dtype, seed=4)
        p.scale = scale
        ctx, cache = p.context(), p.cache()
        p.attend(ctx, cache, ctx.attend_workspace(cache, t), k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
        torch.cuda.synchronize()
        p.scale = abs(scale)                               # (the bound's)
        p.reference = lambda b, g: _with_scale(p, b, g, scale)
        p.check_attention()


def _with_scale(p, b, g, scale):
    q, k, v, pos = p.head(b, g)
    return D.attend(q, k, v, pos, int(p.n[b, g]), scale, p.softcap, None, None)


@pytest.mark.parametrize("n,budget,spare", [(500, 499, 0), (9000, 8999, 0), (20001, 20000, 0), (17, 16, 9000), (2, 1, 0)])
def test_one_token_goes(cuda_device, n, budget, spare):
    """Ties (the last of the lowest goes), NaN, weights of both signs, recent ones only."""
    from tests.test_gpu_decode_cache import Store
    rng = np.random.default_rng(n)
    w = rng.choice(np.array([0.0, -0.0, 0.5, 0.25, np.inf, 1e-40, np.nan], dtype=np.float32), size=(1, 4, n + spare))
    w[0, 1] = 1.0
    w[0, 2] = np.nan
    w[0, 3] = -rng.random(n + spare)
    s = Store(cuda_device, [[n, n, n, n]], n + spare, seed=1, weights=w)
    s.evict(budget, 5)
    s.check()
    s = Store(cuda_device, [[n, budget]], n + spare, seed=2)
    s.evict(budget, n + spare)                             # all are recent
    s.check()
