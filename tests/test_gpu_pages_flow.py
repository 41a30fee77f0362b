"""GPU tests of the paged cache's operators together, as pipeline.PagedDecode uses them: prompts of different lengths, steps with drafts that
are dropped, sequences that end and begin, behind a Prefill and by themselves; graphs, streams, shared workspaces, views beyond 32 bits."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from paper_2604_06746_b200 import synth
from tests.pages_cases import HALF, TURN, Paged, check_attend

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
L, H, G, D = 2, 8, 2, 64


class View:
    """One layer of a PagedDecode as check_attend takes it; codes and scales as the device has them now."""

    def __init__(self, dec, layer, batch):
        torch.cuda.synchronize()
        p = dec.layers[layer]
        self.b, self.h, self.g, self.d, self.group, self.dtype = batch, H, G, D, H // G, dec.ctx.dtype
        self.n, self.table = dec.lengths.tolist(), dec.table.cpu().numpy()
        self.codes = {"k": p.k.view(torch.uint8).cpu().numpy(), "v": p.v.view(torch.uint8).cpu().numpy()}
        self.exps = {x: s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127 for x, s in (("k", p.k_scales), ("v", p.v_scales))}

    head = Paged.head


def noise(gen, dtype, dev, *shape):
    return torch.randn(shape, generator=gen).to(dtype).to(dev)


@pytest.mark.parametrize("dtype,softcap", [(BF, 0.0), (F32, 0.0), (BF, 20.0)])
def test_a_batch_from_prompt_to_prompt(cuda_device, dtype, softcap):
    """Prompts kept by index with rotation, single tokens, drafts of which some stay, a sequence that ends and one that takes its pages; every
    step's attention and every row that stays are compared with the statement."""
    from paper_2604_06746_b200 import binding, pipeline
    rope = binding.Rope(48, interleaved=True, scaling="bands", factor=4.0, original=64, slow=1.0, fast=4.0)
    dec = pipeline.PagedDecode(L, H, G, D, pages=24, columns=8, dtype=dtype, batch=3, page_size=16, max_new=5, rope=rope, softcap=softcap,
                               device=cuda_device)
    gen, rng, f = torch.Generator().manual_seed(3), np.random.default_rng(3), None
    f, amp = P.frequencies(48, 10000.0, "bands", 4.0, 64, 1.0, 4.0)
    want = [[[[], []] for _ in range(3)] for _ in range(L)]   # rows [G, D] that stay, of K and V

    def turned(rows, positions):
        return P.rotate(rows.double().cpu().numpy(), np.asarray(positions), f, amp, True)

    def begin(sequence, n, kept):
        dec.reserve(sequence, kept + 20)
        index = np.sort(rng.permutation(n)[:kept]).astype(np.int32)
        positions = torch.arange(n, dtype=torch.int32, device=cuda_device)
        for l in range(L):
            k, v = noise(gen, dtype, cuda_device, G, n, D), noise(gen, dtype, cuda_device, G, n, D)
            dec.keep(l, sequence, k, v, torch.from_numpy(index).to(cuda_device), positions)
            want[l][sequence] = [list(turned(k.transpose(0, 1)[index.tolist()], index)), list(v.transpose(0, 1)[index.tolist()].double().cpu().numpy())]
        dec.advance(torch.tensor([kept if i == sequence else 0 for i in range(3)], dtype=torch.int32, device=cuda_device))

    def step(n_new, counts, stay):
        first = dec.lengths.cpu()[:, None] * 3
        positions = (first + torch.arange(n_new)).to(torch.int32).to(cuda_device)
        c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=cuda_device)
        for l in range(L):
            q, k, v = (noise(gen, dtype, cuda_device, 3, n_new, x, D) for x in (H, G, G))
            out, lse = torch.empty_like(q), torch.empty((3, n_new, H), device=cuda_device)
            dec.step(l, q, k, v, positions, D ** -0.5, out, counts=c, lse=lse)
            view = View(dec, l, 3)
            rotated = dec._q[:q.numel()].view_as(q).cpu()
            check_attend(view, rotated, out, lse, counts, D ** -0.5, softcap)
            for b in range(3):
                rows = turned(q[b], positions[b].cpu().numpy())
                assert (np.abs(rotated[b].double().numpy() - rows) <= 1.001 * HALF[dtype] * np.abs(rows) + TURN[dtype] * 8).all()
                m = stay[b] if isinstance(stay, list) else stay
                want[l][b][0] += list(turned(k[b], positions[b].cpu().numpy())[:m])
                want[l][b][1] += list(v[b].double().cpu().numpy()[:m])
        dec.advance(torch.tensor(stay, dtype=torch.int32, device=cuda_device) if isinstance(stay, list) else stay)

    def compare():
        for l in range(L):
            view = View(dec, l, 3)
            for b in range(3):
                for x, rows in zip("kv", want[l][b]):
                    rows = np.stack(rows)
                    assert len(rows) == view.n[b]
                    for g in range(G):
                        c, e = view.head(x, b, g)
                        got = P.values(c, e)[:len(rows)]
                        # a code is rounded when it is written and whenever its block's scale grows: half a step of 2^-4 or of the smallest
                        # numbers each, and a block of 16 grows at most a few times (the largest of 16 x 64 normal numbers: twice)
                        step_of = np.maximum(2.0 ** -4 * np.abs(rows[:, g]), 2.0 ** (np.repeat(e, 16)[:len(rows), None] - 10.0))
                        assert (np.abs(got - rows[:, g]) <= 3 * step_of + TURN[dtype] * 8).all(), (l, b, x, g)

    begin(0, 100, 37)
    begin(2, 30, 30)
    begin(1, 16, 1)
    step(1, None, 1)
    step(5, [5, 2, 0], [3, 2, 0])
    step(4, None, [0, 4, 1])
    compare()
    dec.release(0)
    assert dec.lengths.tolist()[0] == 0
    for l in range(L):
        want[l][0] = [[], []]
    begin(0, 90, 60)
    step(1, None, 1)
    compare()
    assert dec.ctx.poll_device_status() == 0
    with pytest.raises(ValueError):
        dec.reserve(1, 8 * 16 + 1)
    # a sequence without room: it stays, and the others go on
    dec.lengths[1] = 8 * 16 - 1
    q, k, v = (noise(gen, dtype, cuda_device, 3, 2, x, D) for x in (H, G, G))
    out = torch.empty_like(q)
    dec.step(0, q, k, v, torch.zeros((3, 2), dtype=torch.int32, device=cuda_device), 1.0, out)
    assert dec.ctx.poll_device_status() == 1 and (out[1] == 0).all() and out[0].abs().sum() > 0


def test_behind_a_prefill(cuda_device):
    from paper_2604_06746_b200 import binding, pipeline
    wl = synth.WORKLOADS["llama32k"].scaled(1500, n_layers=3, n_hubs=4, budgets=(150,))
    pl = synth.plan(wl)
    layers = [synth.make_layer(wl, pl, l, device=cuda_device) for l in range(3)]
    pf = pipeline.Prefill(3, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, wl.window, wl.seq, 150, wl.struct_budget(), BF, device=cuda_device)
    positions = torch.arange(wl.seq, dtype=torch.int32, device=cuda_device)
    rope = binding.Rope(wl.head_dim, 500000.0)
    for t in layers:
        before = t["k"].clone(), t["q_win"].clone()
        pf.rotate(t["q_win"], t["k"], rope, positions)
        f, _ = P.frequencies(wl.head_dim, 500000.0)
        for x, y, at in ((before[0], t["k"], np.arange(wl.seq)), (before[1], t["q_win"], np.arange(wl.seq - wl.window, wl.seq))):
            rows = P.rotate(x[1].double().cpu().numpy(), at, f)
            assert (np.abs(y[1].double().cpu().numpy() - rows) <= 1.001 * HALF[BF] * np.abs(rows) + TURN[BF] * 2 * x[1].abs().max().item()).all()
    pf.run(layers)
    dec = pipeline.PagedDecode(3, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, pages=8, columns=4, dtype=BF, rope=rope, device=cuda_device)
    with pytest.raises(ValueError):
        dec.take(pf)
    dec.reserve(0, 160)
    dec.take(pf)
    assert dec.lengths.tolist() == [150]
    gen = torch.Generator().manual_seed(1)
    for l in range(3):
        for g in range(wl.n_kv_heads):
            for x, rows in (("k", pf.k_out[l, g]), ("v", pf.v_out[l, g])):
                p = dec.layers[l]
                codes = torch.cat([getattr(p, x)[i, g] for i in dec.table[0, :3].tolist()])[:150].view(torch.uint8).cpu().numpy()
                exps = torch.cat([getattr(p, x + "_scales")[i, g] for i in dec.table[0, :3].tolist()]).view(torch.uint8).cpu().numpy().astype(np.int64) - 127
                want = P.append(np.zeros((160, wl.head_dim), dtype=np.uint8), [P.LOW] * 10, 0, rows.double().cpu().numpy())
                assert np.array_equal(codes, want[0][:150]) and np.array_equal(exps[:10], want[1])
        # a token attends over what was kept
        q, k, v = (noise(gen, BF, cuda_device, 1, 1, n, wl.head_dim) for n in (wl.n_q_heads, wl.n_kv_heads, wl.n_kv_heads))
        out = torch.empty_like(q)
        dec.step(l, q, k, v, torch.tensor([[wl.seq]], dtype=torch.int32, device=cuda_device), layers[l]["scale"], out)
        full = torch.cat([pf.k_out[l].double(), torch.from_numpy(P.rotate(k[0].double().cpu().numpy(), [wl.seq], f)).to(cuda_device).transpose(0, 1)], 1)
        vals = torch.cat([pf.v_out[l].double(), v[0].transpose(0, 1).double()], 1)
        rq = torch.from_numpy(P.rotate(q[0].double().cpu().numpy(), [wl.seq], f)).to(cuda_device)[0].view(wl.n_kv_heads, -1, wl.head_dim)
        exact = torch.softmax(torch.einsum("ghd,gnd->ghn", rq, full) * layers[l]["scale"], -1) @ vals
        # (what 8 bits cost: three significant bits a code, K's and V's)
        assert (out[0, 0].double().view_as(exact) - exact).norm() <= 0.1 * exact.norm()
    dec.advance(1)
    assert dec.ctx.poll_device_status() == 0


def paged(device, seed, t=1, shape="llama", lengths=(300, 20)):
    p = Paged(device, shape, list(lengths), 64, seed=seed)
    rows = [p.noise(p.b, t, p.g, p.d)[1] for _ in range(2)]
    q, dq = p.noise(p.b, t, p.h, p.d)
    out, lse = torch.zeros_like(dq), torch.zeros((p.b, t, p.h), device=device)
    return p, rows, q, dq, out, lse


@pytest.mark.parametrize("t", [1, 5, 20])
def test_graphs_that_share_a_workspace(cuda_device, t):
    """Two captured steps of different caches over one workspace, replayed in turn and with other inputs, beside eager calls."""
    a, b = paged(cuda_device, 1, t), paged(cuda_device, 2, t, lengths=(40, 1000, 3))
    ws = max((x[0].ctx.attend_pages_workspace(x[0].pages, t) for x in (a, b)), key=lambda w: w.numel())

    def run(x):
        p, rows, _, dq, out, lse = x
        p.ctx.append_pages(p.pages, *rows)
        p.ctx.attend_pages(p.pages, dq, p.d ** -0.5, out, ws, lse=lse)

    graphs = []
    for x in (a, b):
        run(x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(x)
        graphs.append(g)
    for turn in range(3):
        for g, x in zip(graphs, (a, b)):
            x[3].copy_(torch.randn(x[3].shape, generator=torch.Generator().manual_seed(turn)))
            x[4].fill_(float("nan"))
            g.replay()
            run(a if x is b else b)
        for x in (a, b):
            codes, exps = x[0].read()
            check_attend(x[0], x[3].cpu(), x[4], x[5], None, x[0].d ** -0.5, codes=codes, exps=exps)


def test_on_another_stream(cuda_device):
    p, rows, q, dq, out, lse = paged(cuda_device, 3, 3)
    ws, side = p.ctx.attend_pages_workspace(p.pages, 3), torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=cuda_device)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            busy = busy @ busy * 1e-2
        p.ctx.append_pages(p.pages, *rows)
    p.ctx.attend_pages(p.pages, dq, p.d ** -0.5, out, ws, lse=lse, stream=side)
    side.synchronize()
    codes, exps = p.read()
    check_attend(p, q, out, lse, None, p.d ** -0.5, codes=codes, exps=exps)


def test_the_same_inputs_give_the_same_bits(cuda_device):
    for t in (1, 4, 30):
        p, rows, q, dq, out, lse = paged(cuda_device, 4, t, lengths=(3000, 17, 900))
        ws, before = p.ctx.attend_pages_workspace(p.pages, t), p.read()
        p.ctx.append_pages(p.pages, *rows)
        first = None
        for _ in range(5):
            ws.fill_(255)
            out.fill_(float("nan"))
            p.ctx.attend_pages(p.pages, dq, p.d ** -0.5, out, ws, lse=lse)
            got = out.clone(), lse.clone()
            assert first is None or all(torch.equal(x, y) for x, y in zip(first, got))
            first = got


def test_pages_far_apart(cuda_device):
    """Pages 2^31 bytes and more from one another, as in a pool that many layers share."""
    from paper_2604_06746_b200 import binding
    p = Paged(cuda_device, "single", [30, 9], 16, seed=5, spare=2)
    stride, n = (1 << 31) + 4096, p.codes["k"].shape[0]
    if torch.cuda.mem_get_info()[0] < 2 * n * stride + (8 << 30):
        pytest.skip("not enough memory")
    far = []
    for x in "kv":
        store = torch.empty(n * stride, dtype=torch.uint8, device=cuda_device)
        view = store.as_strided((n, p.g, 16, p.d), (stride, 16 * p.d, p.d, 1))
        view.copy_(torch.from_numpy(p.codes[x]))
        far.append(view.view(torch.float8_e4m3fn))
    t = p.pages
    p.pages = binding.Pages(*far, t.k_scales, t.v_scales, t.table, t.lengths)
    rows = [p.noise(p.b, 1, p.g, p.d)[1] for _ in range(2)]
    p.ctx.append_pages(p.pages, *rows)
    q, dq = p.noise(p.b, 1, p.h, p.d)
    out, lse = torch.empty_like(dq), torch.empty((p.b, 1, p.h), device=cuda_device)
    p.ctx.attend_pages(p.pages, dq, p.d ** -0.5, out, p.ctx.attend_pages_workspace(p.pages, 1), lse=lse)
    codes, exps = p.read()
    check_attend(p, q, out, lse, None, p.d ** -0.5, codes=codes, exps=exps)


def test_large_scores_pick_their_key(cuda_device):
    """Scores of 2^26 and more bits, where a step of fp32 is whole bits: the key far above the others is what comes out."""
    for shape, dtype, t in (("llama", BF, 1), ("llama", BF, 4), ("llama", BF, 20), ("small", F32, 2)):
        p = Paged(cuda_device, shape, [200, 90], 64, dtype=dtype, seed=6)
        p.ctx.append_pages(p.pages, *[p.noise(p.b, t, p.g, p.d)[1] for _ in range(2)])
        codes, exps = p.read()
        q, dq = p.noise(p.b, t, p.h, p.d)
        for scale in (2.0 ** 22, -2.0 ** 27):
            out = torch.empty_like(dq)
            p.ctx.attend_pages(p.pages, dq, scale, out, p.ctx.attend_pages_workspace(p.pages, t))
            assert out.isfinite().all()
            for b in range(p.b):
                for g in range(p.g):
                    k, v = (P.values(*p.head(x, b, g, codes, exps)) for x in "kv")
                    for i in range(t):
                        n = p.n[b] + i + 1
                        for h in range(p.group):
                            x = k[:n] @ q[b, i, g * p.group + h].double().numpy() * np.sign(scale)
                            first, second = np.sort(x)[::-1][:2]
                            if first - second > 1e-3 * abs(first) + 1e-3:      # (far more than 2^-20 of a score)
                                assert np.abs(out[b, i, g * p.group + h].double().cpu().numpy() - v[np.argmax(x)]).max() <= 2.0 ** -8 * np.abs(v[np.argmax(x)]).max()
