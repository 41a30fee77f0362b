"""GPU tests of attention over a compacted cache (single tokens and trees of drafted ones) and of the weights it gathers,
against the 64-bit statement in oracle/decode_oracle.py."""
import numpy as np
import pytest
import torch

from tests.decode_cases import Problem, signed

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

CASES = [
    # shape, lengths, new tokens, dtype, more
    ("llama", [1024], 1, BF, {}),
    ("llama", [0, 1, 63, 64, 65, 700], 1, BF, {}),
    ("qwen", [333, 4097], 1, BF, dict(softcap=20.0)),
    ("small", [129, 2000], 1, BF, dict(distance=True)),
    ("wide", [511, 3], 1, BF, dict(softcap=5.0, distance=True)),
    ("single", [100], 1, BF, dict(token_major=True)),
    ("llama", [2048, 77], 8, BF, dict(tree="random")),
    ("qwen", [1000, 0, 64], 16, BF, dict(tree="random", softcap=30.0)),
    ("llama", [500], 64, BF, dict(tree="random")),
    ("llama", [61, 1], 63, BF, dict(tree="empty rows", token_major=True)),
    ("qwen", [0, 0], 5, BF, dict(tree="empty rows")),
    ("llama", [300, 20], 12, BF, dict()),
    ("wide", [200], 33, BF, dict(tree="random", distance=True)),
    ("single", [1000, 10], 64, BF, dict(tree="random", softcap=50.0, distance=True)),
    ("small", [2048, 777, 0], 1, F32, dict(distance=True)),
    ("small", [130], 7, F32, dict(tree="random", softcap=10.0)),
    ("llama", [300, 64], 3, F32, dict(tree="empty rows", token_major=True)),
    ("wide", [65], 1, F32, dict(softcap=3.0)),
    ("qwen", [17, 1], 64, F32, {}),
    ("llama", [900], 1, BF, dict(spread=12.0)),           # sharp rows: the running maximum grows late
    ("llama", [900], 17, BF, dict(spread=12.0, tree="random")),
    # several tiles and several short KV heads to a CTA
    ("qwen", [4096, 1001, 2500, 333, 4095, 64, 3777, 2049], 16, BF, dict(tree="random", softcap=30.0)),
    ("llama", [5000, 30, 128, 4097, 127, 200, 1, 6000], 9, BF, dict(tree="random", distance=True)),
    ("llama", [9000, 40, 70, 2000], 64, BF, dict(tree="random")),
    ("small", [100, 20000, 64, 65] * 8, 40, BF, dict(tree="random", softcap=9.0, distance=True)),
    ("single", [50] * 70 + [5000], 30, BF, dict(tree="empty rows")),
    ("llama", [3000, 50, 64, 10] * 6, 1, BF, {}),
    ("qwen", [20000, 9, 100], 2, BF, dict(tree="random")),
]


def run(p, **more):
    from paper_2604_06746_b200 import binding
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, p.t)
    p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos, **more)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.OK
    return ctx, cache, ws


def check_weights(p, b, g, before, got, decay, gave):
    """decay w + the probabilities of some rows: each off by the logit's error (twice) and 2^-20, and two more roundings."""
    n = p.n[b, g]
    want = decay * np.concatenate([before[b, g, :n], np.zeros(p.t)]) + gave
    tol = (2 * p.logit_error(b, g) + 2.0 ** -20) * gave + 2.0 ** -22 * np.abs(want) + 1e-30
    assert (np.abs(got[b, g, :n + p.t] - want) <= tol).all(), (b, g)


@pytest.mark.parametrize("shape,lengths,t,dtype,more", CASES)
def test_attention_matches_the_definition(cuda_device, shape, lengths, t, dtype, more):
    p = Problem(cuda_device, shape, lengths, t, dtype, seed=len(lengths) + t, **more)
    run(p)
    p.check_attention()
    # the rows that were appended, and nothing else
    for b in range(p.b):
        for g in range(p.g):
            n = p.n[b, g]
            assert torch.equal(p.dk[b, g, n:n + t].cpu(), p.k_new[b, :, g]) and torch.equal(p.dv[b, g, n:n + t].cpu(), p.v_new[b, :, g])
            assert torch.equal(p.dpos[b, g, n:n + t].cpu(), p.new_pos[b]) and (p.dw[b, g, n:n + t] == 0).all()
            assert torch.equal(p.dk[b, g, :n].cpu(), p.k[b, g, :n]) and torch.isnan(p.dk[b, g, n + t:].float()).all()
            assert torch.equal(p.dw[b, g, :n].cpu(), p.w[b, g, :n]) and torch.isnan(p.dw[b, g, n + t:]).all()
    assert torch.equal(p.dlen.cpu().long(), torch.from_numpy(p.n))


@pytest.mark.parametrize("decay", [1.0, 0.5])
@pytest.mark.parametrize("shape,lengths,dtype,more", [
    ("llama", [0, 5, 64, 3001], BF, {}), ("qwen", [700], BF, dict(softcap=15.0)), ("small", [100, 1025], F32, dict(distance=True)),
    ("wide", [400], BF, dict(token_major=True)), ("llama", [200, 30], F32, {}), ("llama", [300] * 9, BF, {})])
def test_single_tokens_gather_weights(cuda_device, shape, lengths, dtype, more, decay):
    p = Problem(cuda_device, shape, lengths, 1, dtype, seed=5, **more)
    before = p.w.double().numpy()
    run(p, accumulate=True, decay=decay)
    p.check_attention()
    got = p.dw.double().cpu().numpy()
    for b in range(p.b):
        for g in range(p.g):
            check_weights(p, b, g, before, got, decay, p.reference(b, g)[2].sum(axis=(0, 1)))
            assert np.isnan(got[b, g, p.n[b, g] + 1:]).all()


@pytest.mark.parametrize("shape,lengths,t,dtype,accepted,more", [
    ("llama", [2048, 1], 8, BF, [0b10110101, 1], dict(tree="random")),
    ("llama", [0, 300, 64], 64, BF, [(1 << 64) - 1, 0, 1 << 63], dict(tree="random")),
    ("qwen", [1000], 16, BF, [0b1010], dict(softcap=25.0, distance=True, token_major=True)),
    ("wide", [70], 9, BF, [0b111111111], dict(tree="empty rows")),
    ("qwen", [0], 5, BF, [0b11111], dict(tree="empty rows")),
    ("small", [130, 64], 7, F32, [0b1100110, 0b1], dict(tree="random", distance=True)),
    ("llama", [33], 4, F32, [0b1111], dict(softcap=8.0)),
])
def test_accepted_tokens_weigh(cuda_device, shape, lengths, t, dtype, accepted, more):
    p = Problem(cuda_device, shape, lengths, t, dtype, seed=t, **more)
    before = p.w.double().numpy()
    ctx, cache, _ = run(p)
    acc = torch.tensor([signed(a) for a in accepted], dtype=torch.int64, device=cuda_device)
    ctx.weigh(cache, p.dq, p.scale, p.lse, acc, decay=0.75, **p.options())
    torch.cuda.synchronize()
    got = p.dw.double().cpu().numpy()
    for b in range(p.b):
        rows = [i for i in range(t) if accepted[b] >> i & 1]
        for g in range(p.g):
            check_weights(p, b, g, before, got, 0.75, p.reference(b, g)[2][rows].sum(axis=(0, 1)))
            assert np.isnan(got[b, g, p.n[b, g] + t:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("t", [2, 6, 50])
def test_a_draft_that_is_not_finite_reaches_only_those_that_see_it(cuda_device, dtype, value, t):
    p = Problem(cuda_device, "llama", [70, 0, 640], t, dtype, seed=3, tree="random")
    bad = min(4, t - 1)
    for b in range(p.b):                                  # that token is nobody's ancestor
        p.tree_words[b] = [m & ~(1 << bad) if i != bad else m for i, m in enumerate(p.tree_words[b])]
    p.dtree = torch.tensor([[signed(m) for m in row] for row in p.tree_words], dtype=torch.int64, device=cuda_device)
    p.k_new[:, bad] = value
    p.v_new[:, bad] = value
    p.dk_new, p.dv_new = p.k_new.to(cuda_device), p.v_new.to(cuda_device)
    run(p)
    p.check_attention(rows=[i for i in range(t) if i != bad])
    assert not torch.isfinite(p.out[:, bad].float()).any()


def test_results_do_not_depend_on_the_run(cuda_device):
    p = Problem(cuda_device, "llama", [3000, 40, 999], 4, BF, seed=8, tree="random")
    ctx, cache, ws = run(p)
    first = (p.out.clone(), p.lse.clone())
    for _ in range(3):
        p.out.zero_()
        ws.fill_(255)
        p.attend(ctx, cache, ws)
        torch.cuda.synchronize()
        assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])


def test_captured_calls_follow_the_lengths(cuda_device):
    """A graph of one step (append, attend with weights, commit, evict), replayed: the lengths live on the device."""
    p = Problem(cuda_device, "llama", [200, 120], 1, BF, seed=2, spare=40)
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, 1)
    state = (p.dk, p.dv, p.dpos, p.dw, p.dlen, p.dnew_pos)
    start = [x.clone() for x in state]

    def restore():
        torch.cuda.synchronize()
        for x, y in zip(state, start):
            x.copy_(y)

    def step():
        p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos, accumulate=True)
        ctx.commit(cache, 1)
        ctx.evict(cache, 205, 16)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    restore()
    results = []
    for i in range(12):
        p.dnew_pos += 1
        g.replay()
        results.append((p.out.clone(), p.dw.clone(), p.dlen.clone()))
    restore()
    for i in range(12):
        p.dnew_pos += 1
        step()
        torch.cuda.synchronize()
        assert torch.equal(p.out, results[i][0]) and torch.equal(p.dlen, results[i][2])
        live = torch.arange(p.cap, device=cuda_device) < p.dlen[:, :, None]
        assert torch.equal(p.dw[live], results[i][1][live])
    assert p.dlen.max().item() == 205 and p.dlen.min().item() == 120 - 7 + 12


def test_bad_lengths_are_reported_and_left_alone(cuda_device):
    from paper_2604_06746_b200 import binding
    p = Problem(cuda_device, "llama", [100, 200], 2, BF, seed=4)
    good = p.n.copy()
    p.dlen[0, 3] = -1
    p.dlen[1, 0] = p.cap - 1
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, 2)
    p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.ERR_INVALID_ARG and ctx.poll_device_status() == binding.OK
    assert (p.out[0, :, 12:16] == 7).all() and (p.out[1, :, 0:4] == 7).all()
    assert torch.isnan(p.dk[0, 3, good[0, 3]:].float()).all()
    fine = Problem(cuda_device, "llama", [100, 200], 2, BF, seed=4)
    run(fine)
    p.out[0, :, 12:16], p.out[1, :, 0:4] = fine.out[0, :, 12:16], fine.out[1, :, 0:4]
    p.lse[0, :, 12:16], p.lse[1, :, 0:4] = fine.lse[0, :, 12:16], fine.lse[1, :, 0:4]
    p.check_attention()                                    # the others are as they should be
    p.dlen.fill_(-5)
    p.out.fill_(7)
    p.attend(ctx, cache, ws)
    torch.cuda.synchronize()
    assert (p.out == 7).all() and ctx.poll_device_status() == binding.ERR_INVALID_ARG


def test_refusals(cuda_device):
    from paper_2604_06746_b200 import binding
    p = Problem(cuda_device, "llama", [50], 3, BF, seed=1)
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, 3)
    with pytest.raises(binding.StructKVError, match="unsupported"):
        p.attend(ctx, cache, ws, accumulate=True)
    with pytest.raises(binding.StructKVError, match="workspace"):
        p.attend(ctx, cache, ws[:1024])
    with pytest.raises(binding.StructKVError, match="workspace"):
        p.attend(ctx, cache, ws[1:])
    for bad in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=1e-45), dict(decay=float("inf"))):
        with pytest.raises(binding.StructKVError, match="invalid"):
            p.attend(ctx, cache, ws, **bad)
    for bad in (dict(lse=p.lse[:, :2]), dict(tree=torch.zeros((1, 3), dtype=torch.int32, device=cuda_device)),
                dict(tree=torch.zeros((1, 3), dtype=torch.int64)), dict(slopes=torch.zeros(8, device=cuda_device)),
                dict(k_new=p.dk_new, v_new=p.dv_new, positions=None), dict(k_new=p.dk_new, v_new=p.dv_new[:, :2], positions=p.dnew_pos),
                dict(k_new=p.dk_new.float(), v_new=p.dv_new.float(), positions=p.dnew_pos)):
        with pytest.raises(AssertionError):
            p.attend(ctx, cache, ws, **bad)
    with pytest.raises(AssertionError):
        ctx.attend(cache, p.dq.transpose(2, 3).contiguous().transpose(2, 3), p.scale, p.out, ws)
    with pytest.raises(AssertionError):
        ctx.attend(cache, p.dq.cpu(), p.scale, p.out, ws)
    with pytest.raises(binding.StructKVError):
        ctx.attend_workspace(cache, 65)
    other = Problem(cuda_device, "small", [50], 3, BF, seed=1)
    with pytest.raises(AssertionError):
        other.context().attend(cache, p.dq, p.scale, p.out, ws)
    bare = binding.Cache(p.dk, p.dv, p.dpos, None, p.dlen)
    with pytest.raises(binding.StructKVError, match="invalid"):
        ctx.evict(bare, 10, 1)
    for f in (lambda: ctx.evict(cache, 0, 1), lambda: ctx.evict(cache, 10, -1), lambda: ctx.commit(cache, 0),
              lambda: ctx.commit(cache, p.cap + 1), lambda: ctx.commit(cache, 3, path=torch.zeros((1, 3), dtype=torch.int32, device=cuda_device))):
        with pytest.raises(binding.StructKVError, match="invalid"):
            f()
    odd = torch.zeros((1, 8, 60, 132), dtype=BF, device=cuda_device)[..., :128]   # rows of 264 bytes
    words = torch.zeros((2, 1, 8, 60), dtype=torch.int32, device=cuda_device)
    with pytest.raises(binding.StructKVError, match="invalid"):
        ctx.evict(binding.Cache(odd, odd, words[0], words[1].view(torch.float32), p.dlen), 10, 1)
    with pytest.raises(AssertionError):
        binding.Cache(p.dk, p.dv, p.dpos.long(), p.dw, p.dlen)
    with pytest.raises(AssertionError):
        binding.Cache(p.dk, p.dv[:, :, 1:], p.dpos, p.dw, p.dlen)
