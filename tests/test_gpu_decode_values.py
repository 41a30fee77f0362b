"""GPU tests of V that is not finite in new tokens whose K is finite: it reaches the columns that hold it, of the rows that see the
token, and nothing else."""
import numpy as np
import pytest
import torch

from tests.decode_cases import Problem

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def seen_by(p, b):
    """[t, t]: whether new token i sees new token u."""
    if p.tree_words is None:
        return np.tril(np.ones((p.t, p.t), dtype=bool))
    return np.array([[bool(m >> u & 1) for u in range(p.t)] for m in p.tree_words[b]])


def check(p):
    """Columns that are reached are not finite; the others are as if the values were not there (bounds as in
    decode_cases.Problem.check_attention)."""
    half = torch.finfo(p.dtype).eps / 2
    out, v_new = p.out.double().cpu().numpy(), p.v_new.double().numpy()
    for b in range(p.b):
        for g in range(p.g):
            reached = seen_by(p, b).astype(int) @ (~np.isfinite(v_new[b, :, g])).astype(int) > 0
            o, _, prob = p.reference(b, g)
            v = p.head(b, g)[2]
            v = np.where(np.isfinite(v), v, 0.0)
            o, mass = prob @ v, prob @ np.abs(v)
            tol = half * (mass * (p.dtype != F32) + np.abs(o)) + (2 * p.logit_error(b, g) + 2.0 ** -20) * mass + 1e-30
            got = out[b, :, g * p.group:(g + 1) * p.group]
            for i in range(p.t):
                bad = ~np.isfinite(got[i])
                assert np.array_equal(bad, np.broadcast_to(reached[i], bad.shape)), (b, g, i, np.argwhere(bad != reached[i])[:4])
                assert (np.abs(got[i] - o[i]) <= tol[i])[~bad].all(), (b, g, i)


def put(p, values):
    """values: (new token, column or None for all, value)."""
    for token, column, value in values:
        p.v_new[:, token, :, slice(None) if column is None else column] = value
    p.dv_new = p.v_new.to(p.device)


def repeat(p, times):
    from paper_2604_06746_b200 import binding
    ctx, cache = p.context(), p.cache()
    ws = ctx.attend_workspace(cache, p.t)
    first = None
    for _ in range(times):
        p.out.fill_(7)
        p.attend(ctx, cache, ws, k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
        if first is None:
            first = p.out.clone()
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.OK
    finite = torch.isfinite(first.float())
    assert torch.equal(torch.isfinite(p.out.float()), finite) and torch.equal(p.out[finite], first[finite])
    check(p)


# lengths: a CTA with two tiles of 128 keys whose second has the drafts (200), drafts across a tile's end (125, 60), only drafts (0),
# several tiles (900)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,tree", [(1, None), (2, "random"), (6, "random"), (6, None), (20, "random"), (50, "random")])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_v_that_is_not_finite(cuda_device, dtype, t, tree, value):
    p = Problem(cuda_device, "llama", [200, 125, 60, 0, 900, 250], t, dtype, seed=t, tree=tree)
    put(p, [(t // 2, 5, value), (t - 1, 77, value)] + ([(t // 3, None, value)] if t > 2 else []))
    repeat(p, 25)


@pytest.mark.parametrize("n", [122, 123, 127, 128, 129, 200, 250, 255])
def test_drafts_in_the_second_of_two_tiles(cuda_device, n):
    """Rows of one stream, tiles of two: eight KV heads of n keys and six drafts, many times over."""
    p = Problem(cuda_device, "llama", [n], 6, BF, seed=n, tree="random")
    put(p, [(0, 3, float("inf")), (5, 126, float("nan"))])
    repeat(p, 100)
