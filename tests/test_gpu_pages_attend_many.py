"""GPU: attention over pages of many sequences (their runs are found 32 at a time), most of them short, some without tokens or without new ones."""
import numpy as np
import pytest
import torch

from tests.pages_cases import Paged, check_attend
from tests.test_gpu_pages_attend import attend, filled

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("shape,dtype,t", [("small", BF, 1), ("small", BF, 4), ("small", BF, 6), ("small", F32, 3), ("wide", BF, 1), ("single", F32, 1), ("qwen", BF, 3)])
@pytest.mark.parametrize("batch", [32, 33, 97])
def test_many_sequences(cuda_device, shape, dtype, t, batch):
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, 90, batch)
    lengths[rng.integers(0, batch, 3)] = 700, 333, 129
    lengths[rng.integers(0, batch, 5)] = 0
    counts = rng.integers(0, t + 1, batch)
    counts[[0, -1]] = 0, t
    p = Paged(cuda_device, shape, lengths.tolist(), 16, spare=t, dtype=dtype, seed=batch)
    codes, exps = filled(p, t, counts.tolist())
    q, dq = p.noise(p.b, t, p.h, p.d, spread=2.0)
    check_attend(p, q, *attend(p, dq, counts.tolist()), counts.tolist(), p.d ** -0.5, codes=codes, exps=exps)
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("t", [1, 6])
def test_nobody_has_a_new_token(cuda_device, t):
    p = Paged(cuda_device, "small", [5, 0, 70] * 15, 16, spare=t)
    codes, exps = p.read()
    q, dq = p.noise(p.b, t, p.h, p.d)
    out, lse = attend(p, dq, [0] * p.b)
    assert (out == 0).all() and (lse == -float("inf")).all() and p.ctx.poll_device_status() == 0


def test_sequences_that_are_refused_among_others(cuda_device):
    """Lengths and counts that cannot be, at the beginning, at the end and one after another: rows of nothing, and the others as by themselves."""
    p = Paged(cuda_device, "small", [50] * 40, 16, spare=6, seed=9)
    codes, exps = filled(p, 6)
    q, dq = p.noise(p.b, 6, p.h, p.d)
    good, good_lse = attend(p, dq)
    check_attend(p, q, good, good_lse, None, p.d ** -0.5, codes=codes, exps=exps)
    bad = [0, 1, 17, 31, 32, 33, 39]
    p.dlen[bad] = torch.tensor([-1, p.slots, p.slots - 5, 1 << 30, -5, 2147483647, -2147483648], dtype=torch.int32, device=p.device)
    out, lse = attend(p, dq)
    assert p.ctx.poll_device_status() == 1 and p.ctx.poll_device_status() == 0
    rest = [b for b in range(p.b) if b not in bad]
    assert (out[bad] == 0).all() and (lse[bad] == -float("inf")).all()
    # (cut elsewhere: the order of sums differs)
    assert (out[rest].double() - good[rest].double()).abs().max() <= 2.0 ** -7 * good.abs().max()
    view = Paged.__new__(Paged)
    view.__dict__ = dict(p.__dict__, b=len(rest), table=p.table[rest], n=[50] * len(rest))
    check_attend(view, q[rest], out[rest], lse[rest], None, p.d ** -0.5, codes=codes, exps=exps)
