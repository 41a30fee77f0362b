"""GPU: appending rotated rows in calls of any kind: parts of a head, pairings, scalings, positions to both ends of 32 bits, gathered and counted rows, blocks
that hold tokens already; codes and scales byte by byte against the float64 statement, then attention over them."""
import random

import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from tests.pages_cases import Paged, check_attend
from tests.test_gpu_pages_attend import attend
from tests.test_gpu_pages_codes import rotated

pytestmark = pytest.mark.gpu
SCALINGS = [{}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="bands", factor=8.0, original=8192, slow=1.0, fast=4.0),
            dict(scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0), dict(scaling="ramp", factor=3.7, original=4096, slow=1.0, fast=32.0)]


def plain(c):
    """Codes whose zeros and NaN have one sign."""
    return np.where((c & 127 == 0) | (c & 127 == 127), c & 127, c)


@pytest.mark.parametrize("seed", range(24))
def test_any_call(cuda_device, seed):
    from paper_2604_06746_b200 import binding
    r = random.Random(seed)
    shape, dtype = r.choice(["llama", "qwen", "small", "single", "wide"]), r.choice([torch.bfloat16, torch.float32])
    many = seed % 3 == 0                                           # (so many blocks that a thread block has four heads)
    batch, page = (r.randint(120, 160) if many else r.randint(1, 5)), r.choice([16, 32, 64, 256])
    lengths = [r.choice([0, r.randint(1, 40)]) for _ in range(batch)]
    t = r.randint(30, 40) if many else r.choice([1, r.randint(2, 70)])
    p = Paged(cuda_device, shape, lengths, page, spare=t, dtype=dtype, seed=seed, token_major=r.random() < 0.3)
    dim = r.choice([p.d, p.d, 2 * r.randint(1, p.d // 2), 16 * r.randint(1, p.d // 16)])
    rope = binding.Rope(dim, r.choice([10000.0, 500000.0]), interleaved=r.random() < 0.5, **(r.choice(SCALINGS) if dim > 2 else {}))
    source = t + r.randint(0, 20)
    index = p.rng.integers(0, source, (batch, t)).astype(np.int32) if r.random() < 0.5 else None       # (the same row twice and more, too)
    counts = [r.randint(0, t) for _ in range(batch)] if r.random() < 0.6 else None
    lo, hi = r.choice([(0, 1000), (10 ** 6, 10 ** 6 + 5000), (-(2 ** 31), 2 ** 31 - 1)])
    positions = p.rng.integers(lo, hi, (batch, source), endpoint=True)
    tokens = source if index is not None else t
    (k, dk), (v, dv) = (p.noise(batch, tokens, p.g, p.d, spread=10.0 ** r.uniform(-8, 8)) for _ in range(2))
    words = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=cuda_device)
    p.ctx.append_pages(p.pages, dk, dv, positions=words(positions[:, :tokens]), rope=rope, counts=words(counts), index=words(index))
    codes, exps = p.read()
    assert p.ctx.poll_device_status() == 0
    for b in range(batch):
        at, c = (np.arange(t) if index is None else index[b]), (t if counts is None else counts[b])
        y = rotated(dk[b], positions[b, :tokens], rope)[0].float().double().cpu().numpy()
        for x, rows in (("k", y), ("v", v[b].double().numpy())):
            for g in range(p.g):
                want_c, want_e = P.append(*p.head(x, b, g), p.n[b], rows[at[:c], g])
                got_c, got_e = p.head(x, b, g, codes, exps)
                last = -(-(p.n[b] + c) // 16)
                assert np.array_equal(got_e[:last], want_e[:last]), (b, x, g)
                assert np.array_equal(plain(got_c[:p.n[b] + c]), plain(want_c[:p.n[b] + c])), (b, x, g)
    if t <= 64 and not many:
        q, dq = p.noise(batch, t, p.h, p.d)
        scale = 1.0 / (p.d ** 0.5 * max(1.0, float(y.std())))
        check_attend(p, q, *attend(p, dq, counts, scale=scale), counts, scale, codes=codes, exps=exps)


@pytest.mark.parametrize("dtype,t", [(torch.bfloat16, 1), (torch.bfloat16, 4), (torch.bfloat16, 20), (torch.float32, 2)])
@pytest.mark.parametrize("zeros_first", [True, False])
def test_scales_of_values_as_far_apart_as_they_count(cuda_device, dtype, t, zeros_first):
    """Blocks of zeros, whose scale is 2^-40, among values of 2^84, whose scale is 2^76: every key has the same score and counts in every row's sum."""
    p = Paged(cuda_device, "llama", [0], 64, spare=400, dtype=dtype)
    n = 320
    zero = (torch.arange(n + t) // 16 % 2 == (0 if zeros_first else 1))[:, None, None]
    v = torch.where(zero, 0.0, 2.0 ** 84).expand(n + t, p.g, p.d).to(dtype).to(p.device)
    p.ctx.append_pages(p.pages, torch.zeros_like(v)[None], v[None])
    p.dlen += n
    _, dq = p.noise(1, t, p.h, p.d)
    out, lse = attend(p, dq)
    keys = n + 1 + torch.arange(t)
    share = torch.stack([(~zero[:m, 0, 0]).double().mean() for m in keys.tolist()])[:, None, None]
    # (weights are equal, and so are their roundings: what is left is the result's, of sums and of a logarithm)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20
    assert ((out[0].double().cpu() * 2.0 ** -84 - share).abs() <= 1.01 * half * share).all()
    assert ((lse[0].double().cpu() - keys.double().log()[:, None]).abs() <= 2.0 ** -18).all()
