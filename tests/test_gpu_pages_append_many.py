"""GPU: appending to pages where there are so many blocks of slots that a thread block takes K and V of four heads (rows wait in shared memory), three
of them where no more are left: byte by byte against the statement, and the same as sequence after sequence by itself."""
import numpy as np
import pytest
import torch

from tests.pages_cases import Paged
from tests.test_gpu_pages_append import append, check_exact

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
B, T = 150, 34                                                     # four blocks a sequence


def many(device, shape, dtype, **more):
    rng = np.random.default_rng(11)
    p = Paged(device, shape, [int(n) for n in rng.integers(0, 40, B)], 16, spare=T, seed=12, dtype=dtype, **more)
    counts = rng.integers(0, T + 1, B)
    counts[:3] = 0, 1, T
    return p, counts.tolist()


@pytest.mark.parametrize("shape,dtype", [("small", BF), ("small", F32), ("single", BF), ("single", F32)])
def test_rows_and_scales(cuda_device, shape, dtype):
    p, counts = many(cuda_device, shape, dtype, token_major=dtype == BF)
    (k, _), (v, _) = p.noise(p.b, T, p.g, p.d, spread=3.0), p.noise(p.b, T, p.g, p.d)
    k[3, 2, 1, 3], v[4, 0, 0], v[5, 7, 1, 2] = float("inf"), float("nan"), -float("inf")
    append(p, k.to(p.device), v.to(p.device), counts=counts)
    check_exact(p, k, v, counts=counts)
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gathered_rows(cuda_device, dtype):
    p, counts = many(cuda_device, "small", dtype)
    (k, dk), (v, dv) = p.noise(p.b, 50, p.g, p.d), p.noise(p.b, 50, p.g, p.d)
    index = np.random.default_rng(13).integers(0, 50, (p.b, T))
    counts[7] = counts[8] = T
    index[7, 3], index[8, T - 1] = -1, 50
    append(p, dk, dv, index=index, counts=counts)
    check_exact(p, k, v, index=index, counts=counts)
    assert p.ctx.poll_device_status() == 1 and p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("single", BF), ("single", F32), ("small", F32)])
@pytest.mark.parametrize("more", [dict(), dict(part=0.5, interleaved=True), dict(part=0.625), dict(dim=6)])
def test_the_same_as_sequence_after_sequence(cuda_device, shape, dtype, more):
    from paper_2604_06746_b200 import binding
    (p, counts), (o, _) = many(cuda_device, shape, dtype), many(cuda_device, shape, dtype)
    rope = binding.Rope(more.get("dim", int(p.d * more.get("part", 1.0))), interleaved=more.get("interleaved", False))
    (_, k), (_, v) = p.noise(p.b, T, p.g, p.d, spread=2.0), p.noise(p.b, T, p.g, p.d)
    k[5, 1, 0, 1] = float("inf")
    positions = torch.arange(B * T, dtype=torch.int32, device=p.device).view(B, T) * 7 - 999
    c = torch.tensor(counts, dtype=torch.int32, device=p.device)
    p.ctx.append_pages(p.pages, k, v, positions=positions, rope=rope, counts=c)
    x = o.pages
    for b in range(B):
        one = binding.Pages(x.k, x.v, x.k_scales, x.v_scales, x.table[b:b + 1], x.lengths[b:b + 1])
        o.ctx.append_pages(one, k[b:b + 1], v[b:b + 1], positions=positions[b:b + 1], rope=rope, counts=c[b:b + 1])
    for got, want in zip(p.read(), o.read()):
        for which in "kv":
            assert np.array_equal(got[which], want[which])
    assert p.ctx.poll_device_status() == 0 and o.ctx.poll_device_status() == 0


@pytest.mark.parametrize("more", [dict(scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0), dict(interleaved=True)])
def test_codes_of_rotated_rows_to_the_last_bit(cuda_device, more):
    """17 million values of K: each has the code of the value in 64 bits, rounded to fp32 (those of which much cancels, where fp32 is off by more of
    what is left, are not compared)."""
    from oracle import pages_oracle as P
    from paper_2604_06746_b200 import binding
    n = 16384
    p = Paged(cuda_device, "llama", [0], 256, spare=n, seed=20)
    k, v = (torch.randn((1, n, p.g, p.d), generator=torch.Generator().manual_seed(i)).to(BF).to(p.device) for i in (21, 22))
    positions = torch.arange(n, dtype=torch.int32, device=p.device) * 61 + 5
    p.ctx.append_pages(p.pages, k, v, positions=positions, rope=binding.Rope(p.d, **more))
    inter = more.get("interleaved", False)
    f, amp = P.frequencies(p.d, 10000.0, **{x: y for x, y in more.items() if x != "interleaved"})
    angle = positions.double()[:, None, None] * torch.tensor(f, device=p.device, dtype=torch.float64)
    first, second = P.pairs(p.d, inter)
    a, b = k[0].double()[..., first], k[0].double()[..., second]
    y, size = torch.empty(n, p.g, p.d, dtype=torch.float64, device=p.device), torch.empty(n, p.g, p.d, dtype=torch.float64, device=p.device)
    y[..., first], y[..., second] = amp * (a * angle.cos() - b * angle.sin()), amp * (b * angle.cos() + a * angle.sin())
    size[..., first] = size[..., second] = amp * (a.abs() + b.abs())
    table = p.dtable[0, :n // 256].long()
    codes = p.pages.k[table].view(torch.uint8).transpose(1, 2).reshape(n, p.g, p.d)
    e = (p.pages.k_scales[table].view(torch.uint8).int() - 127).transpose(1, 2).reshape(n // 16, p.g).repeat_interleave(16, 0)[..., None]
    scaled = y.float() * torch.exp2(-e.float())
    want = scaled.to(torch.float8_e4m3fn).view(torch.uint8)
    # fp32 is off by 2^-23 of the parts' size at most, and what is off by 2^-20 of the value is looked at again; below 2^-6 codes are steps of one size
    compared = (y.abs() > size / 8) & (scaled.abs() > 2.0 ** -6)
    assert compared.float().mean() > 0.8 and (codes[compared] == want[compared]).all()
