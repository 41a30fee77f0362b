"""GPU: rotated values are off by no more than work in fp32 is, 2.54 2^-24 of their pair's parts and one rounding of the sum (with an amplitude that is
multiplied in, 2 2^-24 of the parts more), before they are rounded to their type: every result lies between the rounded ends of that interval."""
import numpy as np
import pytest
import torch

from tests.test_gpu_pages_codes import RAMP, rotated

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(x, got, positions, rope, dtype):
    """x, got [tokens, heads, d] on the device."""
    y, size = rotated(x, positions, rope)
    off = (2.54 if rope.amplitude == 1 else 4.54) * 2.0 ** -24 * size + 2.0 ** -24 * y.abs()
    lo, hi = ((y + s * off).to(F32).to(dtype) for s in (-1, 1))
    outside = ((got < lo) | (got > hi)).sum().item()
    assert outside == 0, (outside, (got.double() - y).abs().max().item())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", [dict(), RAMP, dict(interleaved=True), dict(dim=36)])
def test_every_value_of_a_long_prompt(cuda_device, dtype, more):
    from paper_2604_06746_b200 import binding
    rope, n = binding.Rope(**({"dim": 128} | more)), 32768
    ctx = binding.Context(8, 2, 128, 8, 8, dtype, cuda_device)
    x = torch.randn((n, 8, 128), generator=torch.Generator().manual_seed(3)).to(dtype).to(cuda_device)
    positions = np.arange(n) * 977 - (1 << 24)
    at, out = torch.from_numpy(positions.astype(np.int32)).to(cuda_device), torch.empty_like(x)
    ctx.rotate(x[None], at, rope, out=out[None])
    check(x, out, positions, rope, dtype)
    # pairs of which little is left
    steps = np.array(rope._struct.step[:rope.dim // 2], dtype=np.uint64)
    angle = torch.from_numpy((positions.astype(np.uint64)[:, None] * steps).astype(np.int64) * (2 * np.pi * 2.0 ** -64)).to(cuda_device)[:, None]
    half = rope.dim // 2
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if rope.interleaved else (slice(0, half), slice(half, 2 * half))
    r = x[..., first].double()
    x[..., first], x[..., second] = (r * angle.sin()).to(dtype), (r * angle.cos()).to(dtype)
    ctx.rotate(x[None], at, rope, out=out[None])
    check(x, out, positions, rope, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_that_come_along(cuda_device, dtype):
    from paper_2604_06746_b200 import binding
    from tests.pages_cases import Paged
    n = 600
    p, rope = Paged(cuda_device, "llama", [0], 64, spare=n, dtype=dtype), binding.Rope(128, **RAMP)
    rows, dq = [p.noise(1, n, p.g, p.d)[1] for _ in range(2)], p.noise(1, n, p.h, p.d)[1]
    positions, out = np.arange(n) * 13 + 100000, torch.empty_like(dq)
    p.ctx.append_pages(p.pages, *rows, positions=torch.from_numpy(positions.astype(np.int32)).to(cuda_device), rope=rope, q=dq, q_out=out)
    check(dq[0], out[0], positions, rope, dtype)
