"""GPU: rotary positions against their float64 statement: layouts, parts of a head, scalings, far and negative positions, strides; the
inverse as the gradient."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from tests.pages_cases import HALF, TURN

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SCALINGS = [{}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="bands", factor=8.0, original=8192, slow=1.0, fast=4.0),
            dict(scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0)]


def check(x, y, positions, dim, interleaved, inverse, more, base=10000.0):
    """x, y [batch, tokens, heads, d] on the host, positions [batch, tokens]."""
    f, amp = P.frequencies(dim, base, **more)
    a, b = P.pairs(dim, interleaved)
    for i in range(x.shape[0]):
        src = x[i].double().numpy()
        want = P.rotate(src, positions[i], f, amp, interleaved, inverse)
        size = np.zeros_like(want)
        size[..., a] = size[..., b] = amp * (np.abs(src[..., a]) + np.abs(src[..., b]))
        got = y[i].double().numpy()
        assert np.array_equal(got[..., dim:], src[..., dim:])
        assert (np.abs(got - want) <= 1.001 * HALF[x.dtype] * np.abs(want) + TURN[x.dtype] * size).all()


def noise(seed, dtype, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("dim", [2, 6, 16, 24, 32, 48, 62, 64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_head(cuda_device, dtype, d, dim, interleaved):
    from paper_2604_06746_b200 import binding
    if dim > d:
        pytest.skip("more than a head has")
    ctx = binding.Context(4, 2, d, 8, 8, dtype, cuda_device)
    x = noise(dim, dtype, 2, 19, 5, d)
    positions = np.random.default_rng(dim).integers(0, 1 << 17, (2, 19)).astype(np.int32)
    dx, out = x.to(cuda_device), torch.full(x.shape, float("nan"), dtype=dtype, device=cuda_device)
    pos, rope = torch.from_numpy(positions).to(cuda_device), binding.Rope(dim, interleaved=interleaved)
    for inverse in (False, True):
        ctx.rotate(dx, pos, rope, out=out, inverse=inverse)
        check(x, out.cpu(), positions, dim, interleaved, inverse, {})
    ctx.rotate(dx, pos, rope, inverse=True)                # in place
    assert torch.equal(dx, out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", SCALINGS)
def test_scalings_and_far_positions(cuda_device, dtype, more):
    """Positions to both ends of 32 bits.  (The statement's angles are off by 2^-53 of up to 2^31 radians there, 2^-22.)"""
    from paper_2604_06746_b200 import binding
    ctx = binding.Context(8, 2, 128, 8, 8, dtype, cuda_device)
    x = noise(1, dtype, 1, 40, 3, 128)
    positions = np.r_[np.arange(10), (1 << 20) + np.arange(10), -1 - np.arange(8), (1 << 23) - np.arange(8), -(1 << 21) - np.arange(4)].astype(np.int32)[None]
    rope = binding.Rope(128, 500000.0, **more)
    out = torch.empty(x.shape, dtype=dtype, device=cuda_device)
    ctx.rotate(x.to(cuda_device), torch.from_numpy(positions).to(cuda_device), rope, out=out)
    check(x, out.cpu(), positions, 128, False, False, more, 500000.0)
    ends = torch.tensor([-2 ** 31, 2 ** 31 - 1, -2 ** 31 + 1], dtype=torch.int32)
    ctx.rotate(x[:, :3].to(cuda_device), ends.to(cuda_device), rope, out=out[:, :3])
    turns = [[int(round(t * 2 ** 64)) * int(p) % 2 ** 64 / 2.0 ** 64 for t in rope.turns] for p in ends]
    y = x[0, :3].double().numpy()
    cos, sin = (rope.amplitude * f(2 * np.pi * np.array(turns))[:, None] for f in (np.cos, np.sin))
    want = np.concatenate([y[..., :64] * cos - y[..., 64:] * sin, y[..., 64:] * cos + y[..., :64] * sin], -1)
    # (turns as Python floats have 53 bits of 2^-64 steps: times 2^31 they are off by 2^-22 of a turn at most)
    size = rope.amplitude * (np.abs(y[..., :64]) + np.abs(y[..., 64:]))
    size = np.concatenate([size, size], -1)
    assert (np.abs(out[0, :3].double().cpu().numpy() - want) <= HALF[dtype] * np.abs(want) + (TURN[dtype] + 2 * np.pi * 2.0 ** -22) * size).all()


@pytest.mark.parametrize("tokens,heads,batch", [(1, 1, 1), (1, 32, 3), (33, 7, 2), (257, 9, 1), (3001, 2, 1), (5000, 17, 1)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_sizes_and_layouts(cuda_device, tokens, heads, batch, dtype):
    from paper_2604_06746_b200 import binding
    ctx = binding.Context(8, 2, 64, 8, 8, dtype, cuda_device)
    x = noise(tokens, dtype, batch, heads, tokens, 64)
    positions = (np.arange(tokens) + 7).astype(np.int32)
    pos, rope = torch.from_numpy(positions).to(cuda_device), binding.Rope(64)
    dx = x.to(cuda_device)
    # heads before tokens, one list of positions for all; then out inside a wider buffer
    wide = torch.full((batch, tokens, heads + 2, 72), 7.0, dtype=dtype, device=cuda_device)
    ctx.rotate(dx.transpose(1, 2), pos, rope, out=wide[:, :, 1:1 + heads, 8:])
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, -1] == 7).all() and (wide[..., :8] == 7).all()
    got = wide[:, :, 1:1 + heads, 8:].cpu()
    check(x.transpose(1, 2), got, np.stack([positions] * batch), 64, False, False, {})
    ctx.rotate(dx.transpose(1, 2), pos, rope)
    assert torch.equal(dx.transpose(1, 2).cpu(), got)
    # one head for all heads, one token for all tokens
    out = torch.empty((batch, tokens, heads, 64), dtype=dtype, device=cuda_device)
    ctx.rotate(x.to(cuda_device)[:, :1, :1].transpose(1, 2).expand(-1, tokens, heads, -1), pos, rope, out=out)
    check(x[:, :1, :1].transpose(1, 2).expand(-1, tokens, heads, -1), out.cpu(), np.stack([positions] * batch), 64, False, False, {})


def test_the_gradient(cuda_device):
    """<dy, rotate(x + h e) - rotate(x)> / h = the inverse's element: rotation is linear, so differences are exact but for rounding."""
    from paper_2604_06746_b200 import binding
    ctx = binding.Context(2, 2, 64, 8, 8, F32, cuda_device)
    rope = binding.Rope(48, interleaved=True, scaling="ramp", factor=32.0, original=4096, slow=1.0, fast=32.0)
    x, dy = (noise(s, F32, 1, 5, 2, 64).to(cuda_device) for s in (1, 2))
    pos = torch.tensor([3, 10, 99, 1000, 100000], dtype=torch.int32, device=cuda_device)
    dx, y, z = (torch.empty_like(x) for _ in range(3))
    ctx.rotate(dy, pos, rope, out=dx, inverse=True)
    ctx.rotate(x, pos, rope, out=y)
    for at in ((0, 0, 0, 0), (0, 2, 1, 17), (0, 4, 0, 46), (0, 4, 1, 60)):
        moved = x.clone()
        moved[at] += 1.0
        ctx.rotate(moved, pos, rope, out=z)
        # (y and z of size below 6 are rounded to 24 bits, and turned by rounded cosines: 6 2^-21.5 a term, two terms)
        assert abs(((z - y).double() * dy.double()).sum().item() - dx[at].item()) <= 2 * 2 * 6 * 2.0 ** -21.5 * dy.abs().max().item()
    f, amp = P.frequencies(48, 10000.0, "ramp", 32.0, 4096, 1.0, 32.0)
    want = P.rotate(dy[0].double().cpu().numpy(), pos.cpu().numpy(), f, amp, True, True)
    assert np.abs(dx[0].double().cpu().numpy() - want).max() <= TURN[F32] * 2 * amp * dy.abs().max().item()


def test_nothing_to_do_and_refusals(cuda_device):
    from paper_2604_06746_b200 import binding
    ctx = binding.Context(8, 2, 64, 8, 8, BF, cuda_device)
    x, pos, rope = noise(1, BF, 2, 9, 4, 64).to(cuda_device), torch.zeros(9, dtype=torch.int32, device=cuda_device), binding.Rope(64)
    for empty in (x[:0], x[:, :0], x[:, :, :0]):
        ctx.rotate(empty, pos[:empty.shape[1]], rope)
    run = ctx.rotate
    for bad in (lambda: run(x.float(), pos, rope), lambda: run(x[..., :32], pos, rope), lambda: run(x[0], pos, rope), lambda: run(x, pos.long(), rope),
                lambda: run(x, pos[:8], rope), lambda: run(x, pos.cpu(), rope), lambda: run(x.cpu(), pos, rope), lambda: run(x, pos, rope, out=x[:, :8]),
                lambda: run(x, pos, rope, out=x.float()), lambda: run(x.transpose(2, 3), pos, rope)):
        with pytest.raises(AssertionError):
            bad()
    odd = torch.empty((2, 9, 4, 68), dtype=BF, device=cuda_device)[..., :64]
    for bad in (lambda: run(odd, pos, rope), lambda: run(x[..., :], pos, binding.Rope(128)), lambda: run(x[:, :1].expand(-1, 9, -1, -1), pos, rope)):
        with pytest.raises(binding.StructKVError) as e:
            bad()
        assert e.value.status == binding.ERR_INVALID_ARG
