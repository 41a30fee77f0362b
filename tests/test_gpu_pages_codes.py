"""GPU: codes and scales of rotated keys are those of the values in 64 bits, rounded to fp32: every value of a long prompt, pairs of which little is
left, the largest value of a block beside a border between two scales, values at the end of fp32's range."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from tests.pages_cases import Paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
RAMP = dict(scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0)
SURE = 2.0 ** -39           # what two ways to the value in 64 bits may differ by, of its pair's parts: the kernel's polynomials are good to 2^-41


def rotated(k, positions, rope):
    """(values, what their parts add up to) of k [tokens, heads, d] at positions (numpy int64), in 64 bits; angles from the rope's own steps."""
    steps = np.array(rope._struct.step[:rope.dim // 2], dtype=np.uint64)
    turns = (positions.astype(np.uint64)[:, None] * steps).astype(np.int64).astype(np.float64) * (2 * np.pi * 2.0 ** -64)
    cos, sin = (torch.from_numpy(rope.amplitude * f(turns)).to(k.device)[:, None] for f in (np.cos, np.sin))
    first, second = (torch.from_numpy(x).to(k.device) for x in P.pairs(rope.dim, rope.interleaved))
    x = k.double()
    a, b, y, size = x[..., first], x[..., second], x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    size[..., first] = size[..., second] = rope.amplitude * (a.abs() + b.abs())
    return y, size


def exponents(y):
    """Of the scales of 16 rows each."""
    x = y.float()
    top = torch.where(x.isfinite(), x.abs(), 0.0).unflatten(0, (-1, 16)).amax(dim=(1, 3)).double()
    mantissa, e = torch.frexp(top)
    e = e - 9 + (mantissa > 0.875).to(e.dtype)
    return torch.where(top > 0, e, P.LOW).clamp_min(P.LOW)


def codes(y, e):
    x = y.float()
    c = (torch.where(x.isfinite(), x, float("nan")).double() * torch.exp2(-e.double())).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(c & 127 == 0, 0, c) & torch.where(c & 127 == 127, 127, 255).to(torch.uint8)      # (a zero has any sign, as NaN has)


def check(k, positions, dtype, rope, heads="llama", least=0.99):
    """k [tokens, heads, d] goes to an empty cache."""
    n = len(positions)
    p = Paged("cuda:0", heads, [0], 256, spare=n, seed=20, dtype=dtype)
    dk = k.to(dtype).to(p.device)
    p.ctx.append_pages(p.pages, dk[None], dk[None], positions=torch.from_numpy(positions.astype(np.int32)).to(p.device), rope=rope)
    table = p.dtable[0, :-(-n // 256)].long()
    got_e = (p.pages.k_scales[table].view(torch.uint8).int() - 127).transpose(1, 2).reshape(-1, p.g)[:n // 16]
    got = p.pages.k[table].view(torch.uint8).transpose(1, 2).reshape(-1, p.g, p.d)[:n]
    got = torch.where(got & 127 == 0, 0, got) & torch.where(got & 127 == 127, 127, 255).to(torch.uint8)
    y, size = rotated(dk, positions, rope)
    near = y.sign() * size * SURE
    e, sure = exponents(y), (exponents(y + near) == exponents(y - near)) & (exponents(y) == exponents(y + near))
    share, wrong = sure.double().mean().item(), (got_e != e) & sure
    told = wrong.sum().item(), got_e[wrong][:4].tolist(), e[wrong][:4].tolist()
    assert share >= least and told[0] == 0, told
    e = got_e.repeat_interleave(16, 0)[..., None]
    want = codes(y, e)
    sure = (codes(y + near, e) == want) & (codes(y - near, e) == want)
    share, wrong = sure.double().mean().item(), sure & (got != want)
    told = wrong.sum().item(), *(x[wrong][:4].tolist() for x in (y, size, got, want))
    assert share >= least and told[0] == 0, told
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", [RAMP, dict(interleaved=True), dict(dim=48)])
def test_every_value_of_a_long_prompt(cuda_device, dtype, more):
    from paper_2604_06746_b200 import binding
    n = 16384
    k = torch.randn((n, 8, 128), generator=torch.Generator().manual_seed(21))
    check(k, np.arange(n) * 61 + 5, dtype, binding.Rope(**({"dim": 128} | more)))


@pytest.mark.parametrize("more", [RAMP, dict(interleaved=True), dict(dim=44)])
@pytest.mark.parametrize("tokens", [160, 8000])                    # (one head a thread block, four)
def test_pairs_of_which_little_is_left(cuda_device, more, tokens):
    """b lies beside a cos / sin: what is left of a pair is a part of 2^-1 .. 2^-16 of it."""
    from paper_2604_06746_b200 import binding
    rope = binding.Rope(**({"dim": 128} | more))
    positions, rng = np.arange(tokens) * 3 + 1, np.random.default_rng(1)
    steps = np.array(rope._struct.step[:rope.dim // 2], dtype=np.uint64)
    angle = ((positions.astype(np.uint64)[:, None] * steps).astype(np.int64) * (2 * np.pi * 2.0 ** -64))[:, None]
    r, x = rng.uniform(0.5, 2.0, (tokens, 8, rope.dim // 2)), rng.standard_normal((tokens, 8, 128))
    left = 2.0 ** rng.uniform(-16, -1, r.shape) * rng.choice([-1, 1], r.shape)
    a, b = P.pairs(rope.dim, rope.interleaved)
    x[..., a], x[..., b] = r * np.sin(angle + left), r * np.cos(angle + left)
    check(torch.from_numpy(x), positions, F32, rope)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", [dict(), RAMP])
@pytest.mark.parametrize("heads", ["small", "llama"])              # (one head a thread block, four)
def test_the_largest_value_beside_a_border_of_scales(cuda_device, dtype, more, heads):
    """One pair a block, turned to a position where one of its values is 448 2^e within some steps of fp32."""
    from paper_2604_06746_b200 import binding
    d = 128 if heads == "llama" else 64
    rope = binding.Rope(d, **more)
    rng, step = np.random.default_rng(5), np.uint64(rope._struct.step[0])
    positions = np.arange(1 << 22, dtype=np.uint64)
    cos, sin = (rope.amplitude * f((positions * step).astype(np.int64) * (2 * np.pi * 2.0 ** -64)) for f in (np.cos, np.sin))
    rows, at = [], []
    for _ in range(12):                                            # (a pair reaches 448 at angles of its own)
        pair = torch.from_numpy(rng.uniform(300, 500, 2) / rope.amplitude).to(dtype).double().numpy() * rng.choice([-1, 1], 2)
        y = pair[0] * cos - pair[1] * sin
        close = np.abs(np.abs(y) - 448.0) < 448 * 2.0 ** -21
        close &= np.abs(pair[1] * cos + pair[0] * sin) < 440       # (the other value is smaller)
        rows += [pair * 2.0 ** rng.integers(-20, 20)] * int(close.sum())
        at += positions[close].tolist()
    assert len(at) > 20, len(at)
    least = max(len(at), 600 if heads == "llama" else 1)           # (so many blocks that a thread block has four heads)
    k, where = torch.zeros((16 * least, 8 if heads == "llama" else 2, d)), np.zeros(16 * least, dtype=np.int64)
    for i in range(least):
        k[16 * i + i % 16, :, 0], k[16 * i + i % 16, :, d // 2] = (float(x) for x in rows[i % len(at)])
        where[16 * i + i % 16] = at[i % len(at)]
    check(k, where, dtype, rope, heads)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", [RAMP, dict(), RAMP | dict(dim=44)])
@pytest.mark.parametrize("tokens", [48, 9600])
def test_values_at_the_end_of_the_range(cuda_device, dtype, more, tokens):
    """Pairs of some 2^127: parts that fp32 does not hold while what is left of them is a number, and numbers beside its largest."""
    from paper_2604_06746_b200 import binding
    rope = binding.Rope(**({"dim": 128} | more))
    rng, positions = np.random.default_rng(8), np.arange(tokens) * 5 + 3
    x = rng.uniform(0.3, 1.99, (tokens, 8, 128)) * rng.choice([-1, 1], (tokens, 8, 128)) * 2.0 ** 127
    x[::7] = rng.standard_normal(x[::7].shape)
    x[16:32] = rng.standard_normal((16, 8, 128))                   # (a block without any)
    # results within 2^-20 of the end
    steps = np.array(rope._struct.step[:rope.dim // 2], dtype=np.uint64)
    angle = (positions.astype(np.uint64)[:, None] * steps).astype(np.int64) * (2 * np.pi * 2.0 ** -64)
    a, b = P.pairs(rope.dim, rope.interleaved)
    end = (2.0 ** 128 - 2.0 ** 103) / rope.amplitude * (1 + rng.uniform(-1, 1, angle.shape) * 2.0 ** -20)
    x[::3, 5, a], x[::3, 5, b] = (end * np.cos(angle))[::3], (-end * np.sin(angle))[::3]
    check(torch.from_numpy(x), positions, dtype, rope, least=0.9)
