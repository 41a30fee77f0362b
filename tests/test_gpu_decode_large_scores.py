"""GPU tests of scores far from zero: a row's largest score weighs one whatever its size, in every kernel."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
KERNELS = [(1, F32), (7, F32), (1, BF), (4, BF), (20, BF), (32, BF), (64, BF)]


def problem(device, t, dtype, n, q0, k0, scale, tree, distance=False, d=64, h=8):
    """One sequence of n cached keys whose first column is k0 (others zero), queries with q0 there; v random."""
    from paper_2604_06746_b200 import binding
    gen = torch.Generator().manual_seed(t + n)
    ctx = binding.Context(h, 2, d, 8, 8, dtype, device)
    k, v = torch.zeros((1, 2, n + t, d), dtype=dtype), torch.randn((1, 2, n + t, d), generator=gen).to(dtype)
    k[0, :, :n, 0] = k0
    words = torch.zeros((2, 1, 2, n + t), dtype=torch.int32, device=device)
    dk, dv = k.to(device), v.clone().to(device)
    cache = binding.Cache(dk, dv, words[0], words[1].view(F32), torch.full((1, 2), n, dtype=torch.int32, device=device))
    q, new = torch.zeros((1, t, h, d), dtype=dtype), torch.zeros((1, t, 2, d), dtype=dtype)
    q[..., 0] = q0
    new[..., 0] = 1.0
    v_new = torch.randn((1, t, 2, d), generator=gen).to(dtype)
    out, lse = torch.zeros((1, t, h, d), dtype=dtype, device=device), torch.zeros((1, t, h), device=device)
    slopes = torch.zeros(h, device=device) if distance else None
    ctx.attend(cache, q.to(device), scale, out, ctx.attend_workspace(cache, t), k_new=new.to(device), v_new=v_new.to(device),
               positions=torch.zeros((1, t), dtype=torch.int32, device=device), lse=lse, slopes=slopes,
               tree=torch.tensor([tree], dtype=torch.int64, device=device))
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.OK
    return out.cpu(), lse.double().cpu().numpy(), v, v_new


@pytest.mark.parametrize("distance", [False, True])
@pytest.mark.parametrize("t,dtype", KERNELS)
def test_a_token_that_sees_only_itself(cuda_device, t, dtype, distance):
    """out is its V and lse its score: seven roundings of 2^-24 (log2(e), the scale's product with it, the score's, ln 2, the product, the
    sum, the result) are below 2^-21."""
    rng = np.random.default_rng(t)
    x = torch.from_numpy(10.0 ** rng.uniform(-3, 30, size=(1, t, 8)) * rng.choice([-1.0, 1.0], size=(1, t, 8))).to(dtype)
    tree = [(1 << i) - (1 << 64) * (i == 63) for i in range(t)]
    out, lse, _, v_new = problem(cuda_device, t, dtype, 0, x, 0.0, 0.3, tree, distance)
    want = x.double().numpy() * float(np.float32(0.3))
    assert (np.abs(lse - want) <= 2.0 ** -21 * np.abs(want)).all(), np.abs(lse / want - 1).max()
    assert torch.equal(out, v_new.repeat_interleave(4, dim=2))


@pytest.mark.parametrize("size", [1e3, 1e7, 1e10, 1e15, 1e30])
@pytest.mark.parametrize("t,dtype", KERNELS)
def test_one_key_of_many_is_above_all(cuda_device, t, dtype, size):
    """Keys 1 .. 127 times a large query: the last of them takes all the weight, a negative query's the first."""
    n = 400
    k0 = torch.from_numpy(np.random.default_rng(3).integers(2, 127, size=n).astype(np.float32)).to(dtype)
    k0[137], k0[291] = 1.0, 127.0
    q0 = torch.full((1, t, 8), size).to(dtype)
    q0[:, :, 1::2] *= -1
    out, lse, v, _ = problem(cuda_device, t, dtype, n, q0, k0, 1.0, [0] * t)
    q = q0.double().numpy()
    want = np.where(q > 0, q * 127, q)
    assert (np.abs(lse - want) <= 2.0 ** -21 * np.abs(want)).all()
    for h in range(8):
        assert torch.equal(out[0, :, h], v[0, h // 4, 291 if h % 2 == 0 else 137].expand(t, -1)), h
