"""GPU tests of caps so large that scale / softcap has few bits left in fp32: scores are as exact as under any other cap."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("softcap", [1e25, 1e33, 1e36, 1e38, 3.4e38])
@pytest.mark.parametrize("t,dtype", [(1, F32), (1, BF), (20, BF)])
def test_a_score_by_itself(cuda_device, t, dtype, softcap):
    """Every new token sees only itself, in an empty cache: lse is its score.  Relative error as of any capped score: 1.25 x 2^-20
    (test_gpu_decode_softcap.py)."""
    from paper_2604_06746_b200 import binding
    batch, h, d, scale = 6, 8, 64, 0.125
    rng = np.random.default_rng(t)
    ctx = binding.Context(h, 2, d, 8, 8, dtype, cuda_device)
    q = torch.zeros((batch, t, h, d), dtype=dtype)
    q[..., 7] = torch.from_numpy(10.0 ** rng.uniform(-4, 15, size=(batch, t, h)) * rng.choice([-1.0, 1.0], size=(batch, t, h))).to(dtype)
    new = torch.zeros((batch, t, 2, d), dtype=dtype)
    new[..., 7] = 1.0
    new = new.to(cuda_device)
    k, v = (torch.zeros((batch, 2, t + 1, d), dtype=dtype, device=cuda_device) for _ in range(2))
    words = torch.zeros((2, batch, 2, t + 1), dtype=torch.int32, device=cuda_device)
    cache = binding.Cache(k, v, words[0], words[1].view(F32), torch.zeros((batch, 2), dtype=torch.int32, device=cuda_device))
    tree = torch.tensor([[1 << i for i in range(t)]] * batch, dtype=torch.int64, device=cuda_device)
    out, lse = torch.zeros((batch, t, h, d), dtype=dtype, device=cuda_device), torch.zeros((batch, t, h), device=cuda_device)
    ctx.attend(cache, q.to(cuda_device), scale, out, ctx.attend_workspace(cache, t), k_new=new, v_new=new,
               positions=torch.zeros((batch, t), dtype=torch.int32, device=cuda_device), tree=tree, softcap=softcap, lse=lse)
    torch.cuda.synchronize()
    x = q[..., 7].double().numpy() * scale
    cap = float(np.float32(softcap))
    want, got = cap * np.tanh(x / cap), lse.double().cpu().numpy()
    assert (np.abs(got - want) <= 1.25 * 2.0 ** -20 * np.abs(want)).all(), np.abs(got / want - 1).max()
