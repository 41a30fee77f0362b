"""GPU tests of V that is not finite in tokens whose probability is zero in fp32: whoever sees the token is told, in every kernel, for
new tokens and cached ones."""
import numpy as np
import pytest
import torch

from tests.decode_cases import Problem
from tests.test_gpu_decode_values import seen_by

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t", [1, 2, 4, 6, 20, 50])
def test_probability_zero(cuda_device, t, dtype, value):
    p = Problem(cuda_device, "llama", [200, 60, 700], t, dtype, seed=t, tree="random" if t > 1 else None)
    # scores along a column of its own: 0 for all keys, -2000 for the tokens in question
    p.q[..., 0], p.k[..., 0], p.k_new[..., 0] = 1.0, 0.0, 0.0
    low = -2000.0 / p.scale
    cached, new = [(0, 3), (1, 58), (2, 699)], t // 2     # (sequence, slot): at the start, beside the new tokens, the last one
    for b, slot in cached:
        for g in range(0, p.g, 2):
            slot_g = min(slot, int(p.n[b, g]) - 1)
            p.k[b, g, slot_g, 0], p.v[b, g, slot_g, 9] = low, value
    if t > 1:                                              # (a single token sees itself and, here, many others)
        p.k_new[:, new, 1::2, 0], p.v_new[:, new, 1::2, 77] = low, value
    p.dq, p.dk, p.dv, p.dk_new, p.dv_new = (x.to(cuda_device) for x in (p.q, p.k, p.v, p.k_new, p.v_new))
    ctx, cache = p.context(), p.cache()
    p.attend(ctx, cache, ctx.attend_workspace(cache, t), k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
    torch.cuda.synchronize()
    out = p.out.double().cpu().numpy()
    for b in range(p.b):
        see = seen_by(p, b)
        for g in range(p.g):
            bad = np.zeros((t, p.d), dtype=bool)
            bad[:, 9] = g % 2 == 0                         # every row sees the cached tokens
            bad[:, 77] = see[:, new] if g % 2 == 1 and t > 1 else False
            got = ~np.isfinite(out[b, :, g * p.group:(g + 1) * p.group])
            assert np.array_equal(got, np.broadcast_to(bad[:, None], got.shape)), (b, g, np.argwhere(got != bad[:, None])[:4])
