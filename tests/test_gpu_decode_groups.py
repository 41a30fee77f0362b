"""GPU tests of single tokens whose KV heads serve more query heads than a block of threads weighs at a time (128)."""
import numpy as np
import pytest
import torch

from tests import decode_cases
from tests.decode_cases import Problem

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
GROUPS = (4, 5, 127, 128, 129, 130, 132, 260)
decode_cases.SHAPES.update({"group %d" % g: (g, 1, 64) for g in GROUPS})
decode_cases.SHAPES["two of 132"] = (264, 2, 128)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape,lengths", [("group %d" % g, [300, 5]) for g in GROUPS] + [("two of 132", [65, 1200])])
def test_weights_of_many_heads(cuda_device, shape, lengths, dtype):
    from paper_2604_06746_b200 import binding
    p = Problem(cuda_device, shape, lengths, 1, dtype, seed=7)
    before, decay = p.w.double().numpy(), 0.5
    ctx, cache = p.context(), p.cache()
    p.attend(ctx, cache, ctx.attend_workspace(cache, 1), k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos, accumulate=True,
             decay=decay)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.OK
    p.check_attention()
    got = p.dw.double().cpu().numpy()
    for b in range(p.b):
        for g in range(p.g):
            n = p.n[b, g]
            gave = p.reference(b, g)[2].sum(axis=(0, 1))
            want = decay * np.concatenate([before[b, g, :n], [0.0]]) + gave
            # an added probability: twice a logit's error and 2^-20, relative; a sum of G of them in fp32 rounds G times at most,
            # decay and a sum for every 128 heads once more each
            tol = (2 * p.logit_error(b, g) + 2.0 ** -20 + p.group * 2.0 ** -24) * gave + (2 + p.group // 128) * 2.0 ** -24 * np.abs(want) + 1e-30
            assert (np.abs(got[b, g, :n + 1] - want) <= tol).all(), (b, g, (np.abs(got[b, g, :n + 1] - want) / tol).max())
