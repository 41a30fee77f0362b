"""GPU: attention over a paged cache with more than 16 rows of a KV head, whose tiles of 64 keys go through the tensor cores' own memory: up to
64 rows stand twice in a tile, blocks of 128 otherwise; items of one tile and of many; every size of scores and scales."""
import pytest
import torch

from tests.pages_cases import Paged, check_attend
from tests.test_gpu_pages_attend import attend, filled

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
LENGTHS = [0, 30, 64, 65, 128, 129, 1000]


@pytest.mark.parametrize("shape,t", [("llama", 5), ("llama", 9), ("llama", 16), ("llama", 17), ("small", 5), ("small", 13), ("small", 33), ("wide", 1), ("wide", 2),
                                     ("wide", 3), ("many", 3), ("qwen", 19)])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_items_of_one_tile_and_of_many(cuda_device, shape, t, softcap):
    p = Paged(cuda_device, shape, LENGTHS, 32, seed=t)
    codes, exps = filled(p, t)
    q, dq = p.noise(p.b, t, p.h, p.d, spread=2.0)
    check_attend(p, q, *attend(p, dq, softcap=softcap), None, p.d ** -0.5, softcap, codes, exps)


@pytest.mark.parametrize("shape,t", [("llama", 7), ("small", 16), ("llama", 30)])
@pytest.mark.parametrize("spread", [1e-6, 30.0, 1e4])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(cuda_device, shape, t, spread, sign):
    p = Paged(cuda_device, shape, [333, 40, 5000], dtype=BF, seed=t)
    codes, exps = filled(p, t)
    q, dq = p.noise(p.b, t, p.h, p.d, spread=spread)
    scale = sign * p.d ** -0.5 / max(1.0, spread / 4)
    check_attend(p, q, *attend(p, dq, scale=scale), None, scale, codes=codes, exps=exps)


@pytest.mark.parametrize("shape,t", [("llama", 7), ("small", 16), ("llama", 30)])
@pytest.mark.parametrize("spread", [3.0, 8.0])
def test_scales_far_apart(cuda_device, shape, t, spread):
    p = Paged(cuda_device, shape, [2500, 50], dtype=BF, seed=6, v_spread=spread)
    codes, exps = filled(p, t)
    q, dq = p.noise(p.b, t, p.h, p.d, spread=3.0)
    check_attend(p, q, *attend(p, dq), None, p.d ** -0.5, codes=codes, exps=exps)


def test_calls_at_once_on_two_streams(cuda_device):
    """Caches of their own, workspaces of their own: what they give is what they give one after another, every time."""
    calls = []
    for seed, (shape, t) in enumerate([("llama", 16), ("llama", 1), ("small", 40), ("qwen", 5)]):
        p = Paged(cuda_device, shape, [2000, 70, 900], seed=seed)
        filled(p, t)
        dq = p.noise(p.b, t, p.h, p.d)[1]
        calls.append((p, dq, p.ctx.attend_pages_workspace(p.pages, t), attend(p, dq)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(cuda_device) for _ in calls]
    for _ in range(10):
        outs = []
        for (p, dq, ws, _), stream in zip(calls, streams):
            out, lse = torch.empty_like(dq), torch.empty(dq.shape[:3], device=p.device)
            stream.wait_stream(torch.cuda.current_stream())
            for _ in range(3):
                p.ctx.attend_pages(p.pages, dq, p.d ** -0.5, out, ws, lse=lse, stream=stream)
            outs.append((out, lse))
        torch.cuda.synchronize()
        for (p, _, _, want), got in zip(calls, outs):
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(p.ctx.poll_device_status() == 0 for p, *_ in calls)
