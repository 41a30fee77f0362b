"""GPU tests of capped scores: softcap tanh(x / softcap) is relatively exact whatever the cap, in every kernel."""
import numpy as np
import pytest
import torch

from tests.decode_cases import Problem

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# Relative error of a capped score.  tanh: 2^-20.5 (2^-21.4 over all numbers of 32 bits with exact reciprocals, and 2^-23 for the
# instruction's).  Then eight roundings of 2^-24: scale / softcap, its product with the score, softcap log2(e) and that constant, the
# product with tanh, ln 2 and the product with it, the result: 2^-21.  In all 2^-20.5 + 2^-21 < 1.25 x 2^-20.
REL = 1.25 * 2.0 ** -20


def scores_of(rng, n, dtype):
    x = np.concatenate([10.0 ** rng.uniform(-6, 3.5, size=n - 6), [1e30, 0.0, 1.0, 1e-30, 3e38, 1e-7]]) * rng.choice([-1.0, 1.0], size=n)
    return torch.from_numpy(x).to(torch.float32).to(dtype)


@pytest.mark.parametrize("softcap", [0.5, 5.0, 20.0, 50.0, 3000.0, 1e6])
@pytest.mark.parametrize("t,dtype", [(1, F32), (9, F32), (1, BF), (4, BF), (20, BF), (64, BF)])
def test_a_score_by_itself(cuda_device, t, dtype, softcap):
    """Every new token sees only itself, in an empty cache: lse is its score."""
    from paper_2604_06746_b200 import binding
    batch, h, d = 12, 8, 64
    rng = np.random.default_rng(t)
    ctx = binding.Context(h, 2, d, 8, 8, dtype, cuda_device)
    q = torch.zeros((batch, t, h, d), dtype=dtype)
    q[..., 11] = scores_of(rng, batch * t * h, dtype).view(batch, t, h)
    k_new = torch.zeros((batch, t, 2, d), dtype=dtype)
    k_new[..., 11] = 1.0
    k, v = (torch.zeros((batch, 2, t + 3, d), dtype=dtype, device=cuda_device) for _ in range(2))
    words = torch.zeros((2, batch, 2, t + 3), dtype=torch.int32, device=cuda_device)
    cache = binding.Cache(k, v, words[0], words[1].view(F32), torch.zeros((batch, 2), dtype=torch.int32, device=cuda_device))
    tree = torch.tensor([[(1 << i) - (1 << 64) * (i == 63) for i in range(t)]] * batch, dtype=torch.int64, device=cuda_device)
    out, lse = torch.zeros((batch, t, h, d), dtype=dtype, device=cuda_device), torch.zeros((batch, t, h), device=cuda_device)
    new = k_new.to(cuda_device)
    for scale in (1.0, -0.25):
        ctx.attend(cache, q.to(cuda_device), scale, out, ctx.attend_workspace(cache, t), k_new=new, v_new=new,
                   positions=torch.zeros((batch, t), dtype=torch.int32, device=cuda_device), tree=tree, softcap=softcap, lse=lse)
        torch.cuda.synchronize()
        assert ctx.poll_device_status() == binding.OK
        x = q[..., 11].double().numpy() * scale
        want, got = softcap * np.tanh(x / softcap), lse.double().cpu().numpy()
        assert (np.abs(got - want) <= REL * np.abs(want) + 1e-37).all(), np.abs(got / want - 1)[want != 0].max()


@pytest.mark.parametrize("t,dtype", [(1, F32), (3, F32), (1, BF), (20, BF), (40, BF)])
def test_scores_that_are_not_finite(cuda_device, t, dtype):
    """An infinite score is softcap; NaN stays NaN in the rows that see it."""
    from paper_2604_06746_b200 import binding
    p = Problem(cuda_device, "small", [70], t, dtype, seed=2, softcap=10.0)
    p.dq[:, 0, 0], p.dq[:, 0, 1] = 0.0, float("nan")
    p.dq[:, 0, 0, 0] = float("inf")
    p.dk[:, :, :, 0], p.dk_new[:, :, :, 0] = 1.0, -1.0
    ctx, cache = p.context(), p.cache()
    p.attend(ctx, cache, ctx.attend_workspace(cache, t), k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
    torch.cuda.synchronize()
    want = 10.0 + np.log(70.0 + np.exp(-20.0))             # KV head 0 has 70 keys of score 10 and its own of -10
    assert p.n[0, 0] == 70 and abs(p.lse[0, 0, 0].item() - want) <= 10 * REL + 2.0 ** -20 * (1 + want)
    assert torch.isfinite(p.out[0, 0, 0].float()).all() and torch.isnan(p.out[0, 0, 1].float()).all() and torch.isnan(p.lse[0, 0, 1])
    assert torch.isfinite(p.out[0, 0, 2:].float()).all() and torch.isfinite(p.out[0, 1:].float()).all()


@pytest.mark.parametrize("dtype,t", [(F32, 1), (F32, 6), (BF, 1), (BF, 16)])
@pytest.mark.parametrize("softcap", [20.0, 50.0, 1e4])
def test_attention_and_weights_of_capped_scores(cuda_device, dtype, t, softcap):
    """out, lse and weights with a logit's error that has no part of the cap's size: the dot product's (decode_cases) and REL |x|."""
    p = Problem(cuda_device, "qwen", [900, 63], t, dtype, seed=t, softcap=softcap, tree="random" if t > 1 else None)

    def logit_error(b, g):
        q, k, _, _ = p.head(b, g)
        dots = float((np.abs(q).max(axis=(0, 1)) @ np.abs(k).T).max()) * p.scale
        x = np.abs(np.einsum("tgd,nd->tgn", q, k)).max() * p.scale
        return 2.0 ** -24 * (p.d + 8) * dots + REL * float(x)
    p.logit_error = logit_error
    before = p.w.double().numpy()
    ctx, cache = p.context(), p.cache()
    p.attend(ctx, cache, ctx.attend_workspace(cache, t), k_new=p.dk_new, v_new=p.dv_new, positions=p.dnew_pos)
    torch.cuda.synchronize()
    p.check_attention()
    ctx.weigh(cache, p.dq, p.scale, p.lse, torch.full((p.b,), (1 << t) - 1, dtype=torch.int64, device=cuda_device), decay=0.5, **p.options())
    torch.cuda.synchronize()
    got = p.dw.double().cpu().numpy()
    for b in range(p.b):
        for g in range(p.g):
            n = p.n[b, g]
            gave = p.reference(b, g)[2].sum(axis=(0, 1))
            want = 0.5 * np.concatenate([before[b, g, :n], np.zeros(t)]) + gave
            # as many roundings as rows at most: sums of positive numbers, whatever their order
            tol = (2 * p.logit_error(b, g) + 2.0 ** -20) * gave + (2 + t * p.group) * 2.0 ** -24 * np.abs(want) + 1e-30
            assert (np.abs(got[b, g, :n + t] - want) <= tol).all(), (b, g, (np.abs(got[b, g, :n + t] - want) / tol).max())
