"""GPU: attention over a paged cache in 8 bits against its float64 statement: lengths, pages, head layouts, types, padded batches, pages and
slots full of NaN beside the tokens."""
import numpy as np
import pytest
import torch

from tests.pages_cases import Paged, check_attend

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def attend(p, q, counts=None, softcap=0.0, scale=None):
    t = q.shape[1]
    out = torch.full((p.b, t, p.h, p.d), float("nan"), dtype=p.dtype, device=p.device)
    lse = torch.full((p.b, t, p.h), float("nan"), device=p.device)
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=p.device)
    p.ctx.attend_pages(p.pages, q, p.d ** -0.5 if scale is None else scale, out, p.ctx.attend_pages_workspace(p.pages, t), counts=c,
                       softcap=softcap, lse=lse)
    return out, lse


def filled(p, t, counts=None):
    """New tokens' rows behind the lengths, by append_pages; the codes as the device has them then."""
    rows = [p.noise(p.b, t, p.g, p.d)[1] for _ in range(2)]
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=p.device)
    p.ctx.append_pages(p.pages, *rows, counts=c)
    return p.read()


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("qwen", BF), ("small", BF), ("small", F32), ("single", F32), ("wide", BF), ("wide", F32), ("many", BF)])
@pytest.mark.parametrize("lengths,page", [([0], 16), ([1, 15, 16, 17], 16), ([31, 0, 300, 63, 64, 65], 32), ([1500, 7], 64), ([2049, 999], 128),
                                          ([700, 3000], 256)])
def test_single_tokens(cuda_device, shape, dtype, lengths, page):
    p = Paged(cuda_device, shape, lengths, page, dtype=dtype, seed=len(lengths))
    codes, exps = filled(p, 1)
    q, dq = p.noise(p.b, 1, p.h, p.d, spread=2.0)
    check_attend(p, q, *attend(p, dq), None, p.d ** -0.5, codes=codes, exps=exps)
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("qwen", BF), ("small", F32), ("wide", BF), ("many", F32)])
@pytest.mark.parametrize("lengths,page,t", [([5, 0, 40], 16, 2), ([100, 333], 64, 3), ([64, 200, 1], 32, 5), ([1000], 128, 17), ([90, 5], 64, 64)])
@pytest.mark.parametrize("ragged", [False, True])
def test_several_tokens(cuda_device, shape, dtype, lengths, page, t, ragged):
    p = Paged(cuda_device, shape, lengths, page, dtype=dtype, seed=t)
    counts = [(t * (i + 1) // (len(lengths) + 1)) for i in range(len(lengths))] if ragged else None
    codes, exps = filled(p, t, counts)
    q, dq = p.noise(p.b, t, p.h, p.d)
    check_attend(p, q, *attend(p, dq, counts), counts, p.d ** -0.5, codes=codes, exps=exps)
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("small", F32)])
@pytest.mark.parametrize("softcap", [0.01, 30.0, 1e6])
def test_capped_scores(cuda_device, shape, dtype, softcap):
    p = Paged(cuda_device, shape, [200, 3], dtype=dtype, seed=4)
    codes, exps = filled(p, 3)
    q, dq = p.noise(p.b, 3, p.h, p.d, spread=8.0)
    check_attend(p, q, *attend(p, dq, softcap=softcap), None, p.d ** -0.5, softcap, codes, exps)


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("small", BF), ("small", F32)])
@pytest.mark.parametrize("spread", [1e-6, 1e-3, 30.0, 1e4])
def test_scores_and_queries_of_any_size(cuda_device, shape, dtype, spread):
    p = Paged(cuda_device, shape, [333, 40], dtype=dtype, seed=5)
    codes, exps = filled(p, 2)
    q, dq = p.noise(p.b, 2, p.h, p.d, spread=spread)
    scale = p.d ** -0.5 / max(1.0, spread / 4)
    check_attend(p, q, *attend(p, dq, scale=scale), None, scale, codes=codes, exps=exps)
    check_attend(p, q, *attend(p, dq, scale=-scale), None, -scale, codes=codes, exps=exps)


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("qwen", BF), ("small", F32)])
@pytest.mark.parametrize("spread", [3.0, 8.0])
def test_scales_far_apart(cuda_device, shape, dtype, spread):
    """Blocks of V whose magnitudes are many powers of two apart: each counts by what it weighs in the output."""
    p = Paged(cuda_device, shape, [700, 50], dtype=dtype, seed=6, v_spread=spread)
    codes, exps = filled(p, 1)
    q, dq = p.noise(p.b, 1, p.h, p.d, spread=3.0)
    check_attend(p, q, *attend(p, dq), None, p.d ** -0.5, codes=codes, exps=exps)


def test_other_layouts(cuda_device):
    """Token-major pages, queries inside a wider buffer, a table with gaps between its rows, pages that two sequences share."""
    p = Paged(cuda_device, "llama", [150, 200], 32, seed=7, token_major=True, shared=True)
    codes, exps = filled(p, 2)
    q, dq = p.noise(p.b, 2, p.h + 3, p.d)
    from paper_2604_06746_b200 import binding
    wide = torch.full((p.b, p.table.shape[1] + 5), -1, dtype=torch.int32, device=p.device)
    wide[:, :p.table.shape[1]] = p.dtable
    t = p.pages
    p.pages = binding.Pages(t.k, t.v, t.k_scales, t.v_scales, wide[:, :p.table.shape[1]], t.lengths)
    check_attend(p, q[:, :, 1:1 + p.h], *attend(p, dq[:, :, 1:1 + p.h]), None, p.d ** -0.5, codes=codes, exps=exps)
    # one query for all sequences
    check_attend(p, q[:1, :, :p.h].expand(2, -1, -1, -1), *attend(p, dq[:1, :, :p.h].expand(2, -1, -1, -1)), None, p.d ** -0.5,
                 codes=codes, exps=exps)


@pytest.mark.parametrize("shape,dtype,t", [("llama", BF, 1), ("llama", BF, 4), ("small", F32, 3), ("qwen", BF, 9)])
def test_nan_reaches_those_that_see_it(cuda_device, shape, dtype, t):
    p = Paged(cuda_device, shape, [37, 20], dtype=dtype, seed=8)
    k, v = (p.noise(p.b, t, p.g, p.d)[1] for _ in range(2))
    v[0, t - 1, 1, 5] = float("inf")                       # the last token's
    p.ctx.append_pages(p.pages, k, v)
    q, dq = p.noise(p.b, t, p.h, p.d)
    out, lse = attend(p, dq)
    sick = torch.zeros_like(out, dtype=torch.bool)
    sick[0, t - 1, p.group:2 * p.group, 5] = True
    assert torch.equal(out.isnan(), sick) and lse.isfinite().all()
    # in an old token it reaches all
    place = p.pages.v[p.table[0, 0], 1, 3]
    place.view(torch.uint8)[7] = 255
    out, lse = attend(p, dq)
    sick[0, :, p.group:2 * p.group, 7] = True
    assert torch.equal(out.isnan(), sick) and lse.isfinite().all()
    # in K it makes whole rows so
    p.pages.k[p.table[1, 0], 0, 19].view(torch.uint8)[0] = 127
    out, lse = attend(p, dq)
    assert out[1, :, :p.group].isnan().all() and lse[1, :, :p.group].isnan().all() and out[1, :, p.group:].isfinite().all()


def test_bad_pages_lengths_and_counts(cuda_device):
    """What the device finds wrong is said once by the status word; the other sequences have their results."""
    p = Paged(cuda_device, "llama", [100, 100, 100, 100, 100], 32, seed=9)
    codes, exps = filled(p, 2)
    q, dq = p.noise(p.b, 2, p.h, p.d)

    def fine(out, lse, only):                              # (cut otherwise than without the others' mistakes: other roundings)
        check_attend(p, q, out, lse, None, p.d ** -0.5, codes=codes, exps=exps, only=only)

    fine(*attend(p, dq), None)
    assert p.ctx.poll_device_status() == 0
    p.dlen[0], p.dlen[2] = -1, p.slots - 1
    out, lse = attend(p, dq, [2, 2, 2, 3, 2])
    assert p.ctx.poll_device_status() == 1 and p.ctx.poll_device_status() == 0
    for b in (0, 2, 3):
        assert (out[b] == 0).all() and (lse[b] == -float("inf")).all()
    fine(out, lse, [1, 4])
    # a page that is none: its slots are not seen
    p.dlen[:] = 100
    for bad in (-1, 1 << 30):
        p.dtable[1, 1] = bad
        out, lse = attend(p, dq)
        assert p.ctx.poll_device_status() == 1
        from oracle import pages_oracle as P
        k, v = (P.values(*p.head(x, 1, 3, codes, exps))[:102] for x in "kv")
        keep = np.r_[0:32, 64:102]
        want, want_lse, prob = P.attend(q[1, :, 12:16].double().numpy(), k[keep], v[keep], 68, p.d ** -0.5)
        size = prob @ np.abs(v[keep])
        assert (np.abs(out[1, :, 12:16].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * size).all()
        assert np.abs(lse[1, :, 12:16].cpu().numpy() - want_lse).max() < 1e-5
        fine(out, lse, [0, 2, 3, 4])
    p.dtable[1] = -1                                       # nothing is left
    out, lse = attend(p, dq)
    assert p.ctx.poll_device_status() == 1 and (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    # no rows at all
    p.dtable[1] = torch.from_numpy(p.table[1]).to(p.device)
    out, lse = attend(p, dq, [0] * 5)
    assert p.ctx.poll_device_status() == 0 and (out == 0).all() and (lse == -float("inf")).all()


def test_refusals(cuda_device):
    from paper_2604_06746_b200 import binding
    p = Paged(cuda_device, "small", [10, 20], seed=10)
    q = p.noise(2, 2, 8, 64)[1]
    out, ws = torch.empty_like(q), p.ctx.attend_pages_workspace(p.pages, 2)
    run = p.ctx.attend_pages
    for bad in (lambda: run(p.pages, q.float(), 1.0, out, ws), lambda: run(p.pages, q[:, :, :7], 1.0, out, ws),
                lambda: run(p.pages, q[:1], 1.0, out, ws), lambda: run(p.pages, q, 1.0, out[:, :1], ws), lambda: run(p.pages, q, 1.0, out.float(), ws),
                lambda: run(p.pages, q, 1.0, out, ws, counts=torch.ones(3, dtype=torch.int32, device=q.device)),
                lambda: run(p.pages, q, 1.0, out, ws, counts=torch.ones(2, dtype=torch.int64, device=q.device)),
                lambda: run(p.pages, q, 1.0, out, ws, counts=torch.ones(2, dtype=torch.int32)),
                lambda: run(p.pages, q, 1.0, out, ws, lse=torch.empty((2, 2, 7), device=q.device)), lambda: run(p.pages, q.cpu(), 1.0, out, ws),
                lambda: run(p.pages, q.transpose(2, 3).contiguous().transpose(2, 3), 1.0, out, ws),
                lambda: run(p.pages, q[:, :1].expand(-1, 65, -1, -1), 1.0, out[:, :1].expand(-1, 65, -1, -1).contiguous(), ws)):
        with pytest.raises(AssertionError):
            bad()
    for status, bad in ((binding.ERR_WORKSPACE, lambda: run(p.pages, q, 1.0, out, ws[:256])), (binding.ERR_WORKSPACE, lambda: run(p.pages, q, 1.0, out, ws[1:])),
                        (binding.ERR_INVALID_ARG, lambda: run(p.pages, q, float("inf"), out, ws)),
                        (binding.ERR_INVALID_ARG, lambda: run(p.pages, q, 1.0, out, ws, softcap=-1.0)),
                        (binding.ERR_INVALID_ARG, lambda: run(p.pages, q, 1.0, out, ws, softcap=float("nan"))),
                        (binding.ERR_INVALID_ARG, lambda: p.ctx.attend_pages_workspace(p.pages, 65)),
                        (binding.ERR_INVALID_ARG, lambda: p.ctx.attend_pages_workspace(p.pages, 0))):
        with pytest.raises(binding.StructKVError) as e:
            bad()
        assert e.value.status == status
    other = binding.Context(8, 4, 64, 8, 8, BF, cuda_device)
    with pytest.raises(AssertionError):
        other.attend_pages(p.pages, q, 1.0, out, ws)
