"""GPU: a pipeline.PagedDecode whose batch is not full: places without a sequence, sequences that begin where others were, that are full or whose
next page is not theirs yet."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, L, H, G, D, PAGE = torch.bfloat16, 2, 8, 2, 64, 16


def noise(seed, dev, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF).to(dev)


def decode(dev, batch, pages=12, columns=4, max_new=3):
    from paper_2604_06746_b200 import pipeline
    return pipeline.PagedDecode(L, H, G, D, pages=pages, columns=columns, dtype=BF, batch=batch, page_size=PAGE, max_new=max_new, device=dev)


def keep(dec, sequence, n, seed):
    for l in range(L):
        dec.keep(l, sequence, noise(seed + l, dec.table.device, G, n, D), noise(seed + 10 + l, dec.table.device, G, n, D))
    dec.advance(torch.tensor([n if b == sequence else 0 for b in range(dec.B)], dtype=torch.int32, device=dec.table.device))


def step(dec, n, seed, counts=None):
    """Outputs of all layers; a sequence's rows do not depend on the batch."""
    dev, outs = dec.table.device, []
    for l in range(L):
        q, k, v = (noise(seed + 100 * l + i, dev, 1, n, h, D).expand(dec.B, -1, -1, -1) for i, h in enumerate((H, G, G)))
        out = torch.empty((dec.B, n, H, D), dtype=BF, device=dev)
        dec.step(l, q, k, v, None, D ** -0.5, out, counts=counts)
        outs.append(out)
    return torch.stack(outs)


def near(a, b):
    """The same attention, cut otherwise: sums in another order, each result rounded to bf16 (a step is 2^-7 of it at most)."""
    return a.isfinite().all() and (a.double() - b.double()).abs().max() <= 2.0 ** -7 * b.abs().max()


def test_a_place_that_others_passed(cuda_device):
    """Sequence 1 begins after others advanced by a number, sequence 0 anew after its end: both as in a cache of their own."""
    dec = decode(cuda_device, 3)
    for p in dec.layers:                                            # (what nobody wrote is NaN)
        p.k.view(torch.uint8).fill_(127)
        p.v.view(torch.uint8).fill_(127)
    dec.reserve(0, 40)
    keep(dec, 0, 30, 1)
    for i in range(5):
        step(dec, 1, 50 + i)
        dec.advance(1)
    assert dec.lengths.tolist() == [35, 0, 0]
    dec.reserve(1, 40)
    keep(dec, 1, 20, 2)
    dec.release(0)
    step(dec, 1, 60)
    dec.advance(1)
    dec.reserve(0, 40)
    keep(dec, 0, 10, 3)
    assert dec.lengths.tolist() == [10, 21, 0]
    got = step(dec, 2, 70)
    own = decode(cuda_device, 1)
    own.reserve(0, 40)
    keep(own, 0, 10, 3)
    assert near(got[:, 0], step(own, 2, 70)[:, 0])
    own.release(0)
    own.reserve(0, 40)
    keep(own, 0, 20, 2)
    step(own, 1, 60)
    own.advance(1)
    assert own.lengths.tolist() == [21] and near(got[:, 1], step(own, 2, 70)[:, 0])


def test_no_room_in_a_captured_step(cuda_device):
    """A step and its advance as a graph: replayed until the pages end, sequences stop one after another where they are full."""
    from paper_2604_06746_b200 import binding
    dec = decode(cuda_device, 3)
    dec.reserve(0, 64)
    dec.reserve(1, 32)
    keep(dec, 0, 60, 1)
    keep(dec, 1, 25, 2)
    one = torch.ones(3, dtype=torch.int32, device=cuda_device)
    one[2] = 0

    def run():
        for l in range(L):
            dec.step(l, *rows[l], None, D ** -0.5, out, counts=one)
        dec.advance(1)

    rows = [[noise(l * 5 + i, cuda_device, 3, 1, h, D) for i, h in enumerate((H, G, G))] for l in range(L)]
    out = torch.empty((3, 1, H, D), dtype=BF, device=cuda_device)
    run()
    torch.cuda.synchronize()
    assert dec.lengths.tolist() == [61, 26, 0] and dec.ctx.poll_device_status() == binding.OK
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert dec.lengths.tolist() == [64, 29, 0] and dec.ctx.poll_device_status() == binding.OK
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert dec.lengths.tolist() == [64, 32, 0] and dec.ctx.poll_device_status() == binding.ERR_INVALID_ARG
    assert dec.ctx.poll_device_status() == binding.OK
    # a page more, and the second goes on where it stopped
    dec.reserve(1, 48)
    graph.replay()
    torch.cuda.synchronize()
    assert dec.lengths.tolist() == [64, 33, 0] and out[1].abs().sum() > 0 and (out[2] == 0).all()
    assert dec.ctx.poll_device_status() == binding.ERR_INVALID_ARG              # (the first is full)


@pytest.mark.parametrize("n", [1, 3])
def test_a_batch_that_is_not_full_is_no_mistake(cuda_device, n):
    """Steps without counts: the sequence that there is has its results, the other places nothing, and the status word stays clear; in a graph too,
    whose places are filled and emptied between replays."""
    from paper_2604_06746_b200 import binding
    dec, own = decode(cuda_device, 16), decode(cuda_device, 1)
    dec.reserve(5, 40)
    own.reserve(0, 40)
    keep(dec, 5, 30, 1)
    keep(own, 0, 30, 1)
    for i in range(2):
        got, want = step(dec, n, 40 + i), step(own, n, 40 + i)
        dec.advance(1)
        own.advance(1)
        assert near(got[:, 5], want[:, 0]) and (got[:, :5] == 0).all() and (got[:, 6:] == 0).all()
    assert dec.ctx.poll_device_status() == binding.OK and dec.lengths.tolist() == [0] * 5 + [32] + [0] * 10
    rows = [noise(i, cuda_device, 16, n, h, D) for i, h in enumerate((H, G, G))]
    out, graph = torch.empty((16, n, H, D), dtype=BF, device=cuda_device), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        dec.step(0, *rows, None, D ** -0.5, out)
    dec.reserve(9, 16)
    dec.release(5)
    graph.replay()
    torch.cuda.synchronize()
    assert out[9].abs().sum() > 0 and (out[:9] == 0).all() and (out[10:] == 0).all() and dec.ctx.poll_device_status() == binding.OK


def test_positions_without_a_rope_are_refused(cuda_device):
    """Also where rows are appended by the context, or by the library."""
    import ctypes

    from paper_2604_06746_b200 import binding
    dec = decode(cuda_device, 1)
    dec.reserve(0, 40)
    p, (k, v) = dec.layers[0], (noise(i, cuda_device, 1, 4, G, D) for i in range(2))
    positions = torch.arange(4, dtype=torch.int32, device=cuda_device)
    before = p.k.view(torch.uint8).clone()
    with pytest.raises(AssertionError):
        dec.ctx.append_pages(p, k, v, positions=positions)
    # structkv_append_pages_args, field by field
    words = [k.data_ptr(), v.data_ptr(), *k.stride()[:3], 4 | 4 << 32, 0, 0, 0, 0, positions.data_ptr(), 0, 0, 0, 0, 0, 0]
    args = (ctypes.c_longlong * len(words))(*words)
    call = binding.lib.structkv_append_pages
    call.restype, call.argtypes = ctypes.c_int, [ctypes.c_void_p] * 4
    stream = torch.cuda.current_stream().cuda_stream
    assert call(dec.ctx._h, p.native[0], ctypes.addressof(args), stream) == binding.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(before, p.k.view(torch.uint8))
    args[10] = 0
    assert call(dec.ctx._h, p.native[0], ctypes.addressof(args), stream) == binding.OK
    torch.cuda.synchronize()
    assert not torch.equal(before, p.k.view(torch.uint8)) and dec.ctx.poll_device_status() == binding.OK


def test_dropped_rows_stay_in_the_scale(cuda_device):
    """A drafted token far larger than the others is not kept: the block's scale stays raised, its older codes as they were rounded, and they are the
    statement's of all rows that were written."""
    import numpy as np

    from oracle import pages_oracle as P
    dec = decode(cuda_device, 1)
    dec.reserve(0, 16)
    kept, draft, after = (noise(i, cuda_device, 1, n, G, D) for i, n in enumerate((5, 3, 1)))
    draft[0, 2] *= 64.0
    page, host = dec.layers[0], lambda x: x[0, :, 0].double().cpu().numpy()
    codes, exps = np.zeros((16, D), dtype=np.uint8), [P.LOW]
    for x, n in ((kept, 0), (draft, 5), (after, 5)):
        dec.lengths[0] = n
        dec.ctx.append_pages(page, x, x)
        had = exps[0]
        codes, exps = P.append(codes, exps, n, host(x))
    torch.cuda.synchronize()
    at = int(dec.table[0, 0])
    assert page.v_scales[at, 0, 0].view(torch.uint8).item() - 127 == exps[0] == had > P.append(codes, exps, 0, host(kept))[1][0]
    assert np.array_equal(page.v[at, 0, :6].view(torch.uint8).cpu().numpy(), codes[:6])
