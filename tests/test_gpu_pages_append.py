"""GPU: appending rows to a paged cache in 8 bits, with rotation, gather and scales of blocks, against the float64 statement."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from tests.pages_cases import HALF, TURN, Paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def append(p, k, v, counts=None, index=None, **more):
    dev = {"counts": counts, "index": index}
    dev = {n: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=p.device) for n, x in dev.items()}
    p.ctx.append_pages(p.pages, k, v, **dev, **more)


def check_exact(p, k, v, counts=None, index=None):
    """Everything that the pages hold, byte by byte (rows that are not rotated)."""
    got_codes, got_exps = p.read()
    codes, exps = {x: c.copy() for x, c in p.codes.items()}, {x: e.copy() for x, e in p.exps.items()}
    for x, rows in (("k", k), ("v", v)):
        rows = rows.double().numpy()
        for b in range(p.b):
            at = np.arange(rows.shape[1]) if index is None else np.asarray(index)[b]
            c = len(at) if counts is None else counts[b]
            new = np.where(((at >= 0) & (at < rows.shape[1]))[:, None, None], rows[b, np.clip(at, 0, rows.shape[1] - 1)], 0.0)[:c]
            for g in range(p.g):
                hc, he = P.append(*p.head(x, b, g), p.n[b], new[:, g])
                for i in range(p.n[b] // p.page, -(-(p.n[b] + c) // p.page)):
                    codes[x][p.table[b, i], g] = hc[i * p.page:(i + 1) * p.page]
                    exps[x][p.table[b, i], g] = he[i * p.page // 16:(i + 1) * p.page // 16]
        assert np.array_equal(got_exps[x], exps[x]), x
        same = got_codes[x] == codes[x]
        assert (same | ((got_codes[x] & 127 == 127) & (codes[x] & 127 == 127))).all(), x


LENGTHS = [([0], 16, 1), ([0, 1, 15, 16, 17, 31], 16, 1), ([5, 0, 100], 32, 2), ([63, 64, 65], 64, 16), ([0, 7, 300], 128, 33), ([1, 250], 256, 70)]


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("small", BF), ("small", F32), ("single", F32)])
@pytest.mark.parametrize("lengths,page,t", LENGTHS)
def test_rows_and_scales(cuda_device, shape, dtype, lengths, page, t):
    p = Paged(cuda_device, shape, lengths, page, seed=t, dtype=dtype, token_major=t == 2)
    (k, dk), (v, dv) = p.noise(p.b, t, p.g, p.d, spread=3.0), p.noise(p.b, t, p.g, p.d)
    append(p, dk, dv)
    check_exact(p, k, v)
    assert p.ctx.poll_device_status() == 0 and np.array_equal(p.dlen.cpu(), p.n)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_scale_grows_and_old_codes_are_rounded_again(cuda_device, dtype):
    """Token after token into one block, each larger or smaller by powers of two; then values where codes tie and scales change."""
    p = Paged(cuda_device, "small", [3, 16], 16, seed=1, dtype=dtype)
    for step, size in enumerate([1.0, 8.0, 2.0 ** -30, 448.0, 449.0, 2.0 ** 20, 0.0, 1e-12, 2.0 ** 60, 3e38]):
        x = torch.from_numpy(p.rng.uniform(-1, 1, (p.b, 1, p.g, p.d)).astype(np.float32)) * size
        if size:
            x[:, :, :, 0] = size
        x = x.to(dtype)
        append(p, x.to(p.device), x.to(p.device))
        check_exact(p, x, x)
        p.codes, p.exps = p.read()
        p.n = [n + 1 for n in p.n]
        p.dlen += 1
    assert p.ctx.poll_device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_rounding(cuda_device, dtype):
    """All halves between neighbouring codes, and beside them."""
    pos = np.sort(P._POSITIVE)
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -8), pos, -mid, [448.0] * 3])
    x = np.resize(x, (1, 11, 2, 64)).astype(np.float32)
    x[..., 0] = 448.0
    p = Paged(cuda_device, "small", [2], 16, seed=2, dtype=dtype)
    rows = torch.from_numpy(x).to(dtype)
    append(p, rows.to(p.device), -rows.to(p.device))
    check_exact(p, rows, -rows)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_is_not_finite(cuda_device, dtype):
    p = Paged(cuda_device, "llama", [4, 30], 32, seed=3, dtype=dtype)
    (k, _), (v, _) = p.noise(p.b, 20, p.g, p.d), p.noise(p.b, 20, p.g, p.d)
    k[0, 2, 1, 3], k[0, 2, 1, 9], v[1, 0, 0, 0], v[1, 7, 2], k[1, 1, 4] = float("inf"), float("nan"), -float("inf"), float("nan"), float("inf")
    append(p, k.to(p.device), v.to(p.device))
    check_exact(p, k, v)


@pytest.mark.parametrize("shape,dtype", [("llama", BF), ("small", F32)])
def test_gathered_rows_and_counts(cuda_device, shape, dtype):
    p = Paged(cuda_device, shape, [0, 40, 7], 64, seed=4, dtype=dtype)
    (k, dk), (v, dv) = p.noise(p.b, 90, p.g, p.d), p.noise(p.b, 90, p.g, p.d)
    index = np.stack([np.sort(p.rng.permutation(90)[:50]), p.rng.integers(0, 90, 50), np.full(50, 89)])
    append(p, dk, dv, index=index, counts=[50, 0, 23])
    check_exact(p, k, v, index=index, counts=[50, 0, 23])
    assert p.ctx.poll_device_status() == 0
    # one list for all sequences; entries that are no source token
    p = Paged(cuda_device, shape, [0, 40, 7], 64, seed=5, dtype=dtype)
    index = p.rng.integers(0, 90, 18)
    index[4], index[9] = 90, -1
    append(p, dk, dv, index=index)
    check_exact(p, k, v, index=np.stack([index] * 3))
    assert p.ctx.poll_device_status() == 1 and p.ctx.poll_device_status() == 0


def test_rows_from_any_buffer(cuda_device):
    """Rows inside a fused projection's output, heads before tokens, one row for all sequences."""
    p = Paged(cuda_device, "llama", [9, 64], 64, seed=6)
    fused, dfused = p.noise(p.b, 20, p.h + 2 * p.g, p.d)
    append(p, dfused[:, :, p.h:p.h + p.g], dfused[:, :, p.h + p.g:])
    check_exact(p, fused[:, :, p.h:p.h + p.g], fused[:, :, p.h + p.g:])
    p = Paged(cuda_device, "llama", [9, 64], 64, seed=6)
    kv, dkv = p.noise(2, 1, p.g, 20, p.d)
    append(p, *(x.transpose(1, 2).expand(2, -1, -1, -1) for x in dkv))
    check_exact(p, *(x.transpose(1, 2).expand(2, -1, -1, -1) for x in kv))


ROPES = [dict(dim=128), dict(dim=128, interleaved=True, scaling="bands", factor=8.0, original=8192, slow=1.0, fast=4.0),
         dict(dim=64, scaling="linear", factor=4.0), dict(dim=48, scaling="base", factor=8.0), dict(dim=2), dict(dim=10, interleaved=True),
         dict(dim=22), dict(dim=128, scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0)]


def turned(rope, more, rows, positions):
    """(statement, bound of what fp32 may be off) of rotated rows [tokens, heads, d]."""
    dim, inter = more["dim"], more.get("interleaved", False)
    f, amp = P.frequencies(dim, 10000.0, **{k: v for k, v in more.items() if k not in ("dim", "interleaved")})
    y = P.rotate(rows, positions, f, amp, inter)
    a, b = P.pairs(dim, inter)
    size = np.zeros_like(y)
    size[..., a] = size[..., b] = amp * (np.abs(rows[..., a]) + np.abs(rows[..., b]))
    return y, size


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", ROPES)
def test_keys_and_queries_are_rotated(cuda_device, dtype, more):
    from paper_2604_06746_b200 import binding
    p = Paged(cuda_device, "llama", [0, 21], 32, seed=7, dtype=dtype)
    rope = binding.Rope(base=10000.0, **more)
    t = 37
    (k, dk), (v, dv), (q, dq) = p.noise(2, t, p.g, p.d), p.noise(2, t, p.g, p.d), p.noise(2, t, p.h, p.d)
    positions = p.rng.integers(0, 1 << 20, (2, t)).astype(np.int32)
    q_out = torch.full((2, t, p.h, p.d), float("nan"), dtype=dtype, device=p.device)
    append(p, dk, dv, counts=[t, 30], positions=torch.from_numpy(positions).to(p.device), rope=rope, q=dq, q_out=q_out)
    codes, exps = p.read()
    for b, c in ((0, t), (1, 30)):
        y, size = turned(rope, more, q[b].double().numpy(), positions[b])
        assert (np.abs(q_out[b].double().cpu().numpy() - y) <= 1.001 * HALF[dtype] * np.abs(y) + TURN[dtype] * size).all()
        y, size = turned(rope, more, k[b].double().numpy(), positions[b])
        for g in range(p.g):
            hc, he = p.head("k", b, g, codes, exps)
            n, off = p.n[b], TURN[dtype] * size[:c, g]
            got = P.values(hc, he)[n:n + c]
            for j in range(n // 16, -(-(n + c) // 16)):
                rows = slice(max(0, j * 16 - n), min(c, j * 16 + 16 - n))
                top, most = np.abs(y[rows, g]).max(), off[rows].max()
                old = p.head("k", b, g)[1][j] if j * 16 < n else P.LOW
                assert max(P.exponent(top - most), old) <= he[j] <= max(P.exponent(top + most), old), (b, g, j)
                # a code is the nearest to what was rounded: half a step of it, relative, or of the smallest numbers
                step = np.maximum(2.0 ** -4 * np.abs(y[rows, g]), 2.0 ** (he[j] - 10))
                assert (np.abs(got[rows] - y[rows, g]) <= 1.001 * step + off[rows]).all(), (b, g, j)
    # V as without rotation, and queries in place
    append(p, dk, dv, counts=[t, 30], positions=torch.from_numpy(positions).to(p.device), rope=rope, q=dq)
    assert torch.equal(dq, q_out)
    want = Paged(cuda_device, "llama", [0, 21], 32, seed=7, dtype=dtype)
    append(want, dk, dv, counts=[t, 30])
    assert torch.equal(want.pages.v.view(torch.uint8), p.pages.v.view(torch.uint8))


def test_sequences_that_are_refused_stay(cuda_device):
    p = Paged(cuda_device, "small", [30, 30, 30, 30, 30], 32, seed=8)
    (k, dk), (v, dv) = p.noise(p.b, 8, p.g, p.d), p.noise(p.b, 8, p.g, p.d)
    before = p.read()
    p.dlen[0], p.dlen[1] = -3, p.slots - 7
    p.dtable[2, 1] = 1 << 20                               # the page that the last six rows go to
    append(p, dk, dv, counts=[8, 8, 8, 9, 5])
    assert p.ctx.poll_device_status() == 1 and p.ctx.poll_device_status() == 0
    codes, exps = p.read()
    for b in (0, 1, 3):
        for page in p.table[b]:
            for x in "kv":
                assert np.array_equal(codes[x][page], before[0][x][page]) and np.array_equal(exps[x][page], before[1][x][page])
    p.b, p.table, p.n = 2, p.table[[2, 4]], [30, 30]
    rows = [torch.cat([x[2:3], x[4:]]) for x in (k, v)]
    for x, r in zip("kv", rows):                           # two rows of the third, five of the fifth
        for b, c in ((0, 2), (1, 5)):
            for g in range(p.g):
                hc, he = P.append(*p.head(x, b, g), 30, r[b, :c, g].double().numpy())
                got = p.head(x, b, g, codes, exps)
                assert np.array_equal(got[0], hc) and np.array_equal(got[1], he)


def test_refusals(cuda_device):
    from paper_2604_06746_b200 import binding
    p = Paged(cuda_device, "small", [10, 20], seed=9)
    k, q = p.noise(2, 4, 2, 64)[1], p.noise(2, 4, 8, 64)[1]
    pos, rope, run, i32 = torch.zeros((2, 4), dtype=torch.int32, device=k.device), binding.Rope(64), p.ctx.append_pages, torch.int32
    for bad in (lambda: run(p.pages, k.float(), k), lambda: run(p.pages, k, k[:, :3]), lambda: run(p.pages, k[:1], k[:1]), lambda: run(p.pages, k.cpu(), k.cpu()),
                lambda: run(p.pages, k, k.transpose(1, 2).contiguous().transpose(1, 2)), lambda: run(p.pages, k, k, rope=rope),
                lambda: run(p.pages, k, k, positions=pos.long(), rope=rope), lambda: run(p.pages, k, k, positions=pos[:, :3], rope=rope),
                lambda: run(p.pages, k, k, counts=torch.ones(3, dtype=i32, device=k.device)), lambda: run(p.pages, k, k, q=q),
                lambda: run(p.pages, k, k, positions=pos, rope=rope, q_out=q), lambda: run(p.pages, k, k, positions=pos, rope=rope, q=q[:, :3]),
                lambda: run(p.pages, k, k, positions=pos, rope=rope, q=q, index=pos), lambda: run(p.pages, k, k, positions=pos, rope=rope, q=q, q_out=q.float()),
                lambda: run(p.pages, k[:, :0], k[:, :0]), lambda: run(p.pages, k, k, index=pos.float()),
                lambda: run(p.pages, k[:, :1].expand(-1, 999, -1, -1), k[:, :1].expand(-1, 999, -1, -1))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(binding.StructKVError):
        run(p.pages, k, k, positions=pos, rope=binding.Rope(128))          # more than a head has
    assert p.ctx.poll_device_status() == 0
    t = p.pages
    for change in (dict(k=t.k.view(torch.uint8)), dict(k_scales=t.k_scales[:, :1]), dict(table=t.table.long()), dict(lengths=t.lengths[:1]),
                   dict(v=t.v[:, :, :32]), dict(table=t.table[0])):
        parts = dict(k=t.k, v=t.v, k_scales=t.k_scales, v_scales=t.v_scales, table=t.table, lengths=t.lengths) | change
        with pytest.raises(AssertionError):
            binding.Pages(**parts)
