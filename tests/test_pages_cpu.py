"""CPU: the statement of rotary positions and of the paged cache in 8 bits, frequencies as the library works them out, and what is refused before
the library is reached."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as P


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_b200 import build
    build.build()
    from paper_2604_06746_b200 import binding
    return binding


SCALINGS = [{}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="bands", factor=8.0, original=8192, slow=1.0, fast=4.0),
            dict(scaling="ramp", factor=32.0, original=32768, slow=1.0, fast=32.0), dict(scaling="ramp", factor=0.5, original=100, slow=0.5, fast=2.0)]


@pytest.mark.parametrize("more", SCALINGS)
@pytest.mark.parametrize("dim,base", [(128, 500000.0), (64, 10000.0), (48, 1.5), (4, 10000.0)])
def test_frequencies(B, dim, base, more):
    f, amp = P.frequencies(dim, base, **more)
    rope = B.Rope(dim, base, **more)
    turns = np.array(f) / (2 * math.pi) % 1.0
    # (64-bit steps: 2^-65 of a turn; the statement is in fp64: 2^-50 after a few operations)
    assert np.allclose(rope.turns, turns, rtol=2.0 ** -48, atol=2.0 ** -64)
    assert abs(rope.amplitude - amp) <= 2.0 ** -23 * amp and rope.dim == dim and not rope.interleaved


def test_frequencies_that_are_refused(B):
    good = dict(dim=64, base=10000.0)
    for bad in (dict(dim=63), dict(dim=0), dict(dim=130), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.0),
                dict(scaling="linear", factor=float("inf")), dict(scaling="bands", factor=2.0), dict(scaling="bands", factor=2.0, original=100, slow=4.0, fast=4.0),
                dict(scaling="ramp", factor=2.0, original=-1.0), dict(scaling="base", factor=2.0, dim=2), dict(scaling="base", factor=1e-9)):
        with pytest.raises(B.StructKVError) as e:
            B.Rope(**(good | bad))
        assert e.value.status == B.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        B.Rope(64, scaling="other")
    assert B.lib.structkv_rope_init(None, 64, 0, 10000.0, 0, 1.0, 0.0, 0.0, 0.0) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(0)
    f, amp = P.frequencies(32, 10000.0, "ramp", 8.0, 512, 1.0, 32.0)
    x, at = rng.standard_normal((20, 48)), rng.integers(-1000, 1000, 20)
    y = P.rotate(x, at, f, amp, interleaved)
    a, b = P.pairs(32, interleaved)
    z = (x[:, a] + 1j * x[:, b]) * amp * np.exp(1j * at[:, None] * f)
    assert np.allclose(y[:, a], z.real) and np.allclose(y[:, b], z.imag) and np.array_equal(y[:, 32:], x[:, 32:])
    # the inverse is the transpose: <y, R x> = <R^T y, x>
    w = rng.standard_normal((20, 48))
    assert np.allclose((w * y).sum(1), (P.rotate(w, at, f, amp, interleaved, inverse=True) * x).sum(1))


def test_codes_are_torchs():
    rng = np.random.default_rng(1)
    x = np.concatenate([np.clip(rng.standard_normal(20000) * np.exp(3 * rng.standard_normal(20000)), -448, 448), (P._POSITIVE[1:] + P._POSITIVE[:-1]) / 2,
                        -P._POSITIVE, [0.0, -0.0, np.nan]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    got = P.code_of(x)
    assert np.array_equal(got[:-1], want.view(torch.uint8).numpy()[:-1]) and np.isnan(P.CODES[got[-1]])
    assert np.array_equal(P.CODES, torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_scales_of_blocks():
    assert [P.exponent(x) for x in (0.0, 448.0, 448.5, 224.0, 1.75, 1.76, 1e-30, 3.3e38)] == [-40, 0, 1, -1, -8, -7, -40, 120]
    rng = np.random.default_rng(2)
    rows = rng.standard_normal((40, 8))
    codes, exps = np.zeros((64, 8), dtype=np.uint8), [-40] * 4
    once = P.append(codes, exps, 0, rows)
    # at once or in pieces: blocks that are begun anew have the same codes, and no value is far off
    c, e = codes, exps
    for lo, hi in ((0, 1), (1, 17), (17, 40)):
        c, e = P.append(c, e, lo, rows[lo:hi])
    for got in (once, (c, e)):
        step = np.maximum(2.0 ** -4 * np.abs(rows), 2.0 ** (np.repeat(got[1], 16)[:40, None] - 10.0))
        assert (np.abs(P.values(*got)[:40] - rows) <= 2 * step).all()
    assert list(once[1]) == list(e) and (c[40:] == 0).all()
    bad = rows.copy()
    bad[3, 2], bad[20, 1] = np.inf, np.nan
    c, e = P.append(codes, exps, 0, bad)
    v = P.values(c, e)[:40]
    assert np.isnan(v[3, 2]) and np.isnan(v[20, 1]) and np.isfinite(np.delete(v, [3, 20], 0)).all()


def test_workspace(B):
    cfg = B.Config(32, 8, 128, 8, 8, B.BF16)
    size = lambda *a: B.lib.structkv_attend_pages_workspace_bytes(ctypes.byref(cfg), *a)
    assert size(4, 1, 1024) > 0 and size(4, 64, 1024) > size(4, 1, 1024) and size(8, 1, 1 << 30) > 0
    for bad in ((0, 1, 1024), (4, 0, 1024), (4, 65, 1024), (4, 1, 0), (4, 1, (1 << 30) + 1), (1 << 28, 64, 1024), (1 << 20, 1, 1 << 30)):
        assert size(*bad) == 0
    assert B.lib.structkv_attend_pages_workspace_bytes(ctypes.byref(B.Config(32, 8, 96, 8, 8, B.BF16)), 4, 1, 1024) == 0


def test_null_arguments(B):
    for call in (B.lib.structkv_rotate, B.lib.structkv_append_pages, B.lib.structkv_attend_pages):
        call.restype = ctypes.c_int
        assert call(None, None, None, None) == B.ERR_INVALID_ARG


def test_checks_before_the_library(B):
    """Tensors that are not on the device, of other types or shapes: refused by the binding (the pages' address is never looked at)."""
    ctx = object.__new__(B.Context)
    ctx._h, ctx.cfg, ctx.dtype, ctx.device = ctypes.c_void_p(), B.Config(4, 2, 64, 8, 8, B.BF16), torch.bfloat16, torch.device("cuda:0")
    pages = object.__new__(B.Pages)
    pages.native, pages.n_kv_heads, pages.head_dim = (0, 0, 2, 2, 64, 128), 2, 64
    q, k = torch.empty((2, 3, 4, 64), dtype=torch.bfloat16), torch.empty((2, 3, 2, 64), dtype=torch.bfloat16)
    out, ws, pos, rope = torch.empty_like(q), torch.empty(1000, dtype=torch.uint8), torch.zeros((2, 3), dtype=torch.int32), B.Rope(64)
    for bad in (lambda: ctx.rotate(q, pos, rope), lambda: ctx.rotate(q[0], pos, rope), lambda: ctx.rotate(q.float(), pos, rope), lambda: ctx.rotate(q[..., :32], pos, rope),
                lambda: ctx.append_pages(pages, k, k), lambda: ctx.append_pages(pages, k, k[:, :2]), lambda: ctx.append_pages(pages, k.float(), k.float()),
                lambda: ctx.append_pages(pages, q, q), lambda: ctx.append_pages(pages, k[:1], k[:1]),
                lambda: ctx.attend_pages(pages, q, 1.0, out, ws), lambda: ctx.attend_pages(pages, q[:, :, :3], 1.0, out, ws), lambda: ctx.attend_pages(pages, q.float(), 1.0, out, ws),
                lambda: ctx.attend_pages(pages, q, 1.0, out[:, :2], ws)):
        with pytest.raises(AssertionError):
            bad()
    ok = dict(k=torch.empty((5, 2, 32, 64), dtype=torch.float8_e4m3fn), v=torch.empty((5, 2, 32, 64), dtype=torch.float8_e4m3fn),
              k_scales=torch.empty((5, 2, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu), v_scales=torch.empty((5, 2, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu),
              table=torch.zeros((3, 4), dtype=torch.int32), lengths=torch.zeros(3, dtype=torch.int32))
    for change in ({}, dict(k=ok["k"].view(torch.uint8)), dict(v=ok["v"][:4]), dict(k=ok["k"][:, :, :24], v=ok["v"][:, :, :24]), dict(k_scales=ok["k_scales"].view(torch.uint8)),
                   dict(table=ok["table"].long()), dict(table=ok["table"][:, :0]), dict(lengths=ok["lengths"][:2])):
        with pytest.raises(AssertionError):                # (the first for not being on a device)
            B.Pages(**(ok | change))
