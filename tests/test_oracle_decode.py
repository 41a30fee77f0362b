"""Pins for the statement of decoding over a compacted cache (oracle/decode_oracle.py) and the checks of the calls that need no GPU."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D


@pytest.mark.parametrize("n,t,groups", [(0, 1, 1), (7, 1, 4), (13, 5, 2), (0, 6, 3)])
def test_attention_without_a_tree_is_causal_softmax(n, t, groups):
    rng = np.random.default_rng(n + t)
    q, k, v = rng.normal(size=(t, groups, 8)), rng.normal(size=(n + t, 8)), rng.normal(size=(n + t, 8))
    out, lse, p = D.attend(q, k, v, np.arange(n + t), n, 0.3)
    x = torch.einsum("tgd,nd->tgn", torch.from_numpy(q), torch.from_numpy(k)) * 0.3
    x = x.masked_fill(~torch.ones(t, n + t).tril(n).bool()[:, None], float("-inf"))
    assert np.allclose(lse, torch.logsumexp(x, 2).numpy(), rtol=1e-13)
    assert np.allclose(p, torch.softmax(x, 2).numpy(), rtol=1e-12, atol=0)
    assert np.allclose(out, (torch.softmax(x, 2) @ torch.from_numpy(v)).numpy(), rtol=1e-11, atol=1e-14)


def test_a_tree_is_each_of_its_paths():
    """A token of a tree gets what it gets at the end of the chain of its ancestors."""
    rng = np.random.default_rng(1)
    n, parents = 9, [-1, 0, 0, 2, -1, 4]
    t = len(parents)
    q, k, v = rng.normal(size=(t, 2, 8)), rng.normal(size=(n + t, 8)), rng.normal(size=(n + t, 8))
    chains = [[i] if p < 0 else None for i, p in enumerate(parents)]
    for i, p in enumerate(parents):
        if p >= 0:
            chains[i] = chains[p] + [i]
    pos = np.concatenate([np.arange(n), [n + len(c) - 1 for c in chains]])
    slopes = np.array([0.5, 0.25])
    out, lse, _ = D.attend(q, k, v, pos, n, 0.3, 4.0, slopes, [sum(1 << u for u in c) for c in chains])
    for i, c in enumerate(chains):
        at = list(range(n)) + [n + u for u in c]
        o, l, _ = D.attend(q[c], k[at], v[at], pos[at], n, 0.3, 4.0, slopes)
        assert np.allclose(out[i], o[-1], rtol=1e-13) and np.allclose(lse[i], l[-1], rtol=1e-13)


def test_a_row_that_sees_nothing():
    out, lse, p = D.attend(np.ones((2, 1, 4)), np.full((2, 4), np.nan), np.full((2, 4), np.nan), np.arange(2), 0, 1.0, masks=[0, 0])
    assert not out.any() and np.isneginf(lse).all() and not p.any()


def test_softcap_and_distance_by_hand():
    q, k = np.array([[[2.0]]]), np.array([[1.0], [3.0], [-5.0]])
    x = 1.5 * np.tanh(np.array([2.0, 6.0, -10.0]) * 0.5 / 1.5) - 0.25 * (10 - np.array([4.0, 9.0, 10.0]))
    _, lse, p = D.attend(q, k, k, np.array([4, 9, 10]), 2, 0.5, 1.5, [0.25])
    assert np.allclose(lse, np.log(np.exp(x).sum())) and np.allclose(p[0, 0], np.exp(x) / np.exp(x).sum())


@pytest.mark.parametrize("n,budget,recent", [(6, 3, 0), (7, 4, 2), (7, 2, 4), (5, 5, 1), (6, 5, 1)])
def test_eviction_keeps_the_best_set(n, budget, recent):
    """Of all sets of `budget` tokens that hold as many of the recent ones as they can, the kept one has the largest weight; tokens that
    stay in place are not moved, moves are ascending and fill exactly the slots that go."""
    rng = np.random.default_rng(n * budget)
    for _ in range(20):
        w, pos = rng.permutation(n).astype(float), rng.permutation(n)
        moves = D.evict_moves(w, pos, n, budget, recent)
        slots = list(range(n))
        for f, to in moves:
            assert f >= budget > to
            slots[to] = f
        kept = set(slots[:min(n, budget)])
        assert len(kept) == min(n, budget) and moves == sorted(moves) and [m[1] for m in moves] == sorted(m[1] for m in moves)
        new = {j for j in range(n) if pos[j] > pos.max() - recent}
        if n > budget:
            best = max(itertools.combinations(range(n), budget), key=lambda c: (len(new & set(c)), sum(w[j] for j in c if j not in new)))
            if len(new) <= budget:
                assert kept == set(best)
            else:
                assert kept == set(sorted(new)[:budget])


def test_commit_slots():
    assert D.commit_slots(5, 3) == [5, 6, 7] and D.commit_slots(5, 3, 2) == [5, 6] and D.commit_slots(5, 4, 2, [1, 3, 0, 0]) == [6, 8]


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_b200 import build
    build.build()
    from paper_2604_06746_b200 import binding
    return binding


def test_workspace_sizes(B):
    def size(batch, n_new, capacity, h=8, g=2, d=64, dtype=None):
        cfg = B.Config(h, g, d, 4, 100, B.BF16 if dtype is None else dtype)
        return B.lib.structkv_attend_workspace_bytes(ctypes.byref(cfg), batch, n_new, capacity)
    for dtype in (B.BF16, B.FP32):
        assert 0 < size(1, 1, 1, dtype=dtype) <= size(2, 1, 1, dtype=dtype) <= size(2, 1, 1000, dtype=dtype) < size(64, 1, 1 << 20, dtype=dtype)
    assert size(1, 64, 64) > 0
    for batch, n_new, capacity in ((0, 1, 8), (-1, 1, 8), (1, 0, 8), (1, 65, 100), (1, 9, 8), (1, 1, 0), (1, 1, (1 << 30) + 1), (1 << 30, 1, 1 << 20)):
        assert size(batch, n_new, capacity) == 0, (batch, n_new, capacity)
    assert size(1, 1, 8, h=7) == 0


def test_checks_before_the_library(B):
    ctx = object.__new__(B.Context)                        # no device: the checks come first
    ctx._h, ctx.cfg, ctx.dtype = ctypes.c_void_p(), B.Config(4, 2, 64, 4, 100, B.BF16), torch.bfloat16
    bf = torch.bfloat16
    k, words, lengths = torch.empty((3, 2, 20, 64), dtype=bf), torch.zeros((3, 2, 20), dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(AssertionError):
        B.Cache(k, k, words, words.float(), lengths)       # not on a device
    cache = object.__new__(B.Cache)
    cache._struct = B.CacheStruct(k.data_ptr(), k.data_ptr(), *k.stride()[:3], words.data_ptr(), None, lengths.data_ptr(), 3, 20)
    cache.native = (ctypes.addressof(cache._struct), B.BF16, 0, 3, 2, 64, 20)
    cache.batch, cache.n_kv_heads, cache.capacity, cache.head_dim, cache.dtype, cache.device = 3, 2, 20, 64, bf, torch.device("cpu")
    q, rows, pos = torch.empty((3, 5, 4, 64), dtype=bf), torch.empty((3, 5, 2, 64), dtype=bf), torch.zeros((3, 5), dtype=torch.int32)
    lse, ws = torch.empty((3, 5, 4)), torch.empty(1 << 20, dtype=torch.uint8)
    acc = torch.zeros(3, dtype=torch.int64)
    ctx._of = lambda c: c.native
    many = torch.empty((3, 65, 4, 64), dtype=bf)
    for bad, what in ((lambda: ctx.attend(cache, q[:, :, :3], 1.0, q, ws), "q:"), (lambda: ctx.attend(cache, q.float(), 1.0, q, ws), "q:"),
                      (lambda: ctx.attend(cache, q, 1.0, q[:, :4], ws), "out:"), (lambda: ctx.attend(cache, many, 1.0, many, ws), "64 new tokens"),
                      (lambda: ctx.attend(cache, q, 1.0, q, ws), "q: on"), (lambda: ctx.attend(cache, q, 1.0, q, ws, v_new=rows), "together"),
                      (lambda: ctx.attend(cache, q, 1.0, q, ws, k_new=rows, v_new=rows.expand(3, 5, 2, 64)[:, :4], positions=pos), "v_new"),
                      (lambda: ctx.attend(cache, q, 1.0, q, ws, k_new=rows, v_new=rows, positions=pos.long()), "positions"),
                      (lambda: ctx.append(cache, rows[..., :32], rows, pos), "k_new"), (lambda: ctx.append(cache, rows, rows, pos), "positions"),
                      (lambda: ctx.weigh(cache, q[:2], 1.0, lse, acc), "q:"), (lambda: ctx.commit(cache, 5, counts=acc), "counts"),
                      (lambda: ctx.commit(cache, 5, counts=lengths[:, 0], path=pos), "counts"),
                      (lambda: ctx.commit(cache, 5, path=pos[:, :4]), "path")):
        with pytest.raises(AssertionError, match=what):
            bad()
