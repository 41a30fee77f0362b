"""GPU tests of the steps between attentions over a compacted cache: append, commit and eviction, against the statement in
oracle/decode_oracle.py.  Rows are moved bit for bit; what is not written stays."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


class Store:
    """A cache of random bits, and its mirror on the host."""

    def __init__(self, device, lengths, cap, d=64, dtype=torch.bfloat16, seed=0, weights=None, positions=None):
        from paper_2604_06746_b200 import binding
        rng = np.random.default_rng(seed)
        b, g = np.shape(lengths)
        bits = np.int16 if dtype == torch.bfloat16 else np.int32
        self.k, self.v = (rng.integers(-2 ** 14, 2 ** 14, size=(b, g, cap, d)).astype(bits) for _ in range(2))
        self.pos = np.argsort(rng.random((b, g, cap)), axis=2).astype(np.int32) if positions is None else positions.astype(np.int32)
        self.w = (rng.random((b, g, cap)) ** 3).astype(np.float32) if weights is None else weights.astype(np.float32)
        self.n = np.array(lengths, dtype=np.int32)
        self.t = [torch.from_numpy(self.k).view(dtype).to(device), torch.from_numpy(self.v).view(dtype).to(device),
                  torch.from_numpy(self.pos).to(device), torch.from_numpy(self.w).to(device), torch.from_numpy(self.n).to(device)]
        self.bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
        self.cache = binding.Cache(*self.t)
        self.ctx = binding.Context(2 * g, g, d, 8, 8, dtype, device)

    def move(self, b, g, pairs):
        """The host's mirror: all sources are read before anything is written."""
        for a in (self.k, self.v, self.pos, self.w):
            rows = [a[b, g, f].copy() for f, _ in pairs]
            for (_, to), r in zip(pairs, rows):
                a[b, g, to] = r

    def check(self):
        torch.cuda.synchronize()
        for a, t in zip((self.k, self.v), self.t):
            assert np.array_equal(t.view(self.bits).cpu().numpy(), a)
        assert np.array_equal(self.t[2].cpu().numpy(), self.pos)
        assert np.array_equal(self.t[3].cpu().numpy().view(np.int32), self.w.view(np.int32))
        assert np.array_equal(self.t[4].cpu().numpy(), self.n)

    def evict(self, budget, recent):
        self.ctx.evict(self.cache, budget, recent)
        for b in range(self.n.shape[0]):
            for g in range(self.n.shape[1]):
                self.move(b, g, D.evict_moves(self.w[b, g], self.pos[b, g], int(self.n[b, g]), budget, recent))
                self.n[b, g] = min(self.n[b, g], budget)


@pytest.mark.parametrize("n,budget,recent,d,dtype", [
    (101, 100, 8, 64, torch.bfloat16), (100, 100, 8, 64, torch.bfloat16), (5, 1, 0, 128, torch.bfloat16), (300, 299, 299, 64, torch.float32),
    (2049, 2048, 64, 128, torch.bfloat16), (1000, 10, 4, 64, torch.bfloat16), (4000, 2000, 2000, 64, torch.float32),
    (8192, 8000, 100, 64, torch.bfloat16), (8193, 8000, 100, 64, torch.bfloat16), (20000, 9000, 500, 64, torch.bfloat16),
    (30001, 10007, 0, 64, torch.bfloat16), (1, 1, 1, 64, torch.bfloat16)])
def test_eviction(cuda_device, n, budget, recent, d, dtype):
    s = Store(cuda_device, [[n, max(0, n - 3)], [budget, n]], n + 9, d, dtype, seed=n)
    s.evict(budget, recent)
    s.check()
    s.evict(budget, recent)                              # nothing to do
    s.check()


@pytest.mark.parametrize("n,budget", [(500, 300), (9000, 8500), (20000, 9000), (33000, 16000)])
def test_eviction_with_ties_nan_and_infinity(cuda_device, n, budget):
    """Few different weights (ties go to the lower slot), NaN, infinities, zeros of both signs."""
    rng = np.random.default_rng(n)
    w = rng.choice(np.array([0.0, -0.0, 0.5, 0.25, np.inf, -np.inf, 1e-40, np.nan], dtype=np.float32), size=(1, 3, n), p=[.3, .1, .2, .2, .05, .05, .05, .05])
    w[0, 1] = 1.0                                        # all equal: the first ones stay
    s = Store(cuda_device, [[n, n, n - 1]], n, seed=1, weights=w)
    s.evict(budget, 40)
    s.check()


def test_all_recent_ones_and_equal_positions(cuda_device):
    """More recent tokens than the budget (positions that repeat): the first slots among them stay."""
    n = 700
    pos = np.zeros((1, 2, n), dtype=np.int32)
    pos[0, 1] = np.arange(n) // 2
    s = Store(cuda_device, [[n, n]], n, seed=2, positions=pos)
    s.evict(100, 300)
    s.check()


def test_eviction_of_bad_lengths(cuda_device):
    from paper_2604_06746_b200 import binding
    s = Store(cuda_device, [[50, 60], [70, 80]], 90, seed=3)
    s.t[4][0, 1], s.t[4][1, 0] = 91, -2
    s.ctx.evict(s.cache, 40, 5)
    torch.cuda.synchronize()
    assert s.ctx.poll_device_status() == binding.ERR_INVALID_ARG
    for b, g in ((0, 0), (1, 1)):
        s.move(b, g, D.evict_moves(s.w[b, g], s.pos[b, g], int(s.n[b, g]), 40, 5))
        s.n[b, g] = 40
    s.n[0, 1], s.n[1, 0] = 91, -2
    s.check()


@pytest.mark.parametrize("t", [1, 2, 9, 33, 64])
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_commit_of_paths(cuda_device, t, dtype, d):
    rng = np.random.default_rng(t)
    b, g = 5, 3
    lengths = rng.integers(0, 200, size=(b, g))
    s = Store(cuda_device, lengths, 200 + t, d, dtype, seed=t)
    counts = np.array([0, t, 1, t // 2, (t + 1) // 2])
    path = np.full((b, t), -7, dtype=np.int32)
    for i in range(b):
        path[i, :counts[i]] = np.sort(rng.choice(t, size=counts[i], replace=False))
    s.ctx.commit(s.cache, t, counts=torch.from_numpy(counts.astype(np.int32)).to(cuda_device), path=torch.from_numpy(path).to(cuda_device))
    for i in range(b):
        for j in range(g):
            n = int(s.n[i, j])
            s.move(i, j, [(f, n + e) for e, f in enumerate(D.commit_slots(n, t, counts[i], path[i]))])
            s.n[i, j] += counts[i]
    s.check()


def test_commit_without_a_path_and_bad_paths(cuda_device):
    from paper_2604_06746_b200 import binding
    s = Store(cuda_device, [[10, 12], [0, 5]], 30, seed=1)
    s.ctx.commit(s.cache, 4)
    s.n += 4
    s.check()
    s.ctx.commit(s.cache, 4, counts=torch.tensor([2, 0], dtype=torch.int32, device=cuda_device))
    s.n += np.array([[2], [0]], dtype=np.int32)
    s.check()
    assert s.ctx.poll_device_status() == binding.OK
    for counts, path in (([2, 1], [[1, 1, 0], [2, 0, 0]]), ([2, 1], [[2, 1, 0], [2, 0, 0]]), ([1, 1], [[3, 0, 0], [2, 0, 0]]),
                         ([4, 1], [[0, 1, 2], [2, 0, 0]]), ([-1, 1], [[0, 1, 2], [2, 0, 0]]), ([1, 1], [[-1, 0, 0], [2, 0, 0]])):
        s.ctx.commit(s.cache, 3, counts=torch.tensor(counts, dtype=torch.int32, device=cuda_device),
                     path=torch.tensor(path, dtype=torch.int32, device=cuda_device))
        for j in range(2):                               # sequence 0 stays, sequence 1 goes on
            n = int(s.n[1, j])
            s.move(1, j, [(n + 2, n)])
        s.n[1] += 1
        s.check()
        assert s.ctx.poll_device_status() == binding.ERR_INVALID_ARG


def test_append_of_strided_rows(cuda_device):
    s = Store(cuda_device, [[3, 7], [0, 26]], 30, 128, seed=9)
    rows = np.random.default_rng(0).integers(-2 ** 14, 2 ** 14, size=(2, 4, 5, 128)).astype(np.int16)   # [batch, token, K and V and more, d]
    dev = torch.from_numpy(rows).to(cuda_device).view(torch.bfloat16)
    pos = np.array([[5, 6, 6, 7], [1, 2, 3, 4]], dtype=np.int32)
    s.ctx.append(s.cache, dev[:, :, 0:2], dev[:, :, 3:5], torch.from_numpy(pos).to(cuda_device))
    for b in range(2):
        for g in range(2):
            n = int(s.n[b, g])
            s.k[b, g, n:n + 4], s.v[b, g, n:n + 4] = rows[b, :, g], rows[b, :, 3 + g]
            s.pos[b, g, n:n + 4], s.w[b, g, n:n + 4] = pos[b], 0
    s.check()


def test_a_long_piece_comes_in(cuda_device):
    """More tokens at once than attend in one call."""
    from paper_2604_06746_b200 import binding
    s = Store(cuda_device, [[3, 0], [40, 7]], 400, 64, seed=10)
    rows = np.random.default_rng(1).integers(-2 ** 14, 2 ** 14, size=(2, 2, 350, 2, 64)).astype(np.int16)
    dev = torch.from_numpy(rows).to(cuda_device).view(torch.bfloat16)
    pos = np.random.default_rng(2).integers(0, 9999, size=(2, 350)).astype(np.int32)
    s.ctx.append(s.cache, dev[0], dev[1], torch.from_numpy(pos).to(cuda_device))
    s.ctx.commit(s.cache, 350, counts=torch.tensor([350, 129], dtype=torch.int32, device=cuda_device))
    for b in range(2):
        for g in range(2):
            n = int(s.n[b, g])
            s.k[b, g, n:n + 350], s.v[b, g, n:n + 350] = rows[0, b, :, g], rows[1, b, :, g]
            s.pos[b, g, n:n + 350], s.w[b, g, n:n + 350] = pos[b], 0
            s.n[b, g] += (350, 129)[b]
    s.check()
    with pytest.raises(binding.StructKVError, match="invalid"):
        s.ctx.commit(s.cache, 65, counts=torch.zeros(2, dtype=torch.int32, device=cuda_device),
                     path=torch.zeros((2, 65), dtype=torch.int32, device=cuda_device))
