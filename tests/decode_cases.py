"""Inputs and comparisons shared by the tests of decoding over a compacted cache."""
import numpy as np
import torch

from oracle import decode_oracle as D

SHAPES = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 2, 64), "wide": (24, 1, 64), "single": (3, 3, 128)}


def signed(m):
    return m - (1 << 64) if m >= 1 << 63 else m


def random_tree(rng, t):
    masks = []
    for i in range(t):
        p = int(rng.integers(-1, i)) if i else -1
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    return masks


class Problem:
    """A cache with lengths [batch][H_kv] and new tokens, on the device; slots beyond the tokens hold NaN."""

    def __init__(self, device, shape, lengths, t, dtype=torch.bfloat16, seed=0, tree=None, softcap=0.0, distance=False,
                 token_major=False, spare=5, spread=1.0):
        h, g, d = SHAPES[shape]
        self.h, self.g, self.d, self.t, self.b, self.group = h, g, d, t, len(lengths), h // g
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.n = np.array([[max(0, n - i * (1 if n > g else 0)) for i in range(g)] for n in lengths])
        self.cap = int(self.n.max()) + t + spare
        b, cap = self.b, self.cap

        def noise(*s):
            return torch.randn(s, generator=gen).to(dtype)

        k, v = noise(b, g, cap, d), noise(b, g, cap, d)
        pos = torch.from_numpy(rng.integers(0, 1 << 20, size=(b, g, cap)).astype(np.int32))
        w = torch.rand((b, g, cap), generator=gen)
        for i in range(b):
            for j in range(g):
                n = self.n[i, j]
                pos[i, j, :n] = torch.from_numpy(rng.permutation(4 * n)[:n].astype(np.int32))
                k[i, j, n:] = float("nan")
                v[i, j, n:] = float("nan")
                w[i, j, n:] = float("nan")
        first = 4 * max(lengths) + 1
        self.tree_words = None
        if tree == "random":
            self.tree_words = [random_tree(rng, t) for _ in range(b)]
        elif tree == "empty rows":                       # some tokens see nothing of the new ones
            self.tree_words = [[m if i % 3 else 0 for i, m in enumerate(random_tree(rng, t))] for _ in range(b)]
        depths = [np.arange(t) if self.tree_words is None else
                  np.array([max(0, bin(m).count("1") - 1) for m in self.tree_words[i]]) for i in range(b)]
        self.q = (noise(b, t, h, d).float() * spread).to(dtype)
        self.k_new, self.v_new = noise(b, t, g, d), noise(b, t, g, d)
        self.new_pos = torch.from_numpy(np.stack([first + x for x in depths]).astype(np.int32))
        self.scale, self.softcap = 1.0 / d ** 0.5, softcap
        self.slopes = torch.from_numpy((2.0 ** (-8.0 * (np.arange(h) + 1) / h)).astype(np.float32)) if distance else None
        self.k, self.v, self.pos, self.w = k, v, pos, w
        self.device, self.dtype = device, dtype

        def dev(x):
            return x.to(device)

        if token_major:                                  # [batch, capacity, heads, d], seen as [batch, heads, capacity, d]
            self.dk = dev(k.transpose(1, 2).contiguous()).transpose(1, 2)
            self.dv = dev(v.transpose(1, 2).contiguous()).transpose(1, 2)
            fused = torch.full((b, t, h + 2 * g + 1, d), float("nan"), dtype=dtype)
            fused[:, :, :h], fused[:, :, h:h + g], fused[:, :, h + g:h + 2 * g] = self.q, self.k_new, self.v_new
            fused = dev(fused)
            self.dq, self.dk_new, self.dv_new = fused[:, :, :h], fused[:, :, h:h + g], fused[:, :, h + g:h + 2 * g]
        else:
            self.dk, self.dv, self.dq, self.dk_new, self.dv_new = dev(k), dev(v), dev(self.q), dev(self.k_new), dev(self.v_new)
        self.dpos, self.dw, self.dlen = dev(pos), dev(w), dev(torch.from_numpy(self.n.astype(np.int32)))
        self.dnew_pos = dev(self.new_pos)
        self.dslopes = dev(self.slopes) if distance else None
        self.dtree = (dev(torch.tensor([[signed(m) for m in row] for row in self.tree_words], dtype=torch.int64))
                      if self.tree_words else None)
        self.out = torch.full((b, t, h, d), 7.0, dtype=dtype, device=device)
        self.lse = torch.full((b, t, h), 7.0, device=device)

    def cache(self):
        from paper_2604_06746_b200 import binding
        return binding.Cache(self.dk, self.dv, self.dpos, self.dw, self.dlen)

    def context(self):
        from paper_2604_06746_b200 import binding
        return binding.Context(self.h, self.g, self.d, 8, 8, self.dtype, self.device)

    def options(self):
        return dict(tree=self.dtree, softcap=self.softcap, slopes=self.dslopes)

    def attend(self, ctx, cache, ws, **more):
        ctx.attend(cache, self.dq, self.scale, self.out, ws, **{"lse": self.lse, **self.options(), **more})

    def head(self, b, g):
        """float64 (q, k, v, positions) of a KV head, new tokens behind the old ones."""
        n = self.n[b, g]

        def f(x):
            return x.to(torch.float64).numpy()

        k = np.concatenate([f(self.k[b, g, :n]), f(self.k_new[b, :, g])])
        v = np.concatenate([f(self.v[b, g, :n]), f(self.v_new[b, :, g])])
        pos = np.concatenate([self.pos[b, g, :n].numpy(), self.new_pos[b].numpy()])
        return f(self.q[b, :, g * self.group:(g + 1) * self.group]), k, v, pos

    def reference(self, b, g):
        q, k, v, pos = self.head(b, g)
        sl = None if self.slopes is None else self.slopes.numpy()[g * self.group:(g + 1) * self.group]
        masks = None if self.tree_words is None else self.tree_words[b]
        return D.attend(q, k, v, pos, int(self.n[b, g]), self.scale, self.softcap, sl, masks)

    def logit_error(self, b, g):
        """Bound of a logit's error in fp32: d products and sums of the dot product, each off by 2^-24 of the sum of absolute
        values, a few more operations of 2^-24 on the result; tanh through an exponential of 2^-22 and a division; the bias
        rounded like its size."""
        q, k, _, pos = self.head(b, g)
        k = np.where(np.isfinite(k), k, 0.0)
        dots = float((np.abs(q).max(axis=(0, 1)) @ np.abs(k).T).max()) * self.scale
        e = 2.0 ** -24 * (self.d + 8) * dots + 2.0 ** -20 * self.softcap
        if self.slopes is not None:
            far = float(pos.max()) - float(pos.min())
            e += 2.0 ** -22 * float(self.slopes[g * self.group:(g + 1) * self.group].max()) * far
        return e

    def check_attention(self, rows=None):
        """out and lse against the 64-bit statement.  out: each p is rounded to storage for its product with V (half a step; fp32 is
        not rounded), the result once more; a logit's error e changes p by e, relative, twice (p itself and the sum); 2^-20
        stands for the exponential, the sums in fp32 and the merging of partial results."""
        half = torch.finfo(self.dtype).eps / 2
        keep = slice(None) if rows is None else rows
        out, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        for b in range(self.b):
            for g in range(self.g):
                o, l, p = self.reference(b, g)
                v = self.head(b, g)[2]
                mass = np.einsum("tgn,nd->tgd", p, np.where(np.isfinite(v), np.abs(v), 0.0), optimize=True)
                e = self.logit_error(b, g)
                go, gl = out[b, :, g * self.group:(g + 1) * self.group], lse[b, :, g * self.group:(g + 1) * self.group]
                go, gl, o, l, mass = (x[keep] for x in (go, gl, o, l, mass))
                tol = half * (mass * (self.dtype != torch.float32) + np.abs(o)) + (2 * e + 2.0 ** -20) * mass + 1e-30
                assert np.isfinite(go).all(), (b, g)
                assert (np.abs(go - o) <= tol).all(), (b, g, np.abs(go - o).max(), (np.abs(go - o) / tol).max())
                none = np.isneginf(l)
                assert np.array_equal(np.isneginf(gl), none), (b, g)
                assert (np.abs(gl - l)[~none] <= e + 2.0 ** -20 * (1 + np.abs(l[~none]))).all(), (b, g)
