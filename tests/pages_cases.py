"""Inputs and comparisons shared by the tests of the paged cache in 8 bits and of rotary positions."""
import numpy as np
import torch

from oracle import pages_oracle as P

SHAPES = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 2, 64), "wide": (24, 1, 64), "single": (3, 3, 128), "many": (20, 1, 128)}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative
# What a rotated element may be off before it is rounded, relative to amplitude (|a| + |b|).  The angle has 24 bits (pi 2^-24 = 2^-22.3); cosine
# and sine are off by 2^-21.2 (bf16) or an ulp, 2^-23 (fp32); products, sum and amplitude are rounded, 2^-24 each.
TURN = {torch.bfloat16: 2.0 ** -20, torch.float32: 2.0 ** -21.5}


class Paged:
    """Pages of `lengths` tokens in a random order of a pool, all other slots and pages full of NaN codes; host mirrors of the codes."""

    def __init__(self, device, shape, lengths, page=64, spare=70, seed=0, token_major=False, dtype=torch.bfloat16, v_spread=1.0, shared=False):
        from paper_2604_06746_b200 import binding
        h, g, d = SHAPES[shape]
        self.h, self.g, self.d, self.b, self.page, self.n, self.dtype, self.device = h, g, d, len(lengths), page, list(lengths), dtype, device
        self.group = h // g
        rng = self.rng = np.random.default_rng(seed)
        cols = (max(lengths) + spare + page - 1) // page
        pool = self.b * cols + 2
        self.table = rng.permutation(pool)[:self.b * cols].reshape(self.b, cols).astype(np.int32)
        if shared:                                         # the second sequence begins with the first one's full pages
            self.table[1, :min(lengths[:2]) // page] = self.table[0, :min(lengths[:2]) // page]
        self.slots = cols * page
        self.codes = {x: np.full((pool, g, page, d), 127, dtype=np.uint8) for x in "kv"}
        self.exps = {x: np.full((pool, g, page // 16), 128, dtype=np.int64) for x in "kv"}      # (no scale: byte 255)
        for i, n in enumerate(lengths):
            for j in range(g):
                for x, spread in (("k", 1.0), ("v", v_spread)):
                    rows = rng.standard_normal((n, d)) * np.exp(rng.standard_normal((n, 1)) * (0.3 if spread == 1.0 else spread))
                    c, e = P.append(np.full((self.slots, d), 127, dtype=np.uint8), [128] * (self.slots // 16), 0, rows)
                    for p in range(cols):
                        if p * page < n:
                            self.codes[x][self.table[i, p], j] = c[p * page:(p + 1) * page]
                            self.exps[x][self.table[i, p], j] = e[p * page // 16:(p + 1) * page // 16]

        def pool_of(c):
            t = torch.from_numpy(c).to(device)
            if token_major:                                # [pages, slots, heads, d], seen as [pages, heads, slots, d]
                t = t.transpose(1, 2).contiguous().transpose(1, 2)
            return t.view(torch.float8_e4m3fn)

        def scales_of(e):
            return torch.from_numpy((e + 127).astype(np.uint8)).to(device).view(torch.float8_e8m0fnu)

        self.dlen = torch.tensor(lengths, dtype=torch.int32, device=device)
        self.dtable = torch.from_numpy(self.table).to(device)
        self.pages = binding.Pages(pool_of(self.codes["k"]), pool_of(self.codes["v"]), scales_of(self.exps["k"]), scales_of(self.exps["v"]),
                                   self.dtable, self.dlen)
        self.ctx = binding.Context(h, g, d, 8, 8, dtype, device)

    def noise(self, *shape, spread=1.0):
        x = torch.from_numpy((self.rng.standard_normal(shape) * spread).astype(np.float32)).to(self.dtype)
        return x, x.to(self.device)

    def head(self, x, b, g, codes=None, exps=None):
        """(codes [slots, d], exponents) of one head of one sequence."""
        c, e = (codes or self.codes)[x], (exps or self.exps)[x]
        return np.concatenate([c[p, g] for p in self.table[b]]), np.concatenate([e[p, g] for p in self.table[b]])

    def read(self):
        """(codes, exponents) as the device has them now."""
        torch.cuda.synchronize()
        t = self.pages
        codes = {"k": t.k.view(torch.uint8).cpu().numpy().copy(), "v": t.v.view(torch.uint8).cpu().numpy().copy()}
        exps = {"k": t.k_scales.view(torch.uint8).cpu().numpy().astype(np.int64) - 127,
                "v": t.v_scales.view(torch.uint8).cpu().numpy().astype(np.int64) - 127}
        return codes, exps


def check_attend(p, q, out, lse, counts, scale, softcap=0.0, codes=None, exps=None, only=None):
    """out, lse of the rows q [batch, new, H, d] (host, of p's dtype) against the statement on the codes that the cache holds."""
    q, out, lse = q.double().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    t = q.shape[1]
    for b in range(p.b) if only is None else only:
        c = t if counts is None else counts[b]
        assert (out[b, c:] == 0).all() and (lse[b, c:] == -np.inf).all()
        if c == 0:
            continue
        for g in range(p.g):
            heads, keys = slice(g * p.group, (g + 1) * p.group), p.n[b] + c
            v_codes, v_exps = p.head("v", b, g, codes, exps)
            k, v = (P.values(*p.head(x, b, g, codes, exps))[:keys] for x in "kv")
            o, l, prob = P.attend(q[b, :c, heads], k, v, p.n[b], scale, softcap)
            size = prob @ np.abs(v)
            # scores: 24 bits of sums of d products, and of the result in bits (2^-23 |x|)
            off = abs(scale) * (np.abs(q[b, :c, heads]) @ np.abs(k).T).max(axis=-1) * 2.0 ** -20 + 2.0 ** -22 * (1 + np.abs(l))
            # weights are fp16, half a step of whose 11 bits is 2^-11 of the value (fp32 storage: two of them, 2^-22); exponentials 2^-22, sums
            # of up to 2^14 terms in order 2^-18
            weights = 2.0 ** -11 if p.dtype == torch.bfloat16 else 2.0 ** -22
            # a weight p 2^e stands in fp16 next to the largest such one, which is 2^7 or more: steps of 2^-24 where it is below 2^-14, so half a
            # step of 2^-32 of the largest for every code
            largest = (prob * 2.0 ** np.repeat(v_exps.astype(np.float64), 16)[:keys]).max(axis=-1)
            floor = 2.0 ** -32 * largest[..., None] * np.abs(P.CODES[v_codes[:keys]]).sum(axis=0)
            e = 1.01 * HALF[p.dtype] * np.abs(o) + (weights + 2.0 ** -18 + 2 * off[..., None]) * size + floor
            bad = ~(np.abs(out[b, :c, heads] - o) <= e)
            assert not bad.any(), (b, g, np.abs(out[b, :c, heads] - o)[bad].max(), e[bad].max(), np.argwhere(bad)[:4])
            assert (np.abs(lse[b, :c, heads] - l) <= off + 2.0 ** -18).all(), (b, g)
