"""Helpers of the speculative step's tests: caches with known contents, trees, and the definitions in 64 bits."""
import math

import numpy as np
import torch

import paper_2507_17769_b200 as ps

PAGE = 16


class Cache:
    """A poisoned pool with the K, V of requests of kv_len tokens in permuted pages; k, v: per request [kv_len, Hkv, d], as the cache
    holds them (FP8: dequantised, fp32)."""

    def __init__(self, heads, kv_heads, dim, kv_len, seed=0, fp8=False, spare_pages=5, spare_columns=2):
        self.heads, self.kv_heads, self.dim, self.fp8 = heads, kv_heads, dim, fp8
        self.kv_len = np.asarray(kv_len, dtype=np.int32)
        need = (self.kv_len + PAGE - 1) // PAGE
        self.num_pages = int(need.sum()) + spare_pages
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        perm = rng.permutation(self.num_pages)
        table = np.full((len(need), int(need.max()) + spare_columns), -1, dtype=np.int32)  # entries past a sequence's end are never read
        at = 0
        for r, n in enumerate(need):
            table[r, :n] = perm[at:at + n]
            at += n
        self.table = torch.from_numpy(table).cuda()
        self.pa = ps.PagedAttention(heads, kv_heads, dim, self.num_pages, poison=True, kv_dtype=int(fp8))
        self.k = [self.normal(int(n), kv_heads, dim) for n in self.kv_len]
        self.v = [self.normal(int(n), kv_heads, dim) for n in self.kv_len]

    def normal(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.gen, device="cuda") * scale).bfloat16()

    def fill(self):
        """Writes k and v (and, FP8, takes what was stored in their place)."""
        some = [r for r, n in enumerate(self.kv_len) if n > 0]
        self.pa.write(torch.cat([self.k[r] for r in some]), torch.cat([self.v[r] for r in some]), self.table[some].contiguous(), [0] * len(some), self.kv_len[some])
        self.pa.check_pool()
        if self.fp8:
            for r in some:
                self.k[r], self.v[r] = self.stored(r)
        return self

    def stored(self, r):
        """Request r's cache: bf16 as it is, FP8 as codes times scales in fp32 (exact)."""
        n = int(self.kv_len[r])
        if not self.fp8:
            return self.pa.gather(self.table[r], n)
        kc, vc, ks, vs = self.pa.gather_fp8(self.table[r], n)
        return tuple(c.view(torch.float8_e4m3fn).float() * s[..., None] for c, s in ((kc, ks), (vc, vs)))


def tree_masks(n_nodes, words, rng, fan=4):
    """Masks of random trees, a node's parent one of the `fan` before it: int64 [T, words] and per request bool [n, n]."""
    rows, sees_all = [], []
    for n in n_nodes:
        sees = np.eye(n, dtype=bool)
        for i in range(1, n):
            sees[i] |= sees[rng.integers(max(0, i - fan), i)]
        sees_all.append(sees)
        rows.append(pack(sees, words))
    return torch.from_numpy(np.concatenate(rows)).cuda(), sees_all


def pack(sees, words):
    bits = np.zeros((sees.shape[0], 64 * words), dtype=bool)
    bits[:, :sees.shape[1]] = sees
    return np.packbits(bits, axis=1, bitorder="little").view(np.int64)


def tree_reference(cache, q, prior, sees_all):
    """(out, lse, bound of out's error, bound of lse's) in 64 bits.

    Bounds.  The weights that multiply V are rounded to bf16 (2^-8 of each), and so is their sum's share of that where it is taken
    over the rounded ones: 2 * 2^-8 of sum |w v|.  The output's own rounding: 2^-8 of it.  A score is a sum of d products in
    fp32: d * 2^-24 * sum |q k| / sqrt(d); twice that relative in the weights (numerator and sum), once absolute in lse;
    ex2.approx and the logarithm are good to 2^-20, the sums to 2^-18 over the lengths here.
    FP8 cache: the weights times their scales are rounded to f16 (2^-11, and 2^-24 at the least, of values up to 2^8 times V's largest scale); q is the
    sum of two E4M3 numbers over a power of two that brings a row's largest to 224 at least, off by at most half of their smallest
    step, 2^-10; its products are twice as many."""
    outs, lses, bounds, lse_bounds, t = [], [], [], [], 0
    d, group = cache.dim, cache.heads // cache.kv_heads
    for r, sees in enumerate(sees_all):
        n, p = sees.shape[0], int(prior[r])
        k, v = (x[r][: p + n].double().repeat_interleave(group, dim=1).transpose(0, 1) for x in (cache.k, cache.v))
        x = q[t:t + n].double().transpose(0, 1)
        hidden = torch.zeros((n, p + n), dtype=torch.bool, device="cuda")
        hidden[:, p:] = ~torch.from_numpy(sees).cuda()
        # (what is not seen has no part, whatever it holds: row by row where it holds infinities or NaN)
        s = (x @ torch.nan_to_num(k, 0, 0, 0).transpose(1, 2) / math.sqrt(d)).masked_fill(hidden, -math.inf)
        odd = ~torch.isfinite(k).all(-1).all(0)
        if bool(odd.any()):
            s = torch.where((odd & ~hidden)[None], math.nan, s)
        lse = torch.logsumexp(s, dim=2)
        w = torch.where(lse[..., None] == -math.inf, 0.0, (s - torch.where(lse == -math.inf, 0.0, lse)[..., None]).exp())
        fin = torch.nan_to_num(v, 0, 0, 0)
        out = w @ fin
        for key in torch.nonzero(~torch.isfinite(v).all(-1).all(0)).flatten().tolist():
            part = torch.where(hidden[:, key][None, :, None], 0.0, w[:, :, key, None] * (v - fin)[:, key][:, None])
            out = out + torch.where(hidden[:, key][None, :, None] | torch.isfinite(v[:, key])[:, None], 0.0, part)
        weight = w @ fin.abs()
        mag = torch.nan_to_num(k, 0, 0, 0).abs().transpose(1, 2)
        score = (d * 2.0 ** -24 / math.sqrt(d)) * (x.abs() @ mag).masked_fill(hidden, 0).amax(-1)
        rounding = 2.0 ** -7
        if cache.fp8:
            split = x.abs().amax(-1, keepdim=True) * (2.0 ** -10 / 224)
            score = 2 * score + (split.expand_as(x) @ mag).masked_fill(hidden, 0).amax(-1) / math.sqrt(d)
            rounding = 2.0 ** -11
        outs.append(out.transpose(0, 1))
        lses.append(lse.transpose(0, 1))
        bounds.append((2.0 ** -8 * out.abs() + (rounding + 2 * score[..., None] + 2.0 ** -18) * weight + (2.0 ** -13 if cache.fp8 else 0.0)).transpose(0, 1))
        lse_bounds.append((score + 2.0 ** -18 + 2.0 ** -22 * torch.nan_to_num(lse, 0, 0, 0).abs()).transpose(0, 1))
        t += n
    return torch.cat(outs), torch.cat(lses), torch.cat(bounds), torch.cat(lse_bounds)


def check_tree(out, lse, want):
    ref, ref_lse, bound, lse_bound = want
    got = out.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isfinite(got), fine)
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
    over = ((got - ref).abs() - bound)[fine]
    assert float(over.max()) <= 0, "out is %.3e over its bound" % float(over.max())
    if lse is not None:
        fine = torch.isfinite(ref_lse)
        assert torch.equal(lse.double()[~fine], ref_lse[~fine]) or bool(torch.isnan(ref_lse).any())
        over = ((lse.double() - ref_lse).abs() - lse_bound)[fine]
        assert float(over.max() if over.numel() else 0) <= 0, "lse is %.3e over its bound" % float(over.max())
