"""Helpers of the tests of the calls around a serving step: pools of pages with random tables, their values as float64, tolerances."""
import numpy as np
import torch

from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb

from attention_common import CODE, HALF_STEP, TORCH, f64, i32

KIND = {"plain": mb.CACHE_PLAIN, "i8": mb.CACHE_I8, "e4m3": mb.CACHE_E4M3}


def values64(t):
    """Stored values of a tensor of any type as float64."""
    return f64(t.float() if t.dtype == torch.float8_e4m3fn else t)


def table(entries, page, rng, spare=3, width=None):
    """(page_table int32 [n_seq, width], pages of the pool): every sequence's pages anywhere in the pool, -1 where there is none."""
    need = [-(-n // page) for n in entries]
    pool = sum(need) + spare
    order = rng.permutation(pool)
    rows = np.full((len(entries), max(max(need), 1) if width is None else width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        rows[s, :n] = order[at:at + n]
        at += n
    return rows, pool


def entries_of(cache, layer, rows, lens, which):
    """Per sequence the values [Hk, n, D] of its entries, as float64."""
    pages, scale = (cache.k_pages, cache.k_scale) if which == "k" else (cache.v_pages, cache.v_scale)
    v = values64(pages[layer])
    if scale is not None:
        v = v * f64(scale[layer])[..., None]
    size, out = v.shape[2], []
    for s, n in enumerate(lens):
        got = np.concatenate([v[p] for p in rows[s][:-(-n // size)]], axis=1) if n else np.zeros((v.shape[1], 0, v.shape[3]))
        out.append(got[:, :n])
    return out


class Pool:
    """A pool of random keys and values with a table, of `layers` layers; what lies behind the lengths is NaN."""

    def __init__(self, dtype, code, Hk, D, lens, page, seed=0, layers=1, H=None, scale=None, capacity=None, width=None):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.code, self.lens, self.page = dtype, code, list(lens), page
        self.rows, n = table(lens, page, rng, width=width)
        self.desc = mb.AttnDesc(H or Hk, Hk, D, capacity or max(max(lens), 1) + 5, CODE[dtype], scale)
        self.scale = D ** -0.5 if scale is None else scale
        self.cache = mb.alloc_paged_cache(self.desc, KIND[code], n, page, torch.from_numpy(self.rows).cuda(), layers)
        c = self.cache
        for pages, scales in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
            x = torch.randn(pages.shape, generator=gen, device="cuda")
            if code == "plain":
                pages.copy_(x)
            elif code == "i8":
                pages.copy_((x * 40).clamp(-127, 127).round())
                scales.copy_(torch.rand(scales.shape, generator=gen, device="cuda") * 0.04 + 0.005)
            else:
                pages.copy_((x * 60).to(torch.float8_e4m3fn))
                scales.copy_(torch.exp2(torch.randint(-8, -4, scales.shape, generator=gen, device="cuda").float()))
        self.cache_len = i32(lens)

    def poison(self):
        """NaN in every place that holds no entry of a sequence."""
        c, live = self.cache, np.zeros((self.cache.k_pages.shape[1], self.page), dtype=bool)
        for s, n in enumerate(self.lens):
            for e in range(n):
                live[self.rows[s][e // self.page], e % self.page] = True
        dead = torch.from_numpy(~live).cuda()[None, :, None, :]
        for pages, scales in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
            if self.code == "plain":
                pages.masked_fill_(dead[..., None], float("nan"))
            else:
                if self.code == "e4m3":
                    pages.view(torch.int8).masked_fill_(dead[..., None], 0x7f)
                scales.masked_fill_(dead, float("nan"))
        return self

    def values(self, which, layer=0):
        return entries_of(self.cache, layer, self.rows, self.lens, which)

    def check(self, q, out, lse, oracle=None, layer=0):
        if oracle is None:
            oracle = V.attention(f64(q), self.values("k", layer), self.values("v", layer), float(np.float32(self.scale)))
        want, want_lse, bound, spread = oracle
        D, n, u = q.shape[2], max(self.lens), HALF_STEP[self.dtype]
        # a score: products and sums of D terms (a whole step each in the matrix cores), the scales, the exponential's argument
        score = (2 * D + 10) * 2.0 ** -24 * spread
        # weights: what the two parts of a bf16 weight leave (the first is cut off: 2^-7; the second is rounded: 2^-8 of that), of an fp32 one
        # over codes the three parts (2^-8 three times), the value's scale, the scores above and below the line, sums over keys
        rel = (2.0 ** -15 if self.dtype == "bf16" else 2.0 ** -24) + 2.0 ** -23 + 2 * score + 2 * (n + 64) * 2.0 ** -24
        tol = u * np.abs(want) * (1 + 2.0 ** -6) + bound * rel[:, :, None] + 1e-37
        err = np.abs(f64(out) - want)
        assert np.all(err <= tol), f"out off by {np.nanmax(err / tol):.2f} of the bound"
        got = f64(lse)
        seen = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got), ~seen)
        base = np.where(seen, want_lse, 0)
        err = np.abs(np.where(seen, got, 0) - base)
        tol = score + (n + 64) * 2.0 ** -24 + np.abs(base) * 2.0 ** -22 + 1e-37
        assert np.all(err <= tol), f"lse off by {np.max(err / tol):.2f} of the bound"
