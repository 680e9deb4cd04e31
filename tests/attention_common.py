"""Helpers of the tests of tree attention and its cache: random batches on the GPU, their stored values as float64, tolerances."""
import numpy as np
import torch

from oracle import attention_oracle as A
from paper_2602_16052_amd import binding as mb

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": mb.BF16, "f32": mb.F32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def random_tree(rng, n, back=6):
    return A.ancestors([t - rng.integers(1, back + 1) if t and rng.random() < 0.9 else -1 for t in range(n)] if n else []) \
        if n else np.zeros((0, 0), dtype=bool)


class Batch:
    """A batch of trees over caches.  trees, lens: rows and entries per sequence; pad: token rows of no sequence behind the last."""

    def __init__(self, dtype, H, Hk, D, trees, lens, kind="tree", fused=False, pad=0, room=5, seed=0, q_scale=2.0, scale=None):
        self.dtype, self.H, self.Hk, self.D, self.trees, self.lens, self.kind = dtype, H, Hk, D, trees, lens, kind
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dt = TORCH[dtype]
        self.off = np.concatenate([[0], np.cumsum(trees)]).astype(np.int64)
        M = self.M = int(self.off[-1]) + pad
        S, cap = len(trees), max(max(lens), 1) + room
        randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
        if fused:
            qkv = randn(M, H + 2 * Hk, D)
            qkv[:, :H] *= q_scale
            qkv = qkv.to(dt)
            self.q, self.kt, self.vt = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:
            self.q, self.kt, self.vt = (randn(M, H, D) * q_scale).to(dt), randn(M, Hk, D).to(dt), randn(M, Hk, D).to(dt)
        self.kc, self.vc = randn(S, Hk, cap, D).to(dt), randn(S, Hk, cap, D).to(dt)
        for s, n in enumerate(lens):  # behind the entries: what a kernel must not let in
            self.kc[s, :, n:] = float("nan")
            self.vc[s, :, n:] = float("nan")
        self.sees = [A.chain(n) if kind == "chain" else random_tree(rng, n) for n in trees]
        if kind == "empty":  # some rows see nothing of their tree
            for m in self.sees:
                m[rng.random(len(m)) < 0.5] = False
        self.max_tree, self.max_len = max(max(trees), 1), max(lens)
        self.mask = None if kind == "chain" else torch.from_numpy(A.pack(self.sees, M, self.max_tree, fill=1)).cuda()
        self.desc = mb.AttnDesc(H, Hk, D, cap, CODE[dtype], scale)
        self.scale = D ** -0.5 if scale is None else scale
        self.args = dict(tree_off=i32(self.off), tree_mask=self.mask, max_tree=self.max_tree, max_len=self.max_len)
        self.cache_len = i32(lens)

    def attention(self, **kw):
        return mb.moespec_tree_attention(self.desc, self.q, self.kt, self.vt, self.kc, self.vc, self.cache_len,
                                         **{**self.args, **kw})

    def oracle(self):
        return A.attention(f64(self.q), f64(self.kt), f64(self.vt), f64(self.kc), f64(self.vc), self.lens, self.off, self.sees,
                           float(np.float32(self.scale)))

    def score_error(self, spread):
        """Bound on the error of a score in fp32: products and sums of D terms, the scale, the exponential's argument; the sums of
        the matrix cores are allowed a whole step each."""
        return (2 * self.D + 8) * 2.0 ** -24 * spread

    def check(self, out, lse, oracle=None):
        want, want_lse, bound, spread = oracle or self.oracle()
        n, u, used = max(self.lens) + max(self.trees), HALF_STEP[self.dtype], slice(0, int(self.off[-1]))
        # weights: their rounding (bf16), the error of a score on both sides of the division, fp32 sums over the keys
        rel = (u if self.dtype == "bf16" else 0.0) + 2 * self.score_error(spread) + 2 * (n + 64) * 2.0 ** -24
        tol = u * np.abs(want) * (1 + 2.0 ** -6) + bound * rel[:, :, None] + 1e-37
        got, got_lse = f64(out), f64(lse)
        err = np.abs(got - want)[used]
        assert np.all(err <= tol[used]), f"out off by {np.nanmax(err / tol[used]):.2f} of the bound"
        seen = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got_lse[used]), ~seen[used])
        tol = self.score_error(spread) + (n + 64) * 2.0 ** -24 + np.abs(np.where(seen, want_lse, 0)) * 2.0 ** -22
        err = np.abs(np.where(seen, got_lse - np.where(seen, want_lse, 0), 0))[used]
        assert np.all(err <= tol[used]), f"lse off by {np.max(err / tol[used]):.2f} of the bound"
