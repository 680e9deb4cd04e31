"""Tree attention and the weights of its keys where a workgroup walks: several stages of keys in one part, in every form of the kernels
(up to 32 rows per KV head, up to 64, more; heads of 192 and 256 in the straight-line form), several tiles of rows in one workgroup."""
import numpy as np
import pytest
import torch

from paper_2602_16052_amd import binding as mb

from attention_common import Batch, f64
from test_gpu_attention import oracle_64

pytestmark = pytest.mark.gpu

TYPES = [(dt, D) for dt in ("bf16", "f32") for D in (64, 96, 128, 192, 256)]
KINDS = ["tree", "chain", "empty"]


def ragged(S, T, n):
    """Trees of T rows and fewer, one empty; caches of n entries and fewer, one of none, one that ends with a stage."""
    trees, lens = [max(1, T - 3 * s) for s in range(S)], [n - (n // S) * s // 2 for s in range(S)]
    trees[S // 2], lens[-1], lens[1] = 0, 0, lens[1] // 128 * 128
    return trees, lens


# ---- attention: one part per sequence (512 workgroups or more), 4 to 19 stages

@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("S,T,n", [(16, 16, 333), (16, 31, 333), (8, 70, 500)])
def test_stages_of_whole_sequences(dtype, D, kind, S, T, n):
    b = Batch(dtype, 64, 32, D, *ragged(S, T, n), kind=kind, fused=T == 31, pad=3, seed=D + T)
    b.check(*b.attention(), oracle_64(b))


# ---- attention: parts of 3 to 18 stages, joined

@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("trees,lens", [([16, 11], [9001, 8700]), ([31, 31], [9001, 8700]), ([40, 33, 7], [6001, 3000, 0])])
def test_stages_of_parts(dtype, D, kind, trees, lens):
    b = Batch(dtype, 16, 8, D, trees, lens, kind=kind, seed=D + trees[0])
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 256), ("f32", 128)])
@pytest.mark.parametrize("T", [16, 31, 70])
def test_lengths_far_below_their_bound(dtype, D, T):
    """max_len is the capacity, as where lengths grow under a captured call."""
    b = Batch(dtype, 16, 8, D, [T, T // 2], [150, 33], seed=T, room=20000)
    b.args["max_len"] = None
    b.check(*b.attention(), oracle_64(b))


def rising(b, n):
    """Scores that grow along the cache: every stage raises the maximum of every row."""
    first = torch.from_numpy(b.off[:-1]).cuda()
    ramp = torch.linspace(0.05, 1.0, b.kc.shape[2], device="cuda")
    q = b.q[first].reshape(len(b.trees), b.Hk, -1, b.D)[:, :, 0]
    b.kc.copy_((q[:, :, None, :].float() * 0.3 + b.kc.float() * 0.2) * ramp[None, None, :, None])
    b.kc[:, :, n:] = float("nan")


@pytest.mark.parametrize("dtype,D,T", [("bf16", 64, 16), ("bf16", 128, 31), ("bf16", 192, 70), ("bf16", 256, 70), ("f32", 128, 16),
                                       ("f32", 64, 31), ("f32", 96, 70)])
@pytest.mark.parametrize("q_scale", [0.1, 12.0])
def test_maxima_that_rise_with_every_stage(dtype, D, T, q_scale):
    b = Batch(dtype, 64, 32, D, [T] * 16, [577] * 16, seed=D, q_scale=q_scale)
    rising(b, 577)
    b.check(*b.attention(), oracle_64(b))


# ---- heads of 192 and 256, more than 64 rows: the straight-line form

WIDE_LENS = [577, 512, 129, 64, 63, 0, 320, 448]  # whole tiles of 64: 9, 8, 2, 1, 0, 0, 5, 7


@pytest.mark.parametrize("D", [192, 256])
@pytest.mark.parametrize("kind", KINDS)
def test_long_heads_in_one_part(D, kind):
    b = Batch("bf16", 64, 32, D, [70, 69, 0, 70, 64, 65, 33, 70], WIDE_LENS, kind=kind, seed=D)
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("D", [192, 256])
@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("trees,lens", [([70], [4500]), ([70, 41], [4500, 2111]), ([131], [9000])])
def test_long_heads_over_parts_of_a_long_cache(D, kind, trees, lens):
    b = Batch("bf16", 32, 16, D, trees, lens, kind=kind, seed=D + len(trees))
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("D", [192, 256])
def test_long_heads_in_chains_of_many_tiles(D):
    b = Batch("bf16", 64, 32, D, [330, 200], [0, 130], kind="chain", seed=D)
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("D", [192, 256])
def test_long_heads_and_values_that_are_not_finite(D):
    b = Batch("bf16", 64, 32, D, [70] * 8, WIDE_LENS, seed=D, room=0)
    first = b.off[:-1]
    want = oracle_64(b)
    for t, col in ((3, 5), (69, 9)):
        b.vt[torch.from_numpy(first + t).cuda(), :, col] = float("nan" if t == 3 else "inf")
    for s, n in enumerate(WIDE_LENS):
        if n:
            b.vc[s, :, n - 1, 7], b.vc[s, :, n // 3, D - 1] = -float("inf"), float("inf")
    out, lse = b.attention()
    got = f64(out)
    for s, n in enumerate(WIDE_LENS):
        rows = np.arange(first[s], first[s] + 70)
        for t, col, is_it in ((3, 5, np.isnan), (69, 9, np.isposinf)):
            see = rows[b.sees[s][:, t]]
            assert is_it(got[see][:, :, col]).all()
            got[see, :, col] = want[0][see, :, col]
        if n:
            assert np.isneginf(got[rows][:, :, 7]).all() and np.isposinf(got[rows][:, :, D - 1]).all()
            got[rows, :, 7], got[rows, :, D - 1] = want[0][rows, :, 7], want[0][rows, :, D - 1]
    b.check(torch.from_numpy(got), lse, want)
    # scores that are no numbers stay in their sequence
    b = Batch("bf16", 64, 32, D, [70] * 8, WIDE_LENS, seed=D, room=0)
    b.kc[0, :, 70] = float("nan")
    out = b.attention()[0]
    assert torch.isnan(out[:70]).all() and torch.isfinite(out[70:]).all()


# ---- weights: 5 to 44 tiles of rows in a workgroup

def weights_64(b, lse, rw):
    """The weights of cached keys [S, Hk, capacity] and of the trees' [M, Hk] in 64 bits, and the same of |row_weight|."""
    G, D = b.H // b.Hk, b.D
    cw = torch.zeros((2, len(b.trees), b.Hk, b.desc.capacity), dtype=torch.float64, device="cuda")
    tw = torch.zeros((2, b.M, b.Hk), dtype=torch.float64, device="cuda")
    scale = float(np.float32(b.scale))
    for s, (n, T) in enumerate(zip(b.lens, b.trees)):
        if T == 0:
            continue
        rows = slice(int(b.off[s]), int(b.off[s + 1]))
        k = torch.cat([b.kc[s, :, :n], b.kt[rows].transpose(0, 1)], dim=1).double()
        q, l, r = (x.double().reshape(T, b.Hk, G, -1).permute(1, 2, 0, 3).reshape(b.Hk, G * T, -1).contiguous()
                   for x in (b.q[rows], lse[rows], rw[rows, None].expand(T, b.H)))
        sees = torch.cat([torch.ones((T, n), dtype=torch.bool), torch.from_numpy(np.asarray(b.sees[s]))], dim=1).cuda().repeat(G, 1)
        p = torch.exp(scale * torch.matmul(q, k.transpose(1, 2).contiguous()) - l)
        p = torch.where(sees & torch.isfinite(l) & (r != 0), p, 0.0)
        for i, x in enumerate((r, r.abs())):
            w = (p * torch.where(torch.isfinite(x), x, 0.0)).sum(dim=1)
            cw[i, s, :, :n], tw[i, rows] = w[:, :n], w[:, n:].transpose(0, 1)
    return cw, tw


def check_weights_64(b, got, lse, rw, w_in=None, decay=0.0):
    cw, tw = weights_64(b, lse, rw)
    top = float(torch.where(torch.isfinite(lse), lse.abs(), 0.0).max())
    # as in test_gpu_cache.check_weights: a score's error, that of lse and of the exponential, fp32 sums over the rows
    rel = b.score_error(oracle_64(b)[3].max()) + (top + 4) * 2.0 ** -22 + (max(b.trees) * b.H // b.Hk + 64) * 2.0 ** -23
    for s, n in enumerate(b.lens):
        old = 0.0 if w_in is None else decay * w_in[s, :, :n].double()
        err = (got[0][s, :, :n].double() - cw[0, s, :, :n] - old).abs()
        assert bool((err <= (cw[1, s, :, :n] + (0.0 if w_in is None else old.abs())) * rel + 1e-37).all()), f"sequence {s}"
    used = slice(0, int(b.off[-1]))
    assert bool(((got[1].double() - tw[0]).abs()[used] <= tw[1][used] * rel + 1e-37).all())


def weights(b, lse, **kw):
    return mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **{**b.args, **kw})


# KV heads x tiles of keys fill the card, so that the rows are not split: 7 tiles of rows; 10 (or two parts of 5); 44; two parts of 16
WALKS = [(128, 64, [97], [1200]), (64, 64, [300], [700]), (64, 32, [700, 650], [1000, 333]), (96, 32, [333, 1, 200], [900, 20, 0])]


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,trees,lens", WALKS[:2])
def test_weights_over_tiles_of_rows(dtype, D, kind, H, Hk, trees, lens):
    b = Batch(dtype, H, Hk, D, trees, lens, kind=kind, fused=Hk == H, seed=D)
    lse = b.attention()[1]
    check_weights_64(b, weights(b, lse), lse, torch.ones(b.M, device="cuda"))


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,trees,lens", WALKS[1:])
def test_weights_over_tiles_of_rows_with_rows_that_have_no_part(dtype, D, kind, H, Hk, trees, lens):
    b = Batch(dtype, H, Hk, D, trees, lens, kind=kind, pad=2, seed=D)
    lse = b.attention()[1]
    g = torch.Generator(device="cuda").manual_seed(D)
    rw = torch.rand(b.M, generator=g, device="cuda") - 0.25
    rw[torch.rand(b.M, generator=g, device="cuda") < 0.3] = 0.0
    lse[torch.rand(lse.shape, generator=g, device="cuda") < 0.1] = -float("inf")
    silent = int(b.off[1]) - 40  # behind the first tiles of rows
    rw[silent], lse[silent] = 0.0, float("nan")
    w_in = torch.rand((len(trees), Hk, b.desc.capacity), generator=g, device="cuda")
    got = weights(b, lse, row_weight=rw, cache_w_in=w_in, decay=0.75)
    check_weights_64(b, got, lse, rw, w_in, 0.75)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_weights_of_a_row_that_is_not_finite_behind_the_first_tiles(dtype, D, kind):
    b = Batch(dtype, 64, 64, D, [300], [0], kind=kind, seed=D, room=700)
    b.args["max_len"] = 700
    lse = b.attention()[1]
    rw = torch.ones(b.M, device="cuda")
    t = 260
    lse[t] = float("nan")
    cache_w, tree_w = weights(b, lse)
    seen = torch.from_numpy(b.sees[0][t]).cuda()
    assert torch.isnan(tree_w[seen]).all()
    lse[t] = -float("inf")
    tree_w[seen] = weights(b, lse)[1][seen]
    check_weights_64(b, (cache_w, tree_w), lse, rw)
