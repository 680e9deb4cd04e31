"""Rows of moespec_cache_weights that have no part, or one that is not finite, and how exact the weights are."""
import numpy as np
import pytest
import torch

from paper_2602_16052_amd import binding as mb

from attention_common import CODE, TORCH, Batch, f64, i32
from test_gpu_cache import check_weights

pytestmark = pytest.mark.gpu


def call(b, lse, **kw):
    return mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **{**b.args, **kw})


@pytest.mark.parametrize("dtype,H,Hk,T", [("bf16", 4, 2, 12), ("bf16", 6, 1, 70), ("f32", 4, 2, 40)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_rows_of_weight_zero_have_no_part(dtype, H, Hk, T, kind):
    """Rejected tokens, whatever their queries and statistics hold."""
    b = Batch(dtype, H, Hk, 64, [T], [90], kind=kind, seed=T)
    lse = b.attention()[1]
    rw = torch.rand(T, device="cuda") + 0.25
    rw[3], rw[5], rw[T - 1], rw[7] = 0.0, -0.0, 0.0, 0.0
    clean = lse.clone()
    clean[[3, 5, T - 1, 7]] = -float("inf")  # for the oracle: no part
    b.q[3], lse[3] = float("nan"), float("nan")
    lse[5], lse[7] = -1e30, float("inf")  # weights of infinity and of nothing
    b.q[T - 1] = float("inf")
    got = call(b, lse, row_weight=rw)
    b.q[[3, T - 1]] = 0
    check_weights(b, *got, clean, rw)


@pytest.mark.parametrize("dtype,H,Hk,T", [("bf16", 4, 2, 12), ("bf16", 6, 1, 70), ("f32", 4, 2, 40)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("what", ["lse", "weight", "infinite weight"])
def test_rows_that_are_not_finite_reach_only_keys_that_they_see(dtype, H, Hk, T, kind, what):
    b = Batch(dtype, H, Hk, 64, [T], [0], kind=kind, seed=T)
    lse = b.attention()[1]
    rw = torch.rand(T, device="cuda") + 0.25
    t = T // 2
    clean = lse.clone()
    clean[t] = -float("inf")
    if what == "lse":
        lse[t] = float("nan")
    else:
        rw[t] = float("nan") if what == "weight" else -float("inf")
    cache_w, tree_w = call(b, lse, row_weight=rw)
    seen = torch.from_numpy(b.sees[0][t]).cuda()
    assert 0 < int(seen.sum()) < T
    assert bool((torch.isneginf(tree_w[seen]) if what == "infinite weight" else torch.isnan(tree_w[seen])).all())
    rw[t] = 1.0
    want = call(b, clean, row_weight=rw)[1]
    assert torch.isfinite(want).all()
    tree_w[seen] = want[seen]
    check_weights(b, cache_w, tree_w, clean, rw)


def test_a_row_with_an_lse_of_nan_reaches_its_own_sequence_and_heads():
    b = Batch("bf16", 4, 2, 64, [9, 6], [70, 50], seed=1)
    lse = b.attention()[1]
    lse[3, 1] = float("nan")  # a query head of the first KV head
    cache_w, tree_w = call(b, lse)
    assert torch.isnan(cache_w[0, 0, :70]).all() and torch.isfinite(cache_w[0, 1, :70]).all()
    assert torch.isfinite(cache_w[1, :, :50]).all() and torch.isfinite(tree_w[:, 1]).all() and torch.isfinite(tree_w[9:]).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 192), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("level", [0.0, 50.0, -50.0])
def test_weights_of_single_rows_are_as_exact_as_their_scores(dtype, D, level):
    """One row per KV head, whose scores have no rounding of their own (one product of two short numbers): what is left is the
    exponential's.  With x the exponent in units of log 2: its rounding and that of its factor, |x| half steps each (times ln 2), two
    half steps of the exponential, one each of the row's weight, its correction and the product, and one for what is of second order."""
    S, Hk, n, scale = 8, 16, 200, 0.3
    g = torch.Generator(device="cuda").manual_seed(D)
    near = (level / scale / 16 + torch.rand((S, Hk, n), generator=g, device="cuda")).bfloat16()  # scores within some 5 of each other
    q, kt, kc = (torch.zeros(s, dtype=TORCH[dtype], device="cuda") for s in ((S, Hk, D), (S, Hk, D), (S, Hk, n, D)))
    q[..., 0], kc[..., 0] = 16.0, near.to(TORCH[dtype])
    score = float(np.float32(scale)) * 16.0 * f64(near)
    lse = torch.from_numpy(score.max(axis=2) + 0.37).float().cuda()
    rw = torch.rand(S, generator=g, device="cuda") + 0.5
    desc = mb.AttnDesc(Hk, Hk, D, n, CODE[dtype], scale)
    cache_w, _ = mb.moespec_cache_weights(desc, q, kt, kc, i32([n] * S), lse, tree_off=i32(np.arange(S + 1)), max_tree=1, row_weight=rw)
    d = score - f64(lse)[:, :, None]
    want = f64(rw)[:, None, None] * np.exp(d)
    x = np.abs(d) / np.log(2.0)
    assert x.max() < 9
    err = np.abs(f64(cache_w) - want) / want / 2.0 ** -24
    assert np.all(err <= 2 * np.log(2.0) * x + 6), np.max(err / (2 * np.log(2.0) * x + 6))
