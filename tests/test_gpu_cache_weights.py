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
