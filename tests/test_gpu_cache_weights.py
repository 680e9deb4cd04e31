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
