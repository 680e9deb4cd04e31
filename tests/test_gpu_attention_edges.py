"""Tree attention where a cache, a tree or a row ends: values that are not finite in last places, over one stage of keys and several."""
import numpy as np
import pytest
import torch

from paper_2602_16052_amd import binding as mb

from attention_common import Batch, f64
from test_gpu_attention import oracle_64

pytestmark = pytest.mark.gpu


def check_odd_ends(b):
    """An infinity in the last value of every tree, another in the last entry of every cache (which fills it: no room behind it), a NaN
    in the tree's middle: each reaches the rows that see it and no other, and nothing else changes."""
    want = oracle_64(b)
    tree, cache, middle = (np.zeros(b.M, dtype=bool) for _ in range(3))
    for s, (T, n) in enumerate(zip(b.trees, b.lens)):
        first = int(b.off[s])
        if T:
            b.vt[first + T - 1, :, 3] = float("inf")
            b.vt[first + T // 2, :, 5] = float("nan")
            tree[first:first + T], middle[first:first + T] = b.sees[s][:, T - 1], b.sees[s][:, T // 2]
        if n:
            b.vc[s, :, n - 1, 7] = float("-inf")
            cache[first:first + T] = True
    out, lse = b.attention()
    got, want_out = f64(out), want[0]
    assert np.all(got[tree][:, :, 3] == np.inf) and np.all(got[cache][:, :, 7] == -np.inf) and np.all(np.isnan(got[middle][:, :, 5]))
    for rows, col in ((tree, 3), (middle, 5), (cache, 7)):
        got[rows, :, col] = want_out[rows, :, col]
    b.check(torch.from_numpy(got), lse, want)


# rows of a KV head: up to 32, up to 64, more; trees that end inside of a stage of 32, 64 and 128 keys
@pytest.mark.parametrize("dtype,H,Hk,D,trees,lens", [
    ("bf16", 2, 2, 64, [9], [45]), ("bf16", 8, 4, 128, [31, 5], [161, 0]), ("bf16", 8, 4, 96, [45, 33], [200, 129]),
    ("bf16", 8, 2, 64, [200, 71], [90, 1]), ("bf16", 8, 4, 192, [70, 3], [90, 600]), ("bf16", 6, 2, 256, [97], [333]),
    ("f32", 4, 4, 64, [21], [77]), ("f32", 4, 2, 128, [31], [65]), ("f32", 6, 2, 96, [45, 33], [100, 3]), ("f32", 2, 1, 256, [9], [50])])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_values_that_are_not_finite_in_last_places(dtype, H, Hk, D, trees, lens, kind):
    check_odd_ends(Batch(dtype, H, Hk, D, trees, lens, kind=kind, fused=True, room=0, seed=D + H))


# in one part per sequence, and (caches) in several
@pytest.mark.parametrize("dtype,H,Hk,D,T,n", [("bf16", 2, 2, 64, 9, 0), ("bf16", 2, 2, 96, 70, 0), ("f32", 4, 2, 128, 9, 0),
                                              ("bf16", 256, 256, 64, 9, 300), ("f32", 256, 256, 64, 9, 90), ("bf16", 2, 2, 64, 3, 40), ("bf16", 8, 2, 128, 9, 700), ("bf16", 8, 1, 64, 40, 300),
                                              ("bf16", 4, 1, 192, 30, 130), ("f32", 4, 2, 64, 9, 90), ("f32", 8, 1, 96, 20, 200)])
def test_rows_whose_every_score_is_minus_infinity_are_zero(dtype, H, Hk, D, T, n):
    """The sequence's keys are -inf and its queries positive; values of infinity and NaN times weights of 0.  Another sequence is as ever."""
    b = Batch(dtype, H, Hk, D, [T, T], [n, n], kind="chain", seed=n)
    b.q[:T] = b.q[:T].abs() + 0.5
    want = oracle_64(b)
    b.kt[:T], b.kc[0, :, :n] = -float("inf"), -float("inf")
    b.vt[0], b.vt[1, :, 5] = float("inf"), float("nan")
    if n:
        b.vc[0, :, n // 2], b.vc[0, :, n - 1, 3] = float("nan"), -float("inf")
    out, lse = b.attention()
    assert torch.all(out[:T] == 0) and torch.all(torch.isneginf(lse[:T]))
    for w, empty in zip(want, (0.0, -np.inf, 0.0, 0.0)):
        w[:T] = empty
    b.check(out, lse, want)


def test_buffers_side_by_side_are_apart():
    """Everything a call uses in one allocation, each right behind the other; what is written lies between what is read."""
    b = Batch("bf16", 4, 2, 64, [9, 6], [70, 33], seed=5)
    want = b.attention()
    n_ws = mb.attn_workspace_bytes(b.desc, 2, b.M, b.max_tree, b.max_len)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    tw, cw = torch.empty((b.M, 2), device="cuda"), torch.zeros((2, 2, b.desc.capacity), device="cuda")
    parts = [torch.empty(n_ws, dtype=torch.uint8, device="cuda"), b.q, out, b.kt, lse, b.kc, cw, b.vt, tw, b.vc]
    arena = torch.empty(sum(-(-t.numel() * t.element_size() // 16) * 16 for t in parts), dtype=torch.uint8, device="cuda")
    at, inside = 0, []
    for t in parts:
        n = t.numel() * t.element_size()
        v = arena[at:at + n].view(t.dtype).view(t.shape)
        inside.append(v.copy_(t))
        at += -(-n // 16) * 16
    ws, b.q, out, b.kt, lse, b.kc, cw, b.vt, tw, b.vc = inside
    b.attention(out=out, lse=lse, ws=ws)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    plain = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, ws=ws, cache_w=cw, tree_w=tw, **b.args)
    assert torch.equal(cw, plain[0]) and torch.equal(tw, plain[1])
    # one projection's output holds q, k and v of every row; the results have a buffer of their own
    with pytest.raises(mb.MoeSpecError):
        b.attention(out=b.q, lse=lse, ws=ws)


def test_a_cache_that_is_not_used_may_lie_anywhere():
    b = Batch("bf16", 1, 1, 64, [12], [0], kind="chain", seed=6, room=11)
    assert b.desc.capacity == 12
    want = b.attention()
    out = torch.empty_like(want[0])
    place = out.view(1, 1, 12, 64)
    mb.moespec_tree_attention(b.desc, b.q, b.kt, b.vt, place, place, b.cache_len, out=out, **{**b.args, "max_len": 0})
    assert torch.equal(out, want[0])
