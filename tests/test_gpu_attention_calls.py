"""Calls that a program may make of tree attention, its cache and the block norm: captured steps, large batches and trees, many query
heads per KV head, and tensors that the binding refuses."""
import numpy as np
import pytest
import torch

from paper_2602_16052_amd import binding as mb

from attention_common import Batch, i32
from test_gpu_attention import oracle_64
from test_gpu_attention_walks import check_weights_64, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,Hk,D,trees,lens", [("bf16", 80, 2, 64, [13, 5], [300, 40]), ("f32", 33, 1, 64, [9], [70]),
                                                     ("bf16", 1024, 1, 64, [3], [200]), ("bf16", 64, 1, 128, [40], [0])])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_many_query_heads_of_a_kv_head(dtype, H, Hk, D, trees, lens, kind):
    b = Batch(dtype, H, Hk, D, trees, lens, kind=kind, seed=H)
    out, lse = b.attention()
    b.check(out, lse, oracle_64(b))
    check_weights_64(b, weights(b, lse), lse, torch.ones(b.M, device="cuda"))


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 192), ("f32", 64)])
def test_long_chains(dtype, D):
    b = Batch(dtype, 2, 1, D, [5003], [65], kind="chain", seed=D)
    out, lse = b.attention()
    b.check(out, lse, oracle_64(b))
    check_weights_64(b, weights(b, lse), lse, torch.ones(b.M, device="cuda"))


def test_a_tree_of_many_mask_words():
    b = Batch("bf16", 4, 1, 64, [2101], [90], kind="empty", seed=1)
    out, lse = b.attention()
    b.check(out, lse, oracle_64(b))
    check_weights_64(b, weights(b, lse), lse, torch.ones(b.M, device="cuda"))


def test_thousands_of_sequences():
    rng = np.random.default_rng(2)
    S = 3000
    trees, lens = [int(v) for v in rng.integers(0, 3, S)], [int(v) for v in rng.integers(0, 90, S)]
    b = Batch("bf16", 2, 1, 64, trees, lens, seed=2)
    out, lse = b.attention()
    b.check(out, lse, oracle_64(b))
    check_weights_64(b, weights(b, lse), lse, torch.ones(b.M, device="cuda"))


def test_a_captured_step_follows_what_is_on_the_device():
    """Attention, weights in place, commit and eviction as one graph, replayed over new queries, lengths, paths and accumulated weights,
    against the same calls made one by one; other work runs between the replays."""
    H, Hk, D, trees, lens, budget = 8, 2, 64, [15, 9], [300, 120], 200
    b = Batch("bf16", H, Hk, D, trees, lens, seed=3, room=40)
    S, cap, M = 2, b.desc.capacity, b.M
    b.kc.nan_to_num_(0.0), b.vc.nan_to_num_(0.0)
    path, n_path = i32([[0, 2, 5], [1, 3, 4]]), i32([3, 1])
    rw = torch.rand(M, device="cuda")
    first = dict(kc=b.kc.clone(), vc=b.vc.clone(), cw=torch.rand((S, Hk, cap), device="cuda"))
    at = {k: v.clone() for k, v in first.items()}
    out, lse, tw = torch.zeros_like(b.q), torch.zeros((M, H), device="cuda"), torch.zeros((M, Hk), device="cuda")
    new_len, short = torch.zeros_like(b.cache_len), torch.zeros_like(b.cache_len)
    k, v = (torch.zeros((1, S, Hk, budget, D), dtype=b.q.dtype, device="cuda") for _ in range(2))
    w, kept = torch.zeros((1, S, Hk, budget), device="cuda"), torch.zeros((1, S, Hk, budget), dtype=torch.int32, device="cuda")
    ws, ws2 = mb.alloc_attn_workspace(b.desc, S, M, b.max_tree, cap), mb.alloc_evict_workspace(b.desc, 1, S, budget)
    args = dict(b.args, max_len=cap)
    off = args["tree_off"]
    calls = [mb.TreeAttentionCall(b.desc, b.q, b.kt, b.vt, at["kc"], at["vc"], b.cache_len, ws, out, lse, **args),
             mb.CacheWeightsCall(b.desc, b.q, b.kt, at["kc"], b.cache_len, lse, ws, at["cw"], tw, at["cw"], 0.5, rw, **args),
             mb.CacheCommitCall(b.desc, b.kt[None], b.vt[None], path, n_path, at["kc"][None], at["vc"][None], b.cache_len, new_len, tw[None],
                                at["cw"][None], off, b.max_tree),
             mb.CacheEvictCall(b.desc, at["kc"][None], at["vc"][None], at["cw"][None], new_len, budget, 8, k, v, w, ws2, kept, short)]
    results = [out, lse, tw, new_len, short, k, v, w, kept, *at.values()]

    def start():
        for name, t in at.items():
            t.copy_(first[name])
        for t in (out, lse, tw, k, v, w, kept):
            t.zero_()

    for c in calls:
        c()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for c in calls:
            c()
    for step, (now, n) in enumerate([([300, 120], [3, 1]), ([cap - 1, 0], [3, 3]), ([1, 199], [0, 2]), ([210, 205], [2, 0])]):
        b.cache_len.copy_(i32(now)), n_path.copy_(i32(n))
        b.q.mul_(0.75).add_(0.125)
        start()
        for c in calls:
            c()
        want = [t.clone() for t in results]
        start()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(results, want)):
            assert torch.equal(x, y), f"step {step}, result {i}"
        assert short.tolist() == [min(budget, cap, m + p) for m, p in zip(now, n)]


# ---- what the binding refuses

def test_tensors_of_another_type_shape_or_layout_are_refused():
    b = Batch("bf16", 4, 2, 64, [5, 3], [40, 20], seed=4)
    lse = b.attention()[1]
    S, M, cap = 2, b.M, b.desc.capacity

    def refused(what, match, **kw):
        with pytest.raises(ValueError, match=match):
            what(**kw)

    at = b.attention
    refused(at, "out must have dtype", out=torch.empty((M, 4, 64), device="cuda"))
    refused(at, "out must have shape", out=torch.empty((M, 4, 32), dtype=b.q.dtype, device="cuda"))
    refused(at, "out must be contiguous", out=torch.empty((4, M, 64), dtype=b.q.dtype, device="cuda").transpose(0, 1))
    refused(at, "lse must have shape", lse=torch.empty((M, 2), device="cuda"))
    refused(at, "tree_off must have dtype", tree_off=torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused(at, "tree_mask must have shape", tree_mask=torch.zeros((M, 2), dtype=torch.int32, device="cuda"))
    refused(at, "tree_mask must be a GPU tensor", tree_mask=b.mask.cpu())
    refused(at, "ws must be a contiguous uint8 tensor", ws=torch.empty(1 << 20, device="cuda"))
    with pytest.raises(mb.MoeSpecError):
        at(ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(mb.MoeSpecError):
        at(max_len=cap + 1)
    with pytest.raises(mb.MoeSpecError):
        at(max_tree=M + 1, tree_mask=None)

    def q(t):
        return lambda **kw: mb.moespec_tree_attention(b.desc, t, b.kt, b.vt, b.kc, b.vc, b.cache_len, **b.args)
    refused(q(b.q[:, :2]), "q must have shape")
    refused(q(b.q.expand(M, 4, 64).transpose(0, 1).contiguous().transpose(0, 1)), "a token's heads must lie in a row")
    refused(q(b.q[:1].expand(M, 4, 64)), "a token's heads must lie in a row")
    wide = torch.zeros((M, 3, 64), dtype=b.q.dtype, device="cuda")
    with pytest.raises(ValueError, match="same row stride"):
        mb.moespec_tree_attention(b.desc, b.q, b.kt, wide[:, :2], b.kc, b.vc, b.cache_len, **b.args)
    with pytest.raises(ValueError, match="cache_len must have shape"):
        mb.moespec_tree_attention(b.desc, b.q, b.kt, b.vt, b.kc, b.vc, b.cache_len[:1], **b.args)
    with pytest.raises(mb.MoeSpecError):  # a cache without lengths
        mb.moespec_tree_attention(b.desc, b.q, b.kt, b.vt, b.kc, b.vc, None, **b.args)

    def wt(**kw):
        return mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **{**b.args, **kw})
    refused(wt, "row_weight must have shape", row_weight=torch.ones(M + 1, device="cuda"))
    refused(wt, "cache_w_in must have dtype", cache_w_in=torch.zeros((S, 2, cap), dtype=torch.float64, device="cuda"))
    with pytest.raises(mb.MoeSpecError):
        wt(decay=float("inf"))
    k = b.kc[None]
    with pytest.raises(ValueError, match="path must have shape"):
        mb.moespec_cache_commit(b.desc, b.kt[None], b.vt[None], i32([[0, 1]]), i32([1, 1]), k, b.vc[None], b.cache_len,
                                tree_off=b.args["tree_off"], max_tree=5)
    with pytest.raises(mb.MoeSpecError):  # weights of the tree without those of the cache
        mb.moespec_cache_commit(b.desc, b.kt[None], b.vt[None], i32([[0], [1]]), i32([1, 1]), k, b.vc[None], b.cache_len,
                                tree_w=torch.zeros((1, M, 2), device="cuda"), tree_off=b.args["tree_off"], max_tree=5)
    w = torch.zeros((1, S, 2, cap), device="cuda")
    for budget, recent in ((0, 0), (10, 11), (10, -1)):
        with pytest.raises(mb.MoeSpecError):
            mb.moespec_cache_evict(b.desc, k, b.vc[None], w, b.cache_len, budget, recent)
    with pytest.raises(ValueError, match="cache_w must have shape"):
        mb.moespec_cache_evict(b.desc, k, b.vc[None], w[..., 1:], b.cache_len, 10, 1)
    layer = mb.LayerDesc(64, 1, 1, 64, mb.F32, False)
    y = torch.zeros((5, 64), device="cuda")
    for kw, match in ((dict(gate=y, gate_kind=mb.BLOCK_GATE_TOKEN), "gate must have shape"), (dict(w_pre=y), "w_pre must have shape"),
                      (dict(residual=y.half()), "residual must have dtype"), (dict(r=y.t().contiguous().t()), "r must be contiguous")):
        with pytest.raises(ValueError, match=match):
            mb.moespec_block_norm(layer, y, **kw)
    with pytest.raises(mb.MoeSpecError):
        mb.moespec_block_norm(layer, y, w_post=y[0])  # a weight of a norm that is not wanted
