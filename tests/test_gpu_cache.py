"""The cache of a verification step: attention weight of its keys, commit of the accepted path, eviction to a budget."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2602_16052_amd import binding as mb

from attention_common import CODE, TORCH, Batch, f64, i32

pytestmark = pytest.mark.gpu


# ---- attention weight

def check_weights(b, cache_w, tree_w, lse, row_weight=None, w_in=None, decay=1.0, before=0.0):
    l64 = f64(lse)
    scale = float(np.float32(b.scale))
    cw, tw, acw, atw = A.weights(f64(b.q), f64(b.kt), f64(b.kc), b.lens, b.off, b.sees, scale, l64,
                                 None if row_weight is None else f64(row_weight), None if w_in is None else f64(w_in), decay)
    spread = b.oracle()[3].max()
    # every weight: error of its score, of lse in units of log 2 and of the exponential; fp32 sums over the rows
    top = np.abs(np.where(np.isfinite(l64), l64, 0)).max()
    rel = b.score_error(spread) + (top + 4) * 2.0 ** -22 + (max(b.trees) * b.H // b.Hk + 64) * 2.0 ** -23
    for s, n in enumerate(b.lens):
        got = f64(cache_w[s])
        assert np.all(np.abs(got[:, :n] - cw[s, :, :n]) <= acw[s, :, :n] * rel + 1e-37), \
            np.max(np.abs(got[:, :n] - cw[s, :, :n]) / (acw[s, :, :n] * rel + 1e-37))
        assert np.all(got[:, n:] == before), "entries behind a length were written"
    used = slice(0, int(b.off[-1]))
    assert np.all(np.abs(f64(tree_w) - tw)[used] <= atw[used] * rel + 1e-37)


WEIGHT_FORMS = [(dt, D, H, Hk, T) for dt in ("bf16", "f32") for D in (64, 96, 128, 192, 256) for H, Hk, T in ((4, 4, 5), (6, 2, 40))]


@pytest.mark.parametrize("dtype,D,H,Hk,T", WEIGHT_FORMS)
def test_weights_of_head_sizes(dtype, D, H, Hk, T):
    b = Batch(dtype, H, Hk, D, [T, T - 2], [301, 97], seed=D + T)
    lse = b.attention()[1]
    check_weights(b, *mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args), lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tree", "chain", "empty"])
@pytest.mark.parametrize("n,T", [(0, 1), (1, 1), (127, 2), (128, 33), (129, 64), (257, 65), (513, 130), (3, 300)])
def test_weights_around_the_tiles(dtype, kind, n, T):
    b = Batch(dtype, 6, 2, 64, [T], [n], kind=kind, seed=n + T)
    lse = b.attention()[1]
    check_weights(b, *mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args), lse)


@pytest.mark.parametrize("in_place", [False, True])
def test_weights_accumulate_with_decay_and_row_weights(in_place):
    b = Batch("bf16", 14, 2, 128, [9, 0, 33, 1], [70, 5, 0, 260], fused=True, pad=4, seed=2)
    lse = b.attention()[1]
    rw = torch.rand(b.M, device="cuda") - 0.25
    rw[3] = 0.0
    w_in = torch.rand((4, 2, b.desc.capacity), device="cuda")
    for s, n in enumerate(b.lens):
        w_in[s, :, n:] = 9.0
    before = w_in.clone()
    out = w_in if in_place else torch.full_like(w_in, 9.0)
    tree_w = torch.full((b.M, 2), 9.0, device="cuda")
    mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, cache_w=out, tree_w=tree_w, cache_w_in=w_in, decay=0.75,
                             row_weight=rw, **b.args)
    check_weights(b, out, tree_w, lse, rw, before, 0.75, before=9.0)
    assert torch.all(tree_w[b.M - 4:] == 9.0)


def test_rows_without_an_lse_have_no_part():
    b = Batch("f32", 4, 2, 64, [12], [90], seed=3)
    lse = b.attention()[1]
    lse[5] = float("-inf")
    lse[7, 2] = float("-inf")
    b.q[5] = float("nan")
    got = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    b.q[5] = 0
    check_weights(b, *got, lse)


def test_weights_of_keys_that_a_row_does_not_see():
    b = Batch("bf16", 4, 2, 64, [40], [0], seed=4)
    b.kt[20] = float("nan")
    lse = b.attention()[1]
    assert torch.isfinite(lse[~torch.from_numpy(b.sees[0][:, 20]).cuda()]).all()
    lse[torch.from_numpy(b.sees[0][:, 20]).cuda()] = float("-inf")
    tree_w = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)[1]
    b.kt[20] = 0
    check_weights(b, torch.zeros((1, 2, b.desc.capacity), device="cuda"), tree_w, lse)


def test_weights_repeat_and_sum_to_the_rows():
    b = Batch("bf16", 16, 4, 128, [63], [3000], seed=5)
    lse = b.attention()[1]
    one = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    two = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    total = float(one[0].double().sum() + one[1].double().sum())
    assert abs(total - 63 * 16) < 63 * 16 * 1e-5  # every row's weights add up to 1


def test_weights_without_tree_or_cache_outputs():
    b = Batch("bf16", 4, 2, 64, [12], [90], seed=6)
    lse = b.attention()[1]
    want = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    ws = mb.alloc_attn_workspace(b.desc, 1, b.M, b.max_tree, b.max_len)
    out = torch.zeros_like(want[0])
    mb.CacheWeightsCall(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, ws, out, None, **b.args)()
    assert torch.allclose(out, want[0], rtol=1e-5)
    only = dict(b.args, max_len=0)
    tree_w = torch.zeros_like(want[1])
    mb.CacheWeightsCall(b.desc, b.q, b.kt, None, None, lse, ws, None, tree_w, **only)()
    assert torch.allclose(tree_w, want[1], rtol=1e-5)


# ---- commit

class Caches:
    def __init__(self, dtype, L, S, Hk, D, cap, lens, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.k = torch.randn((L, S, Hk, cap, D), generator=gen, device="cuda").to(TORCH[dtype])
        self.v = torch.randn((L, S, Hk, cap, D), generator=gen, device="cuda").to(TORCH[dtype])
        self.w = torch.rand((L, S, Hk, cap), generator=gen, device="cuda")
        self.len, self.lens, self.L = i32(lens), lens, L
        self.desc = mb.AttnDesc(Hk, Hk, D, cap, CODE[dtype])


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 96), ("bf16", 256), ("f32", 64), ("f32", 192)])
@pytest.mark.parametrize("fused", [False, True])
def test_commit_appends_the_path(dtype, D, fused):
    L, S, Hk, cap, trees = 3, 4, 2, 40, [7, 0, 5, 9]
    lens, n_path = [10, 3, 38, 40], [4, 2, 6, 1]  # the third runs into the capacity, the fourth is full
    c = Caches(dtype, L, S, Hk, D, cap, lens, seed=D)
    off = np.concatenate([[0], np.cumsum(trees)])
    M = int(off[-1]) + 2
    kv = torch.randn((L, M, 2 * Hk, D), device="cuda").to(TORCH[dtype])
    kt, vt = kv[:, :, :Hk], kv[:, :, Hk:]
    if not fused:
        kt, vt = kt.contiguous(), vt.contiguous()
    tw = torch.rand((L, M, Hk), device="cuda")
    path = np.array([[0, 2, 2, 6, 1, 1], [0, 1, 0, 0, 0, 0], [4, 9, -1, 3, 5, 2], [8, 0, 0, 0, 0, 0]])
    want = [t.clone() for t in (c.k, c.v, c.w)]
    for s in range(S):
        for i in range(min(n_path[s], cap - lens[s])):
            t, at = path[s, i], lens[s] + i
            ok = 0 <= t < trees[s]
            for out, src in zip(want, (kt, vt, tw)):
                out[:, s, :, at] = src[:, off[s] + t] if ok else 0
    new_len = mb.moespec_cache_commit(c.desc, kt, vt, i32(path), i32(n_path), c.k, c.v, c.len, tree_w=tw, cache_w=c.w,
                                      tree_off=i32(off), max_tree=9, n_layers=L)
    for got, ref in zip((c.k, c.v, c.w), want):
        assert torch.equal(got, ref)
    assert new_len.tolist() == [14, 5, 40, 40]
    assert c.len.tolist() == lens


def test_commit_without_weights_and_with_lengths_out_of_range():
    c = Caches("bf16", 1, 2, 1, 64, 8, [-4, 99], seed=1)
    kt, vt = torch.randn((1, 6, 1, 64), device="cuda").bfloat16(), torch.randn((1, 6, 1, 64), device="cuda").bfloat16()
    k0 = c.k.clone()
    new_len = mb.moespec_cache_commit(c.desc, kt, vt, i32([[2, 1], [0, 0]]), i32([77, -1]), c.k, c.v, c.len,
                                      tree_off=i32([0, 3, 6]), max_tree=3)
    assert new_len.tolist() == [2, 8]
    assert torch.equal(c.k[0, 0, 0, 0], kt[0, 2, 0]) and torch.equal(c.v[0, 0, 0, 1], vt[0, 1, 0])
    assert torch.equal(c.k[0, 0, 0, 2:], k0[0, 0, 0, 2:]) and torch.equal(c.k[0, 1], k0[0, 1])


def test_commit_of_single_tokens_out_of_one_projection():
    """One token for a whole model: layers are the only distance there is between rows."""
    c = Caches("bf16", 3, 1, 2, 64, 9, [4], seed=2)
    qkv = torch.randn((3, 1, 8, 64), device="cuda").bfloat16()
    new_len = mb.moespec_cache_commit(c.desc, qkv[:, :, 4:6], qkv[:, :, 6:], i32([[0]]), i32([1]), c.k, c.v, c.len, n_layers=3)
    assert new_len.tolist() == [5]
    assert torch.equal(c.k[:, 0, :, 4], qkv[:, 0, 4:6]) and torch.equal(c.v[:, 0, :, 4], qkv[:, 0, 6:])


def test_commit_behind_32_bits():
    cap = 9_000_000
    desc = mb.AttnDesc(2, 2, 128, cap, mb.BF16)
    k, v = (torch.zeros((1, 2, 2, cap, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kt, vt = torch.randn((1, 6, 2, 128), device="cuda").bfloat16(), torch.randn((1, 6, 2, 128), device="cuda").bfloat16()
    new_len = mb.moespec_cache_commit(desc, kt, vt, i32([[1, 2], [2, 0]]), i32([1, 2]), k, v, i32([5, cap - 2]),
                                      tree_off=i32([0, 3, 6]), max_tree=3)
    assert new_len.tolist() == [6, cap]
    assert torch.equal(k[0, 1, :, cap - 2], kt[0, 5]) and torch.equal(v[0, 1, :, cap - 1], vt[0, 3])
    assert torch.equal(k[0, 0, :, 5], kt[0, 1]) and int((k != 0).any(dim=-1).sum()) == 6


# ---- eviction

def check_evict(c, budget, recent, room=3):
    L, S, Hk, cap, D = c.k.shape
    k, v = (torch.full((L, S, Hk, budget + room, D), 7.0, dtype=c.k.dtype, device="cuda") for _ in range(2))
    w = torch.full((L, S, Hk, budget + room), 7.0, device="cuda")
    kept, new_len = torch.full((L, S, Hk, budget), 77, dtype=torch.int32, device="cuda"), torch.full_like(c.len, 77)
    ws = mb.alloc_evict_workspace(c.desc, L, S, budget)
    mb.CacheEvictCall(c.desc, c.k, c.v, c.w, c.len, budget, recent, k, v, w, ws, kept, new_len, n_layers=L)()
    wn = c.w.cpu().numpy()
    for s in range(S):
        n = min(max(c.lens[s], 0), cap)
        m = min(n, budget)
        assert int(new_len[s]) == m
        for l in range(L):
            for h in range(Hk):
                want = A.kept_entries(wn[l, s, h], n, budget, recent)
                got = kept[l, s, h].cpu().numpy()
                assert np.array_equal(got[:m], want), (l, s, h)
                assert np.all(got[m:] == -1)
                at = torch.from_numpy(want).cuda()
                assert torch.equal(k[l, s, h, :m], c.k[l, s, h, at]) and torch.equal(v[l, s, h, :m], c.v[l, s, h, at])
                assert torch.equal(w[l, s, h, :m].view(torch.int32), c.w[l, s, h, at].view(torch.int32))
                assert torch.all(k[l, s, h, m:] == 7.0) and torch.all(v[l, s, h, m:] == 7.0) and torch.all(w[l, s, h, m:] == 7.0)
    # without the optional outputs: the same
    k2, v2, w2 = torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.full_like(w, 7.0)
    mb.CacheEvictCall(c.desc, c.k, c.v, c.w, c.len, budget, recent, k2, v2, w2, ws, n_layers=L)()
    assert torch.equal(k, k2) and torch.equal(v, v2) and torch.equal(w.view(torch.int32), w2.view(torch.int32))


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 96), ("bf16", 128), ("f32", 64), ("f32", 256)])
@pytest.mark.parametrize("lens,budget,recent", [([200, 64, 63, 65, 0, 1], 64, 16), ([300, 2, 130, 128, 129, 90], 1, 0),
                                                ([300, 2, 130, 128, 129, 90], 1, 1), ([1000, 999, 37, 400, 5, 6], 399, 399)])
def test_eviction_keeps_the_heaviest_and_the_latest(dtype, D, lens, budget, recent):
    check_evict(Caches(dtype, 2, 6, 2, D, 1003, lens, seed=budget), budget, recent)


@pytest.mark.parametrize("what", ["equal", "few", "nan", "all_nan", "signs", "infinite", "close"])
def test_eviction_of_awkward_weights(what):
    c = Caches("bf16", 1, 2, 2, 64, 3000, [2900, 1500], seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    u = torch.rand(c.w.shape, generator=g, device="cuda")
    if what == "equal":
        c.w.fill_(0.25)
    elif what == "few":
        c.w.copy_((u * 3).floor())
    elif what == "nan":
        c.w[u < 0.5] = float("nan")
    elif what == "all_nan":
        c.w.fill_(float("nan"))
    elif what == "signs":
        c.w.copy_(torch.where(u < 0.3, -u, torch.where(u < 0.5, -0.0 * u, torch.where(u < 0.7, 0.0 * u, u))))
    elif what == "infinite":
        c.w[u < 0.3], c.w[u > 0.6] = float("inf"), float("-inf")
    else:  # neighbours of one number
        c.w.copy_((torch.full_like(u, 1.5).view(torch.int32) + (u * 40).int()).view(torch.float32))
    for budget, recent in ((700, 10), (1400, 700), (2899, 0), (1, 0)):
        check_evict(c, budget, recent)


def test_eviction_of_long_caches():
    check_evict(Caches("bf16", 1, 1, 2, 64, 70_001, [70_001], seed=3), 5000, 128)


def test_eviction_with_lengths_out_of_range():
    check_evict(Caches("f32", 1, 2, 1, 64, 100, [-7, 10 ** 8], seed=4), 30, 10)


def test_eviction_behind_32_bits():
    cap = 9_000_000
    c = Caches("bf16", 1, 1, 1, 64, 8, [8])
    c.k, c.v = (torch.zeros((1, 2, 2, cap, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.w = torch.zeros((1, 2, 2, cap), device="cuda")
    at = torch.tensor([7, 100, cap - 90, cap - 5], device="cuda")
    c.w[0, 1, 1, at] = 2.0
    c.k[0, 1, 1, at], c.v[0, 1, 1, at] = 3.0, 4.0
    c.k[0, 1, 1, -2:] = 5.0
    r = mb.moespec_cache_evict(mb.AttnDesc(2, 2, 128, cap, mb.BF16), c.k, c.v, c.w, i32([0, cap]), 6, 2)
    assert r["kept"][0, 1, 1].tolist() == [7, 100, cap - 90, cap - 5, cap - 2, cap - 1]
    assert torch.all(r["k"][0, 1, 1, :4] == 3) and torch.all(r["k"][0, 1, 1, 4:] == 5) and torch.all(r["v"][0, 1, 1, :4] == 4)
    assert r["new_len"].tolist() == [0, 6] and torch.all(r["kept"][0, 0] == -1)


def test_captured_commit_and_evict_follow_the_lengths():
    c = Caches("bf16", 2, 2, 2, 128, 500, [300, 200], seed=6)
    kt, vt = torch.randn((2, 10, 2, 128), device="cuda").bfloat16(), torch.randn((2, 10, 2, 128), device="cuda").bfloat16()
    tw, path, n_path, off = torch.rand((2, 10, 2), device="cuda"), i32([[0, 2], [1, 3]]), i32([2, 1]), i32([0, 5, 10])
    new_len, evicted = torch.zeros_like(c.len), torch.zeros_like(c.len)
    B = 250
    ws = mb.alloc_evict_workspace(c.desc, 2, 2, B)
    k, v = (torch.zeros((2, 2, 2, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w, kept = torch.zeros((2, 2, 2, B), device="cuda"), torch.zeros((2, 2, 2, B), dtype=torch.int32, device="cuda")
    commit = mb.CacheCommitCall(c.desc, kt, vt, path, n_path, c.k, c.v, c.len, new_len, tw, c.w, off, 5, n_layers=2)
    evict = mb.CacheEvictCall(c.desc, c.k, c.v, c.w, new_len, B, 20, k, v, w, ws, kept, evicted, n_layers=2)
    commit(), evict()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        commit(), evict()
    for lens in ([300, 200], [10, 499], [249, 251]):
        c.len.copy_(i32(lens))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (k, v, w, kept, new_len, evicted)]
        commit(), evict()
        torch.cuda.synchronize()
        for a, b in zip(got, (k, v, w, kept, new_len, evicted)):
            assert torch.equal(a, b)
        assert new_len.tolist() == [min(500, lens[0] + 2), min(500, lens[1] + 1)]


def test_functions_allocate_on_the_stream_they_are_given():
    """Results that a function allocates are cleared before its call on another stream, not by work of the present one that
    comes later, and its workspace is not handed out again while the call may still run."""
    c = Caches("bf16", 1, 2, 2, 64, 600, [500, 90], seed=7)
    b = Batch("bf16", 4, 2, 64, [5, 9], [200, 30], seed=8)
    lse = b.attention()[1]
    want = mb.moespec_cache_evict(c.desc, c.k, c.v, c.w, c.len, 100, 10)
    want_w = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, **b.args)
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(40):
        busy = busy @ busy  # the present stream is occupied
    got = mb.moespec_cache_evict(c.desc, c.k, c.v, c.w, c.len, 100, 10, stream=side)
    got_w = mb.moespec_cache_weights(b.desc, b.q, b.kt, b.kc, b.cache_len, lse, stream=side, **b.args)
    torch.cuda.synchronize()
    for name in want:
        assert torch.equal(want[name], got[name]), name
    assert torch.equal(want_w[0], got_w[0]) and torch.equal(want_w[1], got_w[1])
