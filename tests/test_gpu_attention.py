"""Tree attention over a cache (moespec_tree_attention) against the fp64 oracle: types, head layouts, odd and ragged sizes, masks,
values that must not be seen, and the ways a program calls it."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2602_16052_amd import binding as mb

from attention_common import Batch, f64, i32

pytestmark = pytest.mark.gpu

# every head size, type and row-tile form (up to 32, up to 64, more rows per KV head)
FORMS = [(dt, D, H, Hk, T) for dt in ("bf16", "f32") for D in (64, 96, 128, 192, 256)
         for H, Hk, T in ((4, 4, 5), (6, 2, 17), (8, 1, 19))]


@pytest.mark.parametrize("dtype,D,H,Hk,T", FORMS)
def test_head_sizes_and_row_tiles(dtype, D, H, Hk, T):
    b = Batch(dtype, H, Hk, D, [T, max(1, T - 3)], [301, 97], seed=D + T)
    b.check(*b.attention())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 513])
def test_cache_lengths_around_the_tiles(dtype, n):
    b = Batch(dtype, 4, 2, 64, [3, 1], [n, max(0, n - 1)], seed=n)
    b.check(*b.attention())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tree", "chain", "empty"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 130])
def test_tree_sizes_and_masks(dtype, kind, T):
    b = Batch(dtype, 6, 2, 64, [T], [0 if kind == "empty" else 40], kind=kind, seed=T)
    b.check(*b.attention())


@pytest.mark.parametrize("dtype,H,Hk,D", [("bf16", 14, 2, 128), ("bf16", 7, 1, 96), ("f32", 12, 4, 64), ("bf16", 16, 16, 128)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_ragged_batches_with_empty_sequences_and_padding(dtype, H, Hk, D, kind):
    b = Batch(dtype, H, Hk, D, [9, 0, 33, 1, 4], [70, 5, 0, 1, 260], kind=kind, fused=True, pad=6, seed=H)
    out = torch.full((b.M, H, D), 7.0, dtype=b.q.dtype, device="cuda")
    lse = torch.full((b.M, H), 7.0, device="cuda")
    b.attention(out=out, lse=lse)
    b.check(out, lse)
    assert torch.all(out[b.M - 6:] == 7.0) and torch.all(lse[b.M - 6:] == 7.0), "rows behind the last sequence were written"


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("n", [0, 40, 64, 128, 170, 192, 256, 321, 1500])
def test_many_rows_over_few_and_many_tiles(D, n):
    """More than 128 rows per KV head; the last workgroup's waves have rows, some, or none."""
    b = Batch("bf16", 8, 2, D, [33, 70, 49], [n, max(0, n - 64), n // 2], seed=n + D)
    b.check(*b.attention())


@pytest.mark.parametrize("q_scale", [0.1, 12.0])
def test_many_rows_with_a_rising_maximum(q_scale):
    """Scores that grow along the cache: every tile raises the maximum."""
    b = Batch("bf16", 8, 2, 128, [40], [700], seed=1, q_scale=q_scale)
    ramp = torch.linspace(0.05, 1.0, b.kc.shape[2], device="cuda")
    b.kc.copy_((b.q[0, ::4, None, :].float() * 0.3 + b.kc.float() * 0.2) * ramp[None, None, :, None])
    b.kc[0, :, 700:] = float("nan")
    b.check(*b.attention())


@pytest.mark.parametrize("S,T,H,Hk", [(2, 1, 4, 1), (5, 3, 2, 1), (40, 2, 2, 1), (70, 1, 1, 1), (300, 1, 1, 1), (3, 50, 8, 2)])
def test_sequences_that_share_the_parts(S, T, H, Hk):
    """Lengths from nothing to long ones and empty trees: every sequence takes parts by its length."""
    rng = np.random.default_rng(S)
    lens = [int(v) for v in (rng.random(S) ** 6 * 3000)]
    trees = [0 if rng.random() < 0.1 else int(rng.integers(1, T + 1)) for _ in range(S)]
    trees[-1] = T
    b = Batch("bf16", H, Hk, 64, trees, lens, seed=S, pad=2)
    b.check(*b.attention())


def test_large_tree_and_long_cache():
    b = Batch("bf16", 8, 2, 128, [255], [2051], seed=3)
    b.check(*b.attention())


def test_long_prompt_chunk_is_causal():
    b = Batch("bf16", 2, 1, 64, [700], [100], kind="chain", seed=4)
    b.check(*b.attention())


def test_one_sequence_without_offsets_and_without_cache():
    b = Batch("f32", 4, 2, 64, [21], [0], kind="chain", seed=5)
    out, lse = mb.moespec_tree_attention(b.desc, b.q, b.kt, b.vt)
    b.check(out, lse)


def test_other_scales_and_large_scores():
    b = Batch("f32", 2, 2, 64, [9], [77], seed=6, q_scale=30.0, scale=1.7)
    b.check(*b.attention())
    b = Batch("bf16", 2, 2, 64, [9], [77], seed=6, q_scale=1e-3, scale=1.0)
    b.check(*b.attention())


@pytest.mark.parametrize("dtype,H,Hk,T", [("bf16", 2, 1, 40), ("bf16", 8, 1, 40), ("f32", 2, 1, 12), ("f32", 8, 1, 20)])
def test_values_that_are_not_seen_have_no_part(dtype, H, Hk, T):
    """NaN and infinities in keys and values of the tree: rows that do not see them are exact, rows that do are not finite."""
    b = Batch(dtype, H, Hk, 64, [T], [50], seed=7)
    b.kt[3], b.vt[3] = float("nan"), float("inf")
    b.vt[T - 2, :, 5] = float("-inf")
    b.vt[T - 1, :, 9] = float("nan")
    out, lse = b.attention()
    want, want_lse, bound, spread = b.oracle()
    sees = b.sees[0]
    clean = ~(sees[:, 3] | sees[:, T - 2] | sees[:, T - 1])
    assert 0 < clean.sum() < T
    assert np.all(np.isfinite(f64(out)[clean]))
    tidy = lambda v: np.where(clean.reshape(-1, *[1] * (v.ndim - 1)), v, 0.0)  # noqa: E731
    keep = torch.from_numpy(clean).cuda()
    got, got_lse = out.clone(), lse.clone()
    got[~keep], got_lse[~keep] = 0, 0
    b.check(got, got_lse, (tidy(want), tidy(want_lse), tidy(bound), tidy(spread)))
    assert np.all(np.isnan(f64(out)[sees[:, 3]]))
    only = sees[:, T - 2] & ~sees[:, 3] & ~sees[:, T - 1]
    got = f64(out)[only]
    assert np.all(np.isneginf(got[..., 5])) and np.all(np.isfinite(np.delete(got, 5, axis=-1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_seen_comes_through(dtype):
    b = Batch(dtype, 2, 1, 64, [4, 4], [90, 90], seed=8)
    b.vc[0, 0, 17, 3] = float("nan")
    b.kc[1, 0, 30] = float("-inf")  # scores +-inf: rows of this sequence have no softmax, the other sequence has one
    out = f64(b.attention()[0])
    assert np.all(np.isnan(out[:4, :, 3])) and np.all(np.isfinite(np.delete(out[:4], 3, axis=-1)))
    # an infinity in the last entry of a cache stays one, beside the places behind it that fill the tile
    for H in (2, 6, 40):
        b = Batch(dtype, H, 1, 64, [4], [90], seed=8)
        b.vc[0, 0, 89, 3], b.vc[0, 0, 89, 7], b.vc[0, 0, 50, 9] = float("inf"), float("-inf"), float("inf")
        out = f64(b.attention()[0])
        assert np.all(out[:, :, [3, 9]] == np.inf) and np.all(out[:, :, 7] == -np.inf)
        assert np.all(np.isfinite(np.delete(out, [3, 7, 9], axis=-1)))
    b = Batch(dtype, 2, 1, 64, [3], [0], seed=9, kind="empty")
    b.mask.zero_()
    out, lse = b.attention()
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))


def test_lengths_and_offsets_out_of_range_are_clamped():
    b = Batch("bf16", 4, 2, 64, [6, 5], [80, 33], kind="chain", seed=10, room=0)
    b.kc[1, :, 33:], b.vc[1, :, 33:] = 0.5, -0.25
    b.cache_len = i32([-3, 10 ** 9])
    b.lens = [0, 80]
    b.check(*b.attention())
    # offsets: a last one behind the rows, a first one in front of them
    b.args["tree_off"] = i32([-4, 6, 10 ** 6])
    b.check(*b.attention())
    # a tree cut at max_tree
    b.args["max_tree"] = 4
    b.args["tree_off"] = i32(b.off)
    out = torch.full_like(b.q, 3.0)
    lse = torch.full((b.M, 4), 3.0, device="cuda")
    b.attention(out=out, lse=lse)
    assert torch.all(out[4:6] == 3.0) and torch.all(lse[10:] == 3.0)
    want, want_lse, bound, spread = b.oracle()
    out[4:6], lse[4:6], out[10:], lse[10:] = 0, 0, 0, 0
    for v in (want, want_lse, bound, spread):
        v[4:6] = v[10:] = 0
    b.check(out, lse, (want, want_lse, bound, spread))


def test_max_len_below_the_capacity_cuts_the_cache():
    b = Batch("f32", 2, 2, 64, [3], [150], seed=11)
    b.args["max_len"], b.lens = 60, [60]
    b.check(*b.attention())


def test_offsets_beyond_32_bits():
    """Two sequences of two KV heads with room for 9 million entries: the last head starts behind element 3.4e9."""
    cap, D, lens = 9_000_000, 128, [70, 300]
    b = Batch("bf16", 4, 2, D, [3, 7], lens, seed=12)
    b.desc.capacity = cap
    kc, vc = (torch.empty((2, 2, cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for s, n in enumerate(lens):
        kc[s, :, :n], vc[s, :, :n] = b.kc[s, :, :n], b.vc[s, :, :n]
    oracle = b.oracle()
    b.kc, b.vc = kc, vc
    b.check(*b.attention(), oracle)


def test_calls_repeat_bit_for_bit_and_on_other_streams():
    b = Batch("bf16", 8, 2, 128, [31, 17], [900, 411], seed=13)
    out, lse = b.attention()
    ws = mb.alloc_attn_workspace(b.desc, 2, b.M, b.max_tree, b.max_len)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    call = mb.TreeAttentionCall(b.desc, b.q, b.kt, b.vt, b.kc, b.vc, b.cache_len, ws, o2, l2, **b.args)
    with torch.cuda.stream(side):  # the stream that is current at the call
        call()
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    mb.TreeAttentionCall(b.desc, b.q, b.kt, b.vt, b.kc, b.vc, b.cache_len, ws, o2.zero_(), l2, **b.args, stream=side)()
    torch.cuda.synchronize()
    assert torch.equal(out, o2)


def test_two_streams_with_workspaces_of_their_own():
    bs = [Batch("bf16", 8, 2, 128, [31], [1500], seed=14), Batch("f32", 4, 4, 64, [20, 3], [700, 30], seed=15)]
    want = [b.attention() for b in bs]
    calls, outs = [], []
    for b in bs:
        st = torch.cuda.Stream()
        for _ in range(12):
            ws = mb.alloc_attn_workspace(b.desc, len(b.trees), b.M, b.max_tree, b.max_len)
            o = torch.empty_like(want[len(outs) >= 12][0])
            outs.append(o)
            calls.append(mb.TreeAttentionCall(b.desc, b.q, b.kt, b.vt, b.kc, b.vc, b.cache_len, ws, o, **b.args, stream=st))
    torch.cuda.synchronize()
    for i in range(12):
        calls[i]()
        calls[12 + i]()
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, want[i >= 12][0]), f"call {i}"


def test_captured_calls_follow_lengths_and_inputs():
    """Two graphs that share a workspace, replayed in turn with eager calls between them; lengths grow on the device."""
    b = Batch("bf16", 8, 2, 128, [15, 7], [700, 300], seed=16)
    ws = mb.alloc_attn_workspace(b.desc, 2, b.M, b.max_tree, b.max_len)
    b.attention(ws=ws)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        out, lse = torch.empty((b.M, 8, 128), dtype=b.q.dtype, device="cuda"), torch.empty((b.M, 8), device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.attention(out=out, lse=lse, ws=ws)
        graphs.append(g)
        outs.append((out, lse))
    for step, lens in enumerate([[700, 300], [1, 0], [650, 299]]):
        b.cache_len.copy_(i32(lens))
        b.q.mul_(0.5 if step else 1.0)
        want = [v.clone() for v in b.attention(ws=ws)]
        for g, got in zip(graphs, outs):
            got[0].fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), f"step {step}"
    b.lens = lens
    b.check(*outs[0])


def test_parents_to_masks():
    sees = A.ancestors([-1, 0, 0, 1, -1, 4])
    assert [list(np.flatnonzero(r)) for r in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]


# ---- many rows over long caches: the straight-line form, which takes launches that fill the card

def oracle_64(b):
    """Batch.oracle() as products of 64-bit matrices on the GPU, for batches that would take its loops minutes."""
    G, D = b.H // b.Hk, b.D
    out, bound = (torch.zeros((b.M, b.H, D), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((b.M, b.H), -float("inf"), dtype=torch.float64, device="cuda")
    spread = torch.zeros((b.M, b.H), dtype=torch.float64, device="cuda")
    scale = float(np.float32(b.scale))
    for s, (n, T) in enumerate(zip(b.lens, b.trees)):
        if T == 0:
            continue
        rows = slice(int(b.off[s]), int(b.off[s + 1]))
        k, v = (torch.cat([c[s, :, :n], t[rows].transpose(0, 1)], dim=1).double().contiguous()
                for c, t in ((b.kc, b.kt), (b.vc, b.vt)))
        q = b.q[rows].double().reshape(T, b.Hk, G, D).permute(1, 2, 0, 3).reshape(b.Hk, G * T, D).contiguous()
        sees = torch.cat([torch.ones((T, n), dtype=torch.bool), torch.from_numpy(np.asarray(b.sees[s]))], dim=1).cuda().repeat(G, 1)
        kt = k.transpose(1, 2).contiguous()
        a = torch.where(sees, scale * torch.matmul(q, kt), -float("inf"))
        top = a.amax(dim=-1, keepdim=True)
        p = torch.exp(a - torch.where(torch.isinf(top), 0.0, top))
        total = p.sum(dim=-1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        back = lambda x: x.reshape(b.Hk, G, T, -1).permute(2, 0, 1, 3).reshape(T, b.H, -1)  # noqa: E731
        out[rows], bound[rows] = back(torch.matmul(p, v)), back(torch.matmul(p, v.abs()))
        lse[rows] = back(top + torch.log(total))[..., 0]
        most = torch.where(sees, scale * torch.matmul(q.abs(), kt.abs()), 0.0).amax(dim=-1, keepdim=True)
        spread[rows] = back(most)[..., 0]
    return tuple(f64(x) for x in (out, lse, bound, spread))


def test_oracle_of_matrices_is_the_oracle():
    b = Batch("f32", 6, 2, 64, [9, 0, 5], [40, 3, 0], kind="empty", seed=30)
    for x, y in zip(oracle_64(b), b.oracle()):
        assert np.allclose(x, y, rtol=1e-12, atol=1e-12)


LONG_TREES, LONG_LENS = [70, 1, 0, 33, 70, 64, 65, 69], [1409, 1408, 500, 0, 1, 64, 1281, 63]


@pytest.mark.parametrize("kind", ["tree", "chain", "empty"])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_many_rows_in_ragged_batches_that_fill_the_card(D, kind):
    """256 workgroups, one per sequence and KV head; 140 rows: the last waves have some or none."""
    b = Batch("bf16", 64, 32, D, LONG_TREES, LONG_LENS, kind=kind, seed=D)
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("S,H,Hk,T,n", [(1, 64, 16, 40, 20491), (2, 48, 16, 50, 10300), (4, 32, 16, 129, 2650), (1, 64, 16, 131, 6977)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_many_rows_over_parts_of_a_long_cache(S, H, Hk, T, n, kind):
    b = Batch("bf16", H, Hk, 64, [T] + [T - 9] * (S - 1), [n, n // 2, 0, 77][:S], kind=kind, seed=n)
    b.check(*b.attention(), oracle_64(b))


def test_many_rows_of_long_chains_without_a_cache():
    b = Batch("bf16", 32, 16, 64, [2600, 2570], [0, 0], kind="chain", seed=31)
    b.check(*b.attention(), oracle_64(b))


@pytest.mark.parametrize("q_scale", [0.1, 12.0])
def test_many_rows_with_a_maximum_that_rises_along_a_long_cache(q_scale):
    b = Batch("bf16", 64, 32, 128, [70] * 8, [1409] * 8, seed=32, q_scale=q_scale)
    ramp = torch.linspace(0.05, 1.0, b.kc.shape[2], device="cuda")
    b.kc.copy_((b.q[::70, ::2, None, :].float() * 0.3 + b.kc.float() * 0.2) * ramp[None, None, :, None])
    b.kc[:, :, 1409:] = float("nan")
    b.check(*b.attention(), oracle_64(b))


def test_many_rows_and_values_that_are_not_seen_over_a_long_cache():
    b = Batch("bf16", 64, 32, 64, [70] * 8, [1409] * 8, seed=33)
    first = torch.arange(8, device="cuda") * 70
    kt, vt = b.kt, b.vt
    b.kt, b.vt = kt.clone(), vt.clone()
    for t in (3, 40, 68):
        b.kt[first + t], b.vt[first + t] = 0.0, 0.0  # rows that do not see these have the results without them
    want = oracle_64(b)
    b.kt[first + 3], b.vt[first + 3] = float("nan"), float("inf")
    b.vt[first + 40, :, 5] = float("-inf")
    b.vt[first + 68, :, 9] = float("nan")
    out, lse = b.attention()
    sees = np.concatenate(b.sees)
    clean = ~(sees[:, 3] | sees[:, 40] | sees[:, 68])
    assert 0 < clean.sum() < len(clean)
    keep = torch.from_numpy(clean).cuda()
    got, got_lse = out.clone(), lse.clone()
    got[~keep], got_lse[~keep] = 0, 0
    tidy = lambda v: np.where(clean.reshape(-1, *[1] * (v.ndim - 1)), v, 0.0)  # noqa: E731
    b.check(got, got_lse, tuple(tidy(v) for v in want))
    assert np.all(np.isnan(f64(out)[sees[:, 3]]))
    only = sees[:, 40] & ~sees[:, 3] & ~sees[:, 68]
    got = f64(out)[only]
    assert np.all(np.isneginf(got[..., 5])) and np.all(np.isfinite(np.delete(got, 5, axis=-1)))


def test_many_rows_and_infinities_in_a_long_cache():
    """In its whole tiles and in its last entry, beside the places behind it that fill the tile; a score of NaN."""
    b = Batch("bf16", 64, 32, 64, [70] * 8, [1409] * 8, seed=34)
    b.vc[:, :, 1408, 3], b.vc[:, :, 1408, 7], b.vc[:, :, 700, 9] = float("inf"), float("-inf"), float("inf")
    out = f64(b.attention()[0])
    assert np.all(out[:, :, [3, 9]] == np.inf) and np.all(out[:, :, 7] == -np.inf)
    assert np.all(np.isfinite(np.delete(out, [3, 7, 9], axis=-1)))
    b = Batch("bf16", 64, 32, 64, [70] * 8, [1409] * 8, seed=34)
    b.kc[2, :, 30] = float("-inf")  # scores of +-inf: rows of this sequence have no softmax, the others have one
    b.vc[0, :, 17, 3] = float("nan")
    out = f64(b.attention()[0]).reshape(8, 70, 64, 64)
    assert np.all(np.isnan(out[0, :, :, 3])) and np.all(np.isfinite(np.delete(out[0], 3, axis=-1)))
    assert np.all(np.isfinite(out[[1, 3, 4, 5, 6, 7]])) and np.any(np.isnan(out[2]))
