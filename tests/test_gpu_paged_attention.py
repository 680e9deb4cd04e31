"""Attention of single tokens over pages against the fp64 oracle: types, codes, head layouts, lengths, pages, what must not be seen."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb
from attention_common import HALF_STEP, TORCH, f64, i32
from serving_common import Pool

pytestmark = pytest.mark.gpu


def queries(pool, seed=1, scale=2.0):
    d, S = pool.desc, len(pool.lens)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((S, d.n_heads, d.head_dim), generator=gen, device="cuda") * scale).to(TORCH[pool.dtype])


def run(pool, q, **kw):
    return mb.moespec_paged_attention(pool.desc, pool.cache, q, pool.cache_len, max_len=kw.pop("max_len", max(pool.lens)), **kw)


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("code", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_types_and_head_sizes(dtype, code, D):
    pool = Pool(dtype, code, 2, D, [37, 1, 130, 0, 64], 16, seed=D, H=8).poison()
    q = queries(pool)
    pool.check(q, *run(pool, q))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1021])
def test_lengths(n):
    for code in ("plain", "i8", "e4m3"):
        pool = Pool("bf16", code, 1, 64, [n], 32, seed=n, H=4).poison()
        q = queries(pool)
        pool.check(q, *run(pool, q))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_end_inside_of_a_tile(dtype, page):
    pool = Pool(dtype, "plain", 2, 64, [page - 1, page, page + 1, 3 * page + 7], page, seed=page, H=4).poison()
    q = queries(pool)
    pool.check(q, *run(pool, q))


@pytest.mark.parametrize("H,Hk", [(1, 1), (7, 1), (8, 8), (12, 2), (16, 1), (17, 1), (20, 4), (33, 1), (48, 1), (64, 2), (128, 1)])
def test_head_layouts(H, Hk):
    for dtype in ("bf16", "f32"):
        pool = Pool(dtype, "plain", Hk, 64, [200, 33], 16, seed=H, H=H).poison()
        q = queries(pool)
        pool.check(q, *run(pool, q))


@pytest.mark.parametrize("lens", [[5000], [3000, 1, 0, 2999, 700], [17] * 70, [900] * 40 + [0] * 3, list(range(1, 300))])
@pytest.mark.parametrize("code", ["plain", "e4m3"])
def test_batches_in_parts_and_whole(code, lens):
    """One sequence in many parts, sequences that share parts, batches larger than what shares parts."""
    pool = Pool("bf16", code, 2, 64, lens, 16, seed=len(lens), H=4).poison()
    q = queries(pool)
    pool.check(q, *run(pool, q))


def test_long_sequence():
    pool = Pool("bf16", "i8", 1, 128, [65521], 64, seed=3, H=8)
    q = queries(pool)
    pool.check(q, *run(pool, q))


def test_no_entries_at_all():
    pool = Pool("bf16", "plain", 2, 64, [0, 0], 16, H=4)
    q = queries(pool)
    for max_len in (0, 16):
        out, lse = run(pool, q, max_len=max_len)
        assert torch.count_nonzero(out) == 0 and torch.all(lse == -float("inf"))


def test_a_bound_far_above_the_lengths_and_a_layer_of_several():
    pool = Pool("bf16", "i8", 2, 64, [300, 45, 0], 32, seed=8, layers=3, H=8, width=400).poison()
    q = queries(pool)
    for layer in (0, 2):
        pool.check(q, *run(pool, q, max_len=pool.cache.max_entries, layer=layer), layer=layer)


def test_lengths_past_the_bound_are_cut_there():
    pool = Pool("bf16", "plain", 1, 64, [100, 100], 16, seed=4, H=2)
    q = queries(pool)
    out, lse = run(pool, q, max_len=70)
    pool.lens = [70, 70]
    pool.check(q, out, lse)
    pool.cache_len.copy_(i32([-5, 2 ** 31 - 1]))
    out, lse = run(pool, q, max_len=70)
    assert torch.count_nonzero(out[0]) == 0 and torch.all(lse[0] == -float("inf"))
    pool.lens = [0, 70]
    pool.check(q, out, lse)


@pytest.mark.parametrize("code", ["plain", "i8", "e4m3"])
def test_entries_whose_page_is_outside_of_the_pool_are_not_seen(code):
    pool = Pool("bf16", code, 2, 64, [150, 150, 40], 16, seed=9, H=4)
    rows = pool.rows.copy()
    rows[0, [0, 4, 9]] = [-1, pool.cache.k_pages.shape[1], 2 ** 31 - 1]
    rows[2, :] = -7
    pool.cache.page_table.copy_(torch.from_numpy(rows))
    q = queries(pool)
    out, lse = run(pool, q)
    keys, values = pool.values("k"), pool.values("v")
    keep = np.array([e // 16 not in (0, 4, 9) for e in range(150)])
    keys[0], values[0] = keys[0][:, keep], values[0][:, keep]
    keys[2], values[2] = keys[2][:, :0], values[2][:, :0]
    pool.check(q, out, lse, V.attention(f64(q), keys, values, float(np.float32(pool.scale))))


def test_pages_that_sequences_share():
    pool = Pool("bf16", "plain", 2, 64, [90, 90], 16, seed=10, H=4)
    pool.rows[1] = pool.rows[0]
    pool.cache.page_table.copy_(torch.from_numpy(pool.rows))
    q = queries(pool)
    pool.check(q, *run(pool, q))


def test_queries_inside_of_longer_rows_and_given_outputs():
    pool = Pool("bf16", "plain", 2, 128, [77, 300, 12], 16, seed=11, H=8).poison()
    wide = torch.randn((3, 12, 128), device="cuda").to(torch.bfloat16)
    q, out = wide[:, 2:10], torch.full((3, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    got, lse = run(pool, q, out=out)
    assert got is out
    pool.check(q, out, lse)
    call = mb.PagedAttentionCall(pool.desc, pool.cache, q, pool.cache_len,
                                 mb.alloc_paged_attention_workspace(pool.desc, pool.cache, 3, 300), out, None, 300)
    out.fill_(float("nan"))
    call()  # without lse
    pool.check(q, out, lse)


def test_large_scores_and_a_maximum_that_rises_late():
    pool = Pool("f32", "plain", 1, 64, [700], 16, seed=12, H=4, scale=1.0)
    flat = pool.cache.k_pages[0, :, 0]
    for e in (650, 690):  # single keys far above the others, in the last tiles
        flat[pool.rows[0][e // 16], e % 16] *= 6
    q = queries(pool, scale=3.0)
    pool.check(q, *run(pool, q))


@pytest.mark.parametrize("lens", [[5000], [700, 33, 1]])
@pytest.mark.parametrize("dtype,code", [("bf16", "plain"), ("f32", "plain"), ("bf16", "i8"), ("f32", "e4m3")])
def test_scores_whose_rounding_is_larger_than_any_exponent(dtype, code, lens):
    """Scores up to 1.8e10 and down to -1.8e10 (their last bit: 2^11) leave the keys with the largest one alone, which share the row.  Keys are a power of
    two a times a row of signs and queries another times the same signs, so that every product and sum is exact."""
    D, b = 64, 2.0 ** 20
    pool = Pool(dtype, code, 1, D, lens, 16, seed=len(lens), H=4, scale=0.27)
    gen = torch.Generator(device="cuda").manual_seed(5)
    sign = torch.where(torch.rand((D,), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    c = pool.cache
    a = torch.exp2(torch.randint(0, 11, c.k_pages.shape[:-1], generator=gen, device="cuda").float())
    if code == "plain":
        c.k_pages.copy_(a[..., None] * sign)
    else:
        c.k_pages.copy_(sign.expand(c.k_pages.shape).to(c.k_pages.dtype))
        c.k_scale.copy_(a)
    q = (sign * b).expand((len(lens), 4, D)).clone()
    q[:, 1] *= -1.0
    q[:, 2] *= 2.0 ** -20
    q = q.to(TORCH[dtype])
    out, lse = run(pool, q)
    want, want_lse, bound, _ = V.attention(f64(q), pool.values("k"), pool.values("v"), float(np.float32(0.27)))
    # weights are 1 or below 2^-24 of it (head 2: scores of up to 17695, two of which are 17 apart at least)
    rel = (2.0 ** -15 if dtype == "bf16" else 2.0 ** -24) + 2.0 ** -23 + 2 * (max(lens) + 64) * 2.0 ** -24
    u = HALF_STEP[dtype]
    assert np.all(np.abs(f64(out) - want) <= u * np.abs(want) * (1 + 2.0 ** -6) + bound * rel)
    # the scale in units of log 2, its product with a score, the sum with log2 l, ln 2, the product with it: half a step each
    assert np.all(np.abs(f64(lse) - want_lse) <= np.abs(want_lse) * 5 * 2.0 ** -24 * 1.01 + 2.0 ** -15)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity_and_nan(dtype):
    pool = Pool(dtype, "plain", 1, 64, [50, 50, 50], 16, seed=13, H=2)
    k, v = pool.cache.k_pages[0, :, 0], pool.cache.v_pages[0, :, 0]
    q = queries(pool)
    q[:] = q.abs() + 0.5
    for e in range(50):  # every score of the first sequence is -inf; its values hold infinities
        k[pool.rows[0][e // 16], e % 16, 3] = -float("inf")
        v[pool.rows[0][e // 16], e % 16, 5] = float("inf")
    k[pool.rows[1][0], 7, 3] = -float("inf")  # one of the second
    k[pool.rows[2][1], 4, 0] = float("nan")  # a NaN that the third one sees
    out, lse = run(pool, q)
    assert torch.count_nonzero(out[0]) == 0 and torch.all(lse[0] == -float("inf"))
    assert torch.isnan(out[2]).all() and torch.isnan(lse[2]).all()
    keys, values = pool.values("k"), pool.values("v")
    keep = np.arange(50) != 7
    want = V.attention(f64(q[1:2]), [keys[1][:, keep]], [values[1][:, keep]], float(np.float32(pool.scale)))
    pool.lens = [50]
    pool.check(q[1:2], out[1:2], lse[1:2], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_infinity_that_are_seen_stay_infinities(dtype):
    """Under weights that bf16 holds exactly (a single key: 1) and under others."""
    pool = Pool(dtype, "plain", 1, 64, [1, 70, 300], 16, seed=21, H=4)
    v, inf = pool.cache.v_pages[0, :, 0], float("inf")
    for s, e, d, x in ((0, 0, 3, inf), (0, 0, 9, -inf), (1, 69, 5, -inf), (2, 33, 60, inf)):
        v[pool.rows[s][e // 16], e % 16, d] = x
    q = queries(pool)
    out, lse = run(pool, q)
    for s, d, x in ((0, 3, inf), (0, 9, -inf), (1, 5, -inf), (2, 60, inf)):
        assert torch.all(out[s, :, d] == x)
        out[s, :, d] = 0
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_rows_whose_scale_is_nan_make_only_their_own_sequence_nan():
    pool = Pool("bf16", "i8", 1, 64, [40, 40], 16, seed=14, H=2)
    pool.cache.v_scale[0, pool.rows[0][1], 0, 3] = float("nan")
    q = queries(pool)
    out, lse = run(pool, q)
    assert torch.isnan(out[0]).all()
    keys, values = pool.values("k"), pool.values("v")
    want = V.attention(f64(q[1:]), keys[1:], values[1:], float(np.float32(pool.scale)))
    pool.lens = [40]
    pool.check(q[1:], out[1:], lse[1:], want)


def test_offsets_behind_32_bits():
    """The last pages of a pool of more than 2^32 bytes and elements."""
    d = mb.AttnDesc(2, 1, 256, 1, mb.BF16)
    n = (1 << 32) // (256 * 256) + 3
    k, v = (torch.zeros((1, n, 1, 256, 256), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((1, n, 1, 256), device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = np.array([[n - 1, 0, n - 2]], dtype=np.int32)
    for p in rows[0]:
        for t, s in ((k, ks), (v, vs)):
            t[0, p] = torch.randint(-127, 128, (1, 256, 256), generator=gen, device="cuda", dtype=torch.int8)
            s[0, p] = torch.rand((1, 256), generator=gen, device="cuda") * 0.02
    cache = mb.PagedCache(mb.CACHE_I8, k, v, torch.from_numpy(rows).cuda(), ks, vs)
    q = torch.randn((1, 2, 256), generator=gen, device="cuda").to(torch.bfloat16)
    out, lse = mb.moespec_paged_attention(d, cache, q, i32([700]), max_len=768)
    keys, values = (np.concatenate([f64(t[0, p]) * f64(s[0, p])[..., None] for p in rows[0]], axis=1)[:, :700]
                    for t, s in ((k, ks), (v, vs)))
    want, want_lse, _, _ = V.attention(f64(q), [keys], [values], 1 / 16)
    # half a step of the output and 2^-10 for sums over 700 keys: the places are what is tested
    assert np.all(np.abs(f64(out) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(values).max())
    assert np.all(np.abs(f64(lse) - want_lse) <= 1e-4)


def test_bit_identical_runs_and_graph_replays():
    pool = Pool("bf16", "e4m3", 4, 128, [1500, 20, 333, 0], 32, seed=15, H=32, width=64)
    q = queries(pool)
    ws = mb.alloc_paged_attention_workspace(pool.desc, pool.cache, 4, 2000)
    out, lse = torch.zeros_like(q), torch.zeros((4, 32), device="cuda")
    pool2 = Pool("bf16", "e4m3", 4, 128, [800, 1700, 5, 64], 32, seed=16, H=32, width=64)
    out2, lse2 = torch.zeros_like(q), torch.zeros((4, 32), device="cuda")
    a = mb.PagedAttentionCall(pool.desc, pool.cache, q, pool.cache_len, ws, out, lse, 2000)
    b = mb.PagedAttentionCall(pool2.desc, pool2.cache, q, pool2.cache_len, ws, out2, lse2, 2000)
    a(), b()
    first = [t.clone() for t in (out, lse, out2, lse2)]
    stream, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in range(2)]
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for g, call in zip(graphs, (a, b)):  # two graphs that share a workspace, replayed in turn
            with torch.cuda.graph(g, stream=stream):
                call()
        for _ in range(4):
            for t in (out, lse, out2, lse2):
                t.fill_(7)
            graphs[0].replay(), graphs[1].replay()
            stream.synchronize()
            for got, want in zip((out, lse, out2, lse2), first):
                assert torch.equal(got, want)
    # the lengths are device data: a captured call follows them
    with torch.cuda.stream(stream):
        pool.cache_len.copy_(i32([1501 - 40, 21, 300, 1]))
        graphs[0].replay()
        stream.synchronize()
    pool.lens = [1461, 21, 300, 1]
    pool.rows[3, 0] = 0  # (the table has -1 there)
    keys, values = pool.values("k"), pool.values("v")
    keys[3], values[3] = keys[3][:, :0], values[3][:, :0]  # (that sequence has no page)
    pool.check(q, out, lse, V.attention(f64(q), keys, values, float(np.float32(pool.scale))))


def test_the_most_query_heads():
    for dtype, H, Hk in (("bf16", 1024, 1), ("f32", 1024, 512)):
        pool = Pool(dtype, "plain", Hk, 64, [40, 3], 16, seed=22, H=H).poison()
        q = queries(pool)
        pool.check(q, *run(pool, q))


FAR = {"plain": (2.0 ** 12, 2.0 ** 11), "i8": (2.0 ** 16, 127.0), "e4m3": (2.0 ** 15, 256.0)}  # element 0 of queries and of the two keys


@pytest.mark.parametrize("lens,pairs", [([128] * 4, [(5, 9), (5, 40), (69, 120), (3, 69)]),             # one part: a wave's tile, two waves, two tiles
                                        ([5000, 2000, 700], [(5, 4990), (1990, 40), (100, 690)]),       # parts that sequences share
                                        ([5000], [(4000, 2)])])                                         # parts of one sequence
@pytest.mark.parametrize("dtype,code", [("bf16", "plain"), ("f32", "plain"), ("bf16", "i8"), ("f32", "i8"), ("bf16", "e4m3"), ("f32", "e4m3")])
def test_neighbouring_scores_far_from_zero_weigh_what_their_difference_says(dtype, code, lens, pairs):
    """Two keys of every sequence have scores around 2^23 that are 0, 1, 2 and 5 apart, whole numbers throughout, so that scores are exact; the
    others have the score 0, and no weight.  Wherever the two fall, the rest follows from the difference alone: a bound that does not grow with
    the scores."""
    D, diffs = 64, [0.0, 1.0, 2.0, 5.0]
    pool = Pool(dtype, code, 1, D, lens, 16, seed=7, H=4, scale=1.0)
    a, b = FAR[code]
    k = torch.zeros((pool.cache.k_pages.shape[1], 16, D), device="cuda")
    for s, (e0, e1) in enumerate(pairs):
        for e, one in ((e0, 1.0), (e1, 0.0)):
            k[int(pool.rows[s][e // 16]), e % 16, 0] = b
            k[int(pool.rows[s][e // 16]), e % 16, 1] = one
    pool.cache.k_pages.copy_(k.to(pool.cache.k_pages.dtype)[None, :, None])
    if code != "plain":
        pool.cache.k_scale.fill_(1.0)
    q = torch.zeros((len(lens), 4, D), device="cuda")
    q[:, :, 0], q[:, :, 1] = a, torch.tensor(diffs, device="cuda")
    q = q.to(TORCH[dtype])
    out, lse = run(pool, q)
    want, want_lse, bound, _ = V.attention(f64(q), pool.values("k"), pool.values("v"), 1.0)
    # the scale in units of log 2 and its product with the difference: half a step each of 5 / ln 2, times ln 2; two exponentials, sums and quotients
    # of two keys; the parts of a weight
    rel = 2 * 5 * 2.0 ** -24 + 16 * 2.0 ** -24 + (2.0 ** -15 if dtype == "bf16" else 2.0 ** -23)
    assert np.all(np.abs(f64(out) - want) <= HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -6) + bound * rel)
    # the scale in units of log 2, its product with a score, the sum with log2 l, ln 2, the product with it: half a step each
    assert np.all(np.abs(f64(lse) - want_lse) <= np.abs(want_lse) * 5 * 2.0 ** -24 * 1.01)


@pytest.mark.parametrize("n", [300, 3000])  # a part, and parts
@pytest.mark.parametrize("dtype,code", [("bf16", "plain"), ("f32", "plain"), ("bf16", "i8"), ("f32", "i8"), ("bf16", "e4m3"), ("f32", "e4m3")])
def test_large_values_under_a_maximum_that_rises_a_little(dtype, code, n):
    """Results are finite, so they are computed: values of 2^117 and more under weights that a later key passes by e^5, hundreds of them under the
    same weight (the head of negative queries), whose plain sum is beyond the largest number, and a single value of 96 * 2^121."""
    D = 64
    pool = Pool(dtype, code, 1, D, [n, n], 16, seed=11, H=4, scale=1.0)
    c, gen = pool.cache, torch.Generator(device="cuda").manual_seed(12)
    top = [[e % n for e in (133, 134, n - 5, n - 133)], [133]]
    k = torch.zeros((c.k_pages.shape[1], 16, D), device="cuda")
    v = torch.zeros_like(k)
    size = 2.0 ** 120 * (1.0 if n == 300 else 2.0 ** -3)
    v[torch.from_numpy(pool.rows[0][: -(-n // 16)].astype(np.int64)).cuda()] = torch.randint(64, 128, (-(-n // 16), 16, D), generator=gen,
                                                                                           device="cuda").float() / 64
    if code == "e4m3":
        v = v.to(torch.float8_e4m3fn).float()
    for s in range(2):
        for e in top[s]:
            k[int(pool.rows[s][e // 16]), e % 16, 0] = 5.0
    scale = torch.full((c.k_pages.shape[1], 16), size, device="cuda")
    p, i = int(pool.rows[1][133 // 16]), 133 % 16
    v[p, i], scale[p, i] = 96.0, 2.0 ** 121
    q = torch.zeros((2, 4, D), device="cuda")
    q[:, :, 0] = torch.tensor([1.0, 0.5, -1.0, 0.75], device="cuda")
    q = q.to(TORCH[dtype])
    if code == "plain":
        c.k_pages.copy_(k[None, :, None])
        c.v_pages.copy_((v * scale[..., None])[None, :, None])
    else:
        held = 64.0 if code == "i8" else 1.0  # (96 * 64 is no int8: the single value's code stays 96)
        wide = v * held
        wide[p, i] = 96.0
        scale = scale / held
        scale[p, i] = 2.0 ** 121
        c.k_pages.copy_(k.to(c.k_pages.dtype)[None, :, None])
        c.v_pages.copy_(wide.to(c.v_pages.dtype)[None, :, None])
        c.k_scale.fill_(1.0)
        c.v_scale.copy_(scale[None, :, None])
    out, lse = run(pool, q)
    assert torch.isfinite(out.float()).all()
    pool.check(q, out, lse)


def test_the_logarithm_of_a_row_whose_scores_are_near_the_largest_number():
    """lse is the score itself (3e38), though log2(e) times it is no number."""
    pool = Pool("f32", "plain", 1, 64, [1, 700], 16, seed=13, H=4, scale=1.0)
    pool.cache.k_pages.zero_()
    for s in range(2):
        pool.cache.k_pages[0, int(pool.rows[s][0]), 0, 0, 0] = 1.5 * 2.0 ** 63
    q = torch.zeros((2, 4, 64), device="cuda")
    q[:, :, 0] = 2.0 ** 64
    out, lse = run(pool, q)
    values = pool.values("v")
    for s in range(2):
        assert np.array_equal(f64(out[s]), np.broadcast_to(values[s][0, :1], (4, 64)))
    # c, ln 2, their product, the score's with it: half a step each
    assert np.all(np.abs(f64(lse) / (1.5 * 2.0 ** 127) - 1) <= 4 * 2.0 ** -24 * 1.01)


@pytest.mark.parametrize("lens", [[3000, 40], [120]])
@pytest.mark.parametrize("dtype,code", [("bf16", "plain"), ("f32", "plain"), ("bf16", "i8"), ("f32", "i8"), ("bf16", "e4m3"), ("f32", "e4m3")])
def test_small_values_keep_their_bits(dtype, code, lens):
    """Values (codes: scales) down to about 3000 * 2^-102."""
    pool = Pool(dtype, code, 2, 64, lens, 16, seed=17, H=8)
    if code == "plain":
        pool.cache.v_pages.mul_(2.0 ** -86)
    else:
        pool.cache.v_scale.mul_(2.0 ** -82)
    q = queries(pool)
    pool.check(q, *run(pool, q))
