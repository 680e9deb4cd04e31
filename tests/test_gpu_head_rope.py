"""Norm and rotation of queries and keys against the fp64 oracle: types, head sizes, partial and interleaved rotation, places from
trees and given ones, strides and in place, rows that are not touched."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb
from attention_common import CODE, HALF_STEP, TORCH, f64, i32, random_tree

pytestmark = pytest.mark.gpu


def freqs(rot, base=1e6):
    return torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float32, device="cuda") if rot else None


def check(x, w, place, freq, rot, got, dtype, rows=None, **kw):
    w = None if w is None else f64(w)
    fr = np.zeros(0) if freq is None else f64(freq)
    want, size = V.head_rope(f64(x), w, place, fr, rot, **kw)
    D, u = x.shape[2], HALF_STEP[dtype]
    # the sum of squares (a step a term, halved by the root), its root, quotient and weight; cosine, sine (with what is left of the angle
    # rounded: 2.4e-8 and a few steps of the functions), two products and their sum
    rel = ((D / 2 + 8) + 16) * 2.0 ** -24
    tol = u * np.abs(want) * (1 + 2.0 ** -6) + size * rel + 1e-37
    err = np.abs(f64(got) - want)
    if rows is not None:
        err, tol = err[rows], tol[rows]
    assert np.all(err <= tol), f"off by {np.nanmax(err / tol):.2f} of the bound"


def data(dtype, M, H, Hk, D, seed=0, fused=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TORCH[dtype]
    if fused:
        qkv = (torch.randn((M, H + 2 * Hk, D), generator=gen, device="cuda") * 3).to(dt)
        return qkv[:, :H], qkv[:, H:H + Hk], qkv
    q, k = ((torch.randn((M, n, D), generator=gen, device="cuda") * 3).to(dt) for n in (H, Hk))
    return q, k, None


def weights(dtype, D, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(1 + torch.randn(D, generator=gen, device="cuda") * 0.3).to(TORCH[dtype]) for _ in range(2)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rots", [(64, (64, 16, 48)), (96, (96, 32, 80)), (128, (128, 0, 64)), (192, (192, 112)), (256, (256, 16, 240))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_types_heads_and_rotated_parts(dtype, D, rots, interleaved):
    for rot in rots:
        H, Hk, M = 5, 1, 13
        q, k, _ = data(dtype, M, H, Hk, D, seed=D + rot)
        wq, wk = weights(dtype, D)
        d = mb.AttnDesc(H, Hk, D, 1, CODE[dtype])
        fr, place = freqs(rot), np.arange(M) + 1000
        for norm, ws in ((True, (wq, wk)), (True, (None, None)), (False, (None, None))):
            kw = dict(interleaved=interleaved, norm=norm, eps=1e-6 if norm else 0.0)
            qo, ko = mb.moespec_head_rope(d, q, k, freq=fr, rot_dim=rot, w_q=ws[0], w_k=ws[1], cache_len=i32([1000]), **kw)
            check(q, ws[0], place, fr, rot, qo, dtype, **kw)
            check(k, ws[1], place, fr, rot, ko, dtype, **kw)


@pytest.mark.parametrize("H,Hk", [(1, 1), (7, 1), (32, 4), (64, 8), (40, 40)])
def test_head_layouts_and_single_tokens(H, Hk):
    for M in (1, 2):
        q, k, _ = data("bf16", M, H, Hk, 128, seed=H)
        wq, wk = weights("bf16", 128)
        d, fr = mb.AttnDesc(H, Hk, 128, 1, mb.BF16), freqs(128)
        qo, ko = mb.moespec_head_rope(d, q, k, freq=fr, norm=True, w_q=wq, w_k=wk, eps=1e-6)
        check(q, wq, np.arange(M), fr, 128, qo, "bf16", norm=True, eps=1e-6)
        check(k, wk, np.arange(M), fr, 128, ko, "bf16", norm=True, eps=1e-6)


@pytest.mark.parametrize("masked", [False, True])
def test_places_of_trees_of_a_batch(masked):
    """Trees of 0 to 70 tokens behind caches of their own, with rows of no sequence in front of the end that stay as they were."""
    rng = np.random.default_rng(1)
    trees, lens, pad = [70, 0, 1, 33, 64, 5], [1000003, 7, 0, 31, 65535, 2], 4
    sees = [random_tree(rng, n) if masked else A.chain(n) for n in trees]
    off = np.concatenate([[0], np.cumsum(trees)])
    M = int(off[-1]) + pad
    for dtype in ("bf16", "f32"):
        q, k, _ = data(dtype, M, 4, 2, 64, seed=2)
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        mask = torch.from_numpy(A.pack(sees, M, 70, fill=1)).cuda() if masked else None
        d, fr = mb.AttnDesc(4, 2, 64, 1, CODE[dtype]), freqs(64, 1e4)
        mb.moespec_head_rope(d, q, k, qo, ko, fr, cache_len=i32(lens), tree_off=i32(off), tree_mask=mask, max_tree=70)
        place = np.concatenate([V.places(lens, off, sees), np.zeros(pad)])
        used = slice(0, int(off[-1]))
        check(q, None, place, fr, 64, qo, dtype, rows=used)
        check(k, None, place, fr, 64, ko, dtype, rows=used)
        assert torch.all(qo[off[-1]:] == 7) and torch.all(ko[off[-1]:] == 7)


def test_rows_past_the_largest_tree_and_many_sequences():
    trees = [3] * 150
    off = np.concatenate([[0], np.cumsum(trees)])
    q, k, _ = data("f32", 450, 1, 1, 64)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    d, fr, lens = mb.AttnDesc(1, 1, 64, 1, mb.F32), freqs(64), np.arange(150) * 11
    mb.moespec_head_rope(d, q, k, qo, ko, fr, cache_len=i32(lens), tree_off=i32(off), max_tree=2)
    place = V.places(lens, off, [A.chain(3)] * 150)
    rows = np.arange(450) % 3 < 2
    check(q, None, place, fr, 64, qo, "f32", rows=rows)
    assert torch.all(qo[~torch.from_numpy(rows).cuda()] == 7)


def test_given_places_near_and_far():
    place = np.array([0, 1, 2 ** 20 + 1, 2 ** 31 - 1, 5, 0, 123456789])
    for dtype in ("bf16", "f32"):
        q, k, _ = data(dtype, 7, 3, 3, 128)
        d, fr = mb.AttnDesc(3, 3, 128, 1, CODE[dtype]), freqs(128)
        qo, ko = mb.moespec_head_rope(d, q, k, freq=fr, positions=i32(place))
        check(q, None, place.astype(np.float64), fr, 128, qo, dtype)
        check(k, None, place.astype(np.float64), fr, 128, ko, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_inside_of_a_projection(dtype):
    q, k, qkv = data(dtype, 9, 8, 2, 96, fused=True)
    before = qkv.clone()
    wq, wk = weights(dtype, 96)
    d, fr = mb.AttnDesc(8, 2, 96, 1, CODE[dtype]), freqs(96)
    mb.moespec_head_rope(d, q, k, q, k, fr, norm=True, w_q=wq, w_k=wk, eps=1e-5, cache_len=i32([77]))
    assert torch.equal(qkv[:, 10:], before[:, 10:])  # the values
    check(before[:, :8], wq, np.arange(9) + 77, fr, 96, q, dtype, norm=True, eps=1e-5)
    check(before[:, 8:10], wk, np.arange(9) + 77, fr, 96, k, dtype, norm=True, eps=1e-5)


def test_queries_or_keys_alone_and_views_as_outputs():
    q, k, _ = data("bf16", 6, 4, 2, 64)
    d, fr = mb.AttnDesc(4, 2, 64, 1, mb.BF16), freqs(64)
    qo, none = mb.moespec_head_rope(d, q, None, freq=fr)
    assert none is None
    check(q, None, np.arange(6), fr, 64, qo, "bf16")
    room = torch.full((6, 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    mb.moespec_head_rope(d, None, k, None, room[:, 3:5], fr)
    check(k, None, np.arange(6), fr, 64, room[:, 3:5], "bf16")
    assert torch.all(room[:, :3] == 5) and torch.all(room[:, 5:] == 5)


def test_heads_of_zeros_and_not_finite_values():
    q, k, _ = data("f32", 3, 2, 1, 64)
    q[0, 0] = 0
    q[1, 1, 5] = float("inf")
    k[2, 0, 0] = float("nan")
    d, fr = mb.AttnDesc(2, 1, 64, 1, mb.F32), freqs(64)
    qo, ko = mb.moespec_head_rope(d, q, k, freq=fr, norm=True, eps=1e-6)
    assert torch.count_nonzero(qo[0, 0]) == 0 and torch.isnan(ko[2]).all()
    assert torch.isfinite(qo[0, 1]).all() and torch.isfinite(qo[1, 0]).all() and torch.isfinite(qo[2]).all()


def test_a_captured_call_follows_the_lengths():
    q, k, _ = data("bf16", 2, 4, 2, 128)
    d, fr, lens = mb.AttnDesc(4, 2, 128, 1, mb.BF16), freqs(128), i32([5, 900])
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    call = mb.HeadRopeCall(d, q, k, qo, ko, fr, cache_len=lens, tree_off=i32([0, 1, 2]), max_tree=1)
    call()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            call()
        for step in range(4):
            qo.fill_(7), ko.fill_(7)
            graph.replay()
            stream.synchronize()
            place = np.array([5 + step, 900 + 7 * step], dtype=np.float64)
            check(q, None, place, fr, 128, qo, "bf16")
            check(k, None, place, fr, 128, ko, "bf16")
            lens += i32([1, 7])


TWO_OVER_PI = Fraction(63661977236758134307553505349005744813783858296182579499066937623558719053690614036045521106501234, 10 ** 98)


def test_angles_of_far_places_against_exact_ones():
    """Cosine and sine themselves (pairs of 1 and 0) at places up to 2^31 and frequencies up to a thousand, against angles that were reduced as
    fractions: as exact at the last place as at the first."""
    place = [0, 1, -7, 2 ** 20 + 1, 2 ** 24 + 1, 123456789, 2 ** 28 + 3, 2 ** 31 - 1, 2 ** 31 - 10007]
    freq = torch.cat([freqs(128), torch.tensor([3.0, 17.3, 0.9999, 1000.3, 999.7, 2.5, 1.5707964, 0.1], device="cuda")])
    D = 256
    q = torch.zeros((len(place), 1, D), device="cuda")
    q[:, :, :72] = 1.0
    out, _ = mb.moespec_head_rope(mb.AttnDesc(1, 1, D, 1, mb.F32), q, None, freq=freq, rot_dim=144, positions=i32(place))
    turns = [[Fraction(p) * Fraction(float(f)) * TWO_OVER_PI for f in freq.tolist()] for p in place]
    angle = np.array([[float(t - 4 * round(t / 4)) for t in row] for row in turns]) * (np.pi / 2)
    # the angle: half a step of a quarter turn's half; sine and cosine: two steps below 1 (the products with 1 and 0 are exact)
    tol = 2.4e-8 + 2 * 2.0 ** -24
    assert np.max(np.abs(f64(out[:, 0, :72]) - np.cos(angle))) <= tol
    assert np.max(np.abs(f64(out[:, 0, 72:144]) - np.sin(angle))) <= tol
