"""Outputs that overlap something else a call uses are refused before any device work (made-up addresses; every call here is refused)."""
import ctypes
import os

import pytest

from paper_2602_16052_amd import binding as mb

MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mb.LIB_PATH):
        from paper_2602_16052_amd import build
        build.build_library()
    return mb.load_library()


def places(sizes):
    """An address for every name, each 1 MB behind the end of the one before it."""
    at, out = 16 * MB, {}
    for name, size in sizes.items():
        out[name] = at
        at += -(-(size + MB) // MB) * MB
    return out


def check(call, sizes, written, same=()):
    """call(addresses) has to be refused wherever one of `written` starts inside of something else, or ends there."""
    base = places(sizes)
    for w in written:
        for other in sizes:
            if other == w:
                continue
            # the last place of 256 bytes in the other one, the first one that still reaches into it, and its own place
            for at in (base[other] + (sizes[other] - 1) // 256 * 256, base[other] - (sizes[w] - 1) // 256 * 256, base[other]):
                if at == base[other] and (w, other) in same:
                    continue
                assert call({**base, w: at}) == mb.ERR_INVALID_ARG, (w, other, at - base[other])


S, M, T, H, HK, D, CAP = 2, 16, 8, 8, 2, 64, 100
DESC = mb.AttnDesc(H, HK, D, CAP, mb.BF16)


def tree(p, q_stride=0, kv_stride=0):
    return mb.Tree(S, M, T, q_stride, kv_stride, p.get("tree_off"), p.get("tree_mask"))


COMMON = dict(q=M * H * D * 2, k_tree=M * HK * D * 2, tree_off=4 * (S + 1), tree_mask=4 * M, k_cache=S * HK * CAP * D * 2, cache_len=4 * S)


def test_tree_attention(lib):
    need = mb.attn_workspace_bytes(DESC, S, M, T, CAP)
    sizes = dict(COMMON, v_tree=M * HK * D * 2, v_cache=S * HK * CAP * D * 2, out=M * H * D * 2, lse=4 * M * H, ws=need)
    cd = DESC.c()

    def call(p):
        t = tree(p)
        return lib.moespec_tree_attention(ctypes.byref(cd), ctypes.byref(t), p["q"], p["k_tree"], p["v_tree"], p["k_cache"], p["v_cache"],
                                          p["cache_len"], CAP, p["out"], p["lse"], p["ws"], need, None)

    check(call, sizes, ("out", "lse", "ws"))


def test_rows_that_are_further_apart_reach_further(lib):
    need = mb.attn_workspace_bytes(DESC, S, M, T, CAP)
    stride = (H + 2 * HK) * D
    sizes = dict(COMMON, q=((M - 1) * stride + H * D) * 2, k_tree=((M - 1) * stride + HK * D) * 2, v_tree=M * stride * 2,
                 v_cache=S * HK * CAP * D * 2, out=M * H * D * 2, lse=4 * M * H, ws=need)
    cd = DESC.c()

    def call(p):
        t = tree(p, stride, stride)
        return lib.moespec_tree_attention(ctypes.byref(cd), ctypes.byref(t), p["q"], p["k_tree"], p["v_tree"], p["k_cache"], p["v_cache"],
                                          p["cache_len"], CAP, p["out"], p["lse"], p["ws"], need, None)

    base = places(sizes)
    for other in ("q", "k_tree", "v_tree"):
        assert call({**base, "out": base[other] + (M - 1) * stride * 2}) == mb.ERR_INVALID_ARG, other


def test_cache_weights(lib):
    need = mb.attn_workspace_bytes(DESC, S, M, T, CAP)
    w = 4 * S * HK * CAP
    sizes = dict(COMMON, lse=4 * M * H, row_weight=4 * M, w_in=w, w_out=w, tree_w=4 * M * HK, ws=need)
    cd = DESC.c()

    def call(p):
        t = tree(p)
        return lib.moespec_cache_weights(ctypes.byref(cd), ctypes.byref(t), p["q"], p["k_tree"], p["k_cache"], p["cache_len"], CAP,
                                         p["lse"], p["row_weight"], 0.5, p["w_in"], p["w_out"], p["tree_w"], p["ws"], need, None)

    check(call, sizes, ("w_out", "tree_w", "ws"), same={("w_out", "w_in")})


def test_cache_commit(lib):
    L, P = 3, 5
    cache = L * S * HK * CAP * D * 2
    sizes = dict(k_tree=L * M * HK * D * 2, v_tree=L * M * HK * D * 2, tree_off=4 * (S + 1), tree_w=4 * L * M * HK, path=4 * S * P, n_path=4 * S,
                 k_cache=cache, v_cache=cache, cache_w=4 * L * S * HK * CAP, cache_len=4 * S, new_len=4 * S)
    cd = DESC.c()

    def call(p):
        t = tree(p)
        return lib.moespec_cache_commit(ctypes.byref(cd), L, ctypes.byref(t), p["k_tree"], p["v_tree"], p["tree_w"], p["path"],
                                        p["n_path"], P, p["k_cache"], p["v_cache"], p["cache_w"], p["cache_len"], p["new_len"], None)

    check(call, sizes, ("k_cache", "v_cache", "cache_w", "new_len"))


@pytest.mark.parametrize("with_list", [False, True])
def test_cache_evict(lib, with_list):
    L, B, room = 3, 50, 60
    heads = L * S * HK
    need = mb.evict_workspace_bytes(DESC, L, S, B)
    sizes = dict(k_cache=heads * CAP * D * 2, v_cache=heads * CAP * D * 2, cache_w=4 * heads * CAP, cache_len=4 * S, k_out=heads * room * D * 2,
                 v_out=heads * room * D * 2, w_out=4 * heads * room, new_len=4 * S)
    sizes["kept" if with_list else "ws"] = 4 * heads * B
    cd = DESC.c()

    def call(p):
        return lib.moespec_cache_evict(ctypes.byref(cd), L, S, p["k_cache"], p["v_cache"], p["cache_w"], p["cache_len"], B, 10, room,
                                       p["k_out"], p["v_out"], p["w_out"], p.get("kept"), p["new_len"], p.get("ws", 1 << 40), need, None)

    check(call, sizes, ("k_out", "v_out", "w_out", "new_len") + (("kept",) if with_list else ("ws",)))


@pytest.mark.parametrize("kind", [mb.BLOCK_GATE_CHANNEL, mb.BLOCK_GATE_TOKEN, mb.BLOCK_GATE_ELEMENT])
def test_block_norm(lib, kind):
    d, n = 256, 33
    gate = {mb.BLOCK_GATE_CHANNEL: d, mb.BLOCK_GATE_TOKEN: n, mb.BLOCK_GATE_ELEMENT: n * d}[kind] * 4
    sizes = dict(y=4 * n * d, residual=4 * n * d, gate=gate, w_post=4 * d, w_pre=4 * d, r=4 * n * d, x=4 * n * d)
    cd = mb.LayerDesc(d, 1, 1, d, mb.F32, False).c()

    def call(p):
        b = mb.Block(1, kind, 0, 1.0, 1e-6, p["w_post"], p["gate"], p["w_pre"])
        return lib.moespec_block_norm(ctypes.byref(cd), ctypes.byref(b), p["y"], p["residual"], n, p["r"], p["x"], None)

    same = {(o, i) for o in ("r", "x") for i in ("y", "residual") + (("gate",) if kind == mb.BLOCK_GATE_ELEMENT else ())}
    check(call, sizes, ("r", "x"), same)
