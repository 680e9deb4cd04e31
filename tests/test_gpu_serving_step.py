"""Serving steps as a program runs them: queries and keys out of one projection normed and rotated in place; prompts written to pages;
steps of single tokens over the pages; drafted trees verified over the pages laid out as a contiguous cache, the accepted path and the
next token taken from logits, the path written to the pages.  Every call is checked against the oracle on the inputs it had, the pages
against a copy that is kept by hand."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb

from attention_common import CODE, HALF_STEP, TORCH, Batch, f64, i32
from serving_common import KIND, Pool, table

pytestmark = pytest.mark.gpu


def check_rope(before, w, place, freq, got, dtype, eps):
    want, size = V.head_rope(f64(before), f64(w), place, f64(freq), before.shape[2], norm=True, eps=eps)
    tol = HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -6) + size * (before.shape[2] / 2 + 24) * 2.0 ** -24
    assert np.all(np.abs(f64(got) - want) <= tol)


def stored(rows, code, dtype):
    """Rows [n, D] (float64) as they are read back from pages."""
    if code == "plain":
        return rows
    codes, scale = (V.codes_i8 if code == "i8" else V.codes_e4m3)(rows)
    return f64(torch.from_numpy(codes.astype(np.float32) * scale[:, None]).to(TORCH[dtype]))


@pytest.mark.parametrize("dtype,code,H,Hk,D", [("bf16", "e4m3", 8, 2, 64), ("bf16", "plain", 4, 4, 128), ("f32", "i8", 6, 2, 96)])
def test_prompts_single_tokens_and_drafted_trees(dtype, code, H, Hk, D):
    S, L, page, vocab, eps = 2, 2, 16, 300, 1e-6
    rng, gen = np.random.default_rng(3), torch.Generator(device="cuda").manual_seed(3)
    dt = TORCH[dtype]
    randn = lambda *s, scale=1.0: (torch.randn(s, generator=gen, device="cuda") * scale).to(dt)  # noqa: E731
    w_q, w_k = [(1 + torch.randn(D, generator=gen, device="cuda") * 0.2).to(dt) for _ in range(2)]
    freq = torch.tensor([1e4 ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float32, device="cuda")
    rows, pool = table([200] * S, page, rng)
    desc = mb.AttnDesc(H, Hk, D, 160, CODE[dtype])
    cache = mb.alloc_paged_cache(desc, KIND[code], pool, page, torch.from_numpy(rows).cuda(), L)
    scale = float(np.float32(D ** -0.5))
    lens, hand = [0, 0], [[(np.zeros((Hk, 0, D)), np.zeros((Hk, 0, D))) for _ in range(S)] for _ in range(L)]
    cache_len = i32(lens)

    def ready(sees, off, mask, most):
        """Projections of all layers, normed and rotated in place."""
        M = int(off[-1])
        qkv = randn(L, M, H + 2 * Hk, D, scale=1.5)
        place = V.places(lens, off, sees)
        for l in range(L):
            before = qkv[l].clone()
            q, k = qkv[l, :, :H], qkv[l, :, H:H + Hk]
            mb.moespec_head_rope(desc, q, k, q, k, freq, norm=True, w_q=w_q, w_k=w_k, eps=eps, cache_len=cache_len, tree_off=i32(off),
                                 tree_mask=mask, max_tree=most)
            check_rope(before[:, :H], w_q, place, freq, q, dtype, eps)
            check_rope(before[:, H:H + Hk], w_k, place, freq, k, dtype, eps)
            assert torch.equal(qkv[l, :, H + Hk:], before[:, H + Hk:])
        return qkv

    def append(qkv, off, paths):
        for l in range(L):
            k, v = f64(qkv[l, :, H:H + Hk]), f64(qkv[l, :, H + Hk:])
            for s, p in enumerate(paths):
                at = [int(off[s]) + t for t in p]
                new = [np.stack([stored(x[at, g], code, dtype) for g in range(Hk)]) for x in (k, v)]
                hand[l][s] = tuple(np.concatenate([a, b], axis=1) for a, b in zip(hand[l][s], new))

    def dense():
        """The pages as a contiguous cache, checked against the copy."""
        kc, vc = mb.moespec_paged_read(desc, cache, cache_len)
        for l in range(L):
            for s, n in enumerate(lens):
                assert np.array_equal(f64(kc[l, s, :, :n]), hand[l][s][0]) and np.array_equal(f64(vc[l, s, :, :n]), hand[l][s][1])
        return kc, vc

    # prompts
    trees = [37, 21]
    off = np.concatenate([[0], np.cumsum(trees)])
    qkv = ready([A.chain(n) for n in trees], off, None, 37)
    cache_len = mb.moespec_paged_write(desc, cache, qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:], cache_len, tree_off=i32(off), max_tree=37)
    append(qkv, off, [range(n) for n in trees])
    lens = list(trees)
    assert cache_len.tolist() == lens
    dense()
    for step in range(4):
        if step % 2 == 0:  # a single token of every sequence
            off = np.arange(S + 1)
            qkv = ready([A.chain(1)] * S, off, None, 1)
            cache_len = mb.moespec_paged_write(desc, cache, qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:], cache_len, tree_off=i32(off), max_tree=1)
            append(qkv, off, [[0]] * S)
            lens = [n + 1 for n in lens]
            kc, vc = dense()
            check = Pool.__new__(Pool)
            check.dtype, check.lens, check.desc = dtype, lens, desc
            for l in range(L):
                q = qkv[l, :, :H]
                out, lse = mb.moespec_paged_attention(desc, cache, q, cache_len, max_len=max(lens), layer=l)
                # over what the pages hold, before it is rounded to the layer's type: codes times scales
                values = []
                for pages, scales in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
                    x = f64(pages[l].float()) * (1.0 if scales is None else f64(scales[l])[..., None])
                    values.append([np.concatenate([x[p] for p in rows[s]], axis=1)[:, :n] for s, n in enumerate(lens)])
                check.check(q, out, lse, V.attention(f64(q), *values, scale))
            continue
        trees = [int(rng.integers(6, 20)), int(rng.integers(1, 9))]
        off, most = np.concatenate([[0], np.cumsum(trees)]), max(trees)
        M = int(off[-1])
        sees = [A.ancestors([max(t - int(rng.integers(1, 4)), 0) if t else -1 for t in range(n)]) for n in trees]
        mask = torch.from_numpy(A.pack(sees, M, most)).cuda()
        batch = dict(tree_off=i32(off), tree_mask=mask, max_tree=most)
        qkv = ready(sees, off, mask, most)
        kc, vc = dense()
        for l in range(L):
            q, kt, vt = qkv[l, :, :H], qkv[l, :, H:H + Hk], qkv[l, :, H + Hk:]
            o, lse = mb.moespec_tree_attention(desc, q, kt, vt, kc[l], vc[l], cache_len, max_len=max(lens), **batch)
            check = Batch.__new__(Batch)
            check.dtype, check.D, check.lens, check.trees, check.off = dtype, D, lens, trees, off
            check.check(o, lse, A.attention(f64(q), f64(kt), f64(vt), f64(kc[l]), f64(vc[l]), lens, off, sees, scale))
        logits = randn(M, vocab, scale=1.5)
        tokens = rng.integers(0, vocab, M)
        for s, see in enumerate(sees):
            for t in range(1, trees[s]):
                logits[int(off[s]) + max(np.flatnonzero(see[t, :t])), int(tokens[off[s] + t])] = 8.0
        u, w = rng.random(M), rng.random(S)
        got = mb.moespec_draft_verify(mb.VerifyDesc(vocab, CODE[dtype]), logits, i32(tokens), torch.from_numpy(u).cuda(),
                                      torch.from_numpy(w).cuda(), 6, **batch)
        paths = []
        for s in range(S):
            at = slice(off[s], off[s + 1])
            path, token = V.verify(f64(logits)[at], tokens[at], sees[s], u[at], w[s], 6)
            assert got["path"][s].tolist()[:len(path)] == path and int(got["n_path"][s]) == len(path) and int(got["next_token"][s]) == token
            paths.append(path)
        # weights of the verified rows: what the rejected ones attended to has no part
        cw, _ = mb.moespec_cache_weights(desc, q, kt, kc[L - 1], cache_len, lse, row_weight=got["accepted"], max_len=max(lens), **batch)
        want, _, size, _ = A.weights(f64(q), f64(kt), f64(kc[L - 1]), lens, off, sees, scale, f64(lse), f64(got["accepted"]))
        for s, n in enumerate(lens):
            assert np.all(np.abs(f64(cw[s, :, :n]) - want[s, :, :n]) <= 2.0 ** -14 * size[s, :, :n] + 1e-30)
        cache_len = mb.moespec_paged_write(desc, cache, qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:], cache_len, path=got["path"],
                                           n_path=got["n_path"], tree_off=batch["tree_off"], max_tree=most)
        append(qkv, off, paths)
        lens = [n + len(p) for n, p in zip(lens, paths)]
        assert cache_len.tolist() == lens
        dense()


def test_a_step_of_single_tokens_as_a_graph():
    """Rotation in place, write, attention captured once and replayed over growing lengths, against the same calls one by one; other work runs
    between the replays."""
    H, Hk, D, S, page = 8, 2, 128, 3, 32
    rng, gen = np.random.default_rng(4), torch.Generator(device="cuda").manual_seed(4)
    rows, n = table([400] * S, page, rng)
    desc = mb.AttnDesc(H, Hk, D, 1, mb.BF16)
    freq = torch.tensor([1e4 ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float32, device="cuda")
    pools = []
    for _ in range(2):
        cache = mb.alloc_paged_cache(desc, mb.CACHE_I8, n, page, torch.from_numpy(rows).cuda())
        for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale):
            t.zero_()
        lens, new = i32([0, 63, 300]), i32([0, 0, 0])
        qkv = torch.zeros((S, H + 2 * Hk, D), dtype=torch.bfloat16, device="cuda")
        out, lse = torch.zeros((S, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((S, H), device="cuda")
        ws = mb.alloc_paged_attention_workspace(desc, cache, S, 400)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        off = i32(np.arange(S + 1))
        calls = [mb.HeadRopeCall(desc, q, k, q, k, freq, norm=True, eps=1e-6, cache_len=lens, tree_off=off, max_tree=1),
                 mb.PagedWriteCall(desc, cache, k[None], v[None], lens, new_len=new, tree_off=off, max_tree=1),
                 mb.PagedAttentionCall(desc, cache, q, new, ws, out, lse, 400)]
        pools.append((calls, qkv, lens, new, out, lse, cache))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c in pools[1][0]:
            c()
        for t in pools[1][6].tensors():
            if t.dtype != torch.int32:
                t.zero_()
        with torch.cuda.graph(graph, stream=stream):
            for c in pools[1][0]:
                c()
        for step in range(40):
            x = (torch.randn((S, H + 2 * Hk, D), generator=gen, device="cuda") * 2).to(torch.bfloat16)
            for _, qkv, _, _, out, _, _ in pools:
                qkv.copy_(x), out.fill_(9)
            for c in pools[0][0]:
                c()
            graph.replay()
            stream.synchronize()
            for a, b in zip(pools[0][3:6], pools[1][3:6]):
                assert torch.equal(a, b), step
            for p in pools:
                p[2].copy_(p[3])
    assert pools[0][2].tolist() == [40, 103, 340]


def test_calls_on_two_streams_match_serial_runs():
    pools = [Pool("bf16", "i8", 4, 128, [700, 90], 32, seed=s, H=16).poison() for s in (1, 2)]
    qs = [torch.randn((2, 16, 128), device="cuda").to(torch.bfloat16) for _ in pools]
    ref = [mb.moespec_paged_attention(p.desc, p.cache, q, p.cache_len, max_len=700) for p, q in zip(pools, qs)]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in pools], []
    for _ in range(20):
        outs.append([mb.moespec_paged_attention(p.desc, p.cache, q, p.cache_len, max_len=700, stream=s)
                     for p, q, s in zip(pools, qs, streams)])
    torch.cuda.synchronize()
    for pair in outs:
        for got, want in zip(pair, ref):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_tensors_of_another_type_shape_or_layout_are_refused():
    p = Pool("bf16", "i8", 2, 64, [40, 7], 16, H=4)
    d, c = p.desc, p.cache
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    ws, out = mb.alloc_paged_attention_workspace(d, c, 2, 40), torch.zeros_like(q)

    def refused(match, **kw):
        a = dict(desc=d, cache=c, q=q, cache_len=p.cache_len, ws=ws, out=out, max_len=40, **kw.pop("more", {}))
        a.update(kw)
        with pytest.raises(ValueError, match=match):
            mb.PagedAttentionCall(**a)
    refused("q must have dtype", q=q.float())
    refused("q must have shape", q=q[:, :3])
    refused("cache_len must have dtype", cache_len=p.cache_len.long())
    refused("cache_len must have shape", cache_len=p.cache_len[:1])
    refused("out must be contiguous", out=torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")[:, ::2])
    refused("layer must be in", layer=1)
    for field, value in (("k_pages", c.k_pages.float()), ("k_pages", c.k_pages[:, :3]), ("v_scale", None), ("v_scale", c.v_scale.double()),
                         ("page_table", c.page_table.long()), ("page_table", c.page_table[:1]), ("code", 7), ("code", mb.CACHE_E4M3)):
        bad = mb.PagedCache(**{**dict(code=c.code, k_pages=c.k_pages, v_pages=c.v_pages, page_table=c.page_table, k_scale=c.k_scale,
                                      v_scale=c.v_scale), field: value})
        with pytest.raises((ValueError, mb.MoeSpecError)):
            mb.PagedAttentionCall(d, bad, q, p.cache_len, ws, out, max_len=40)()
    with pytest.raises(mb.MoeSpecError):
        mb.moespec_paged_attention(d, c, q, p.cache_len, max_len=c.max_entries + 1)
    with pytest.raises(mb.MoeSpecError):
        mb.PagedAttentionCall(d, c, q, p.cache_len, ws, q, max_len=40)()
    kt = torch.zeros((1, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="k_tree must have shape"):
        mb.moespec_paged_write(d, c, kt.expand(2, 5, 2, 64), kt, i32([0]))
    with pytest.raises(mb.MoeSpecError):
        mb.moespec_paged_write(d, c, kt, kt, p.cache_len, path=i32([[0], [0]]), tree_off=i32([0, 2, 5]))
    v = mb.VerifyDesc(50, mb.F32)
    logits, u, w = torch.zeros((4, 60), device="cuda"), torch.zeros(4, device="cuda", dtype=torch.float64), torch.zeros(1, device="cuda").double()
    with pytest.raises(ValueError, match="logits must be"):
        mb.moespec_draft_verify(v, logits, i32([0] * 4), u, w, 4)
    with pytest.raises(ValueError, match="lie in a row"):
        mb.moespec_draft_verify(v, torch.zeros((4, 100), device="cuda")[:, ::2], i32([0] * 4), u, w, 4)
    with pytest.raises(ValueError, match="u_accept must have dtype"):
        mb.moespec_draft_verify(v, logits[:, :50], i32([0] * 4), u.float(), w, 4)
    with pytest.raises(mb.MoeSpecError):  # sampled drafts in a tree
        mb.moespec_draft_verify(v, logits[:, :50], i32([0] * 4), u, w, 4, draft_logits=logits[:, 10:].contiguous(), tree_mask=i32([[1]] * 4))
