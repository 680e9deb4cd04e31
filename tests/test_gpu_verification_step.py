"""A verification loop as a program runs it: per layer the norm, the tree attention over the cache, the norm between the blocks and the
budgeted MoE layer; then the accepted path is committed to the caches of all layers with the weights that its keys received, and
caches above their budget are cut.  Every call is checked against the oracle on the inputs it had, the caches against a copy
that is kept by hand."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import moespec_oracle as O
from paper_2602_16052_amd import binding as mb
from paper_2602_16052_amd import workloads as wl

from attention_common import CODE, HALF_STEP, TORCH, Batch, f64, i32, random_tree
from gpu_common import assert_out_close, oracle_weights, out_to_numpy, upload_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,Hk,D", [("bf16", 4, 2, 64), ("f32", 2, 1, 96)])
def test_steps_of_a_verification_loop(dtype, H, Hk, D):
    S, L, cap, budget, recent, steps, d = 2, 2, 96, 40, 6, 4, 128
    rng = np.random.default_rng(7)
    gen = torch.Generator(device="cuda").manual_seed(7)
    dt = TORCH[dtype]
    randn = lambda *s, scale=1.0: (torch.randn(s, generator=gen, device="cuda") * scale).to(dt)  # noqa: E731
    cfg = wl.small_config("step", dtype, d=d, n_experts=8, top_k=2, d_ff=64, M=64, budgets=(4,))
    W = [wl.layer_weights(cfg, layer=l) for l in range(L)]
    W_d = [upload_weights(w) for w in W]
    moe = mb.LayerDesc(d, 8, 2, 64, CODE[dtype], cfg.renorm)
    att = mb.AttnDesc(H, Hk, D, cap, CODE[dtype])
    w_qkv = [randn(d, (H + 2 * Hk) * D, scale=0.15) for _ in range(L)]
    w_out = [randn(H * D, d, scale=0.1) for _ in range(L)]
    w_norm = [(1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2 * L + 1)]
    # the caches after a prompt, in two places each: eviction goes from the one to the other
    lens = [37, 12]
    kc, vc = randn(L, S, Hk, cap, D), randn(L, S, Hk, cap, D)
    cw = torch.rand((L, S, Hk, cap), generator=gen, device="cuda")
    hand = [[[(kc[l, s, h, :lens[s]].clone(), vc[l, s, h, :lens[s]].clone()) for h in range(Hk)] for s in range(S)] for l in range(L)]
    cache_len = i32(lens)
    evictions = 0
    for step in range(steps):
        trees = [int(rng.integers(5, 17)), int(rng.integers(1, 9))]
        off = np.concatenate([[0], np.cumsum(trees)])
        M, top = int(off[-1]), max(trees)
        sees = [random_tree(rng, n) for n in trees]
        mask = torch.from_numpy(A.pack(sees, M, top)).cuda()
        batch = dict(tree_off=i32(off), tree_mask=mask, max_tree=top, max_len=cap)
        qkv = torch.empty((L, M, H + 2 * Hk, D), dtype=dt, device="cuda")
        tree_w = torch.empty((L, M, Hk), device="cuda")
        lse = torch.empty((L, M, H), device="cuda")
        h = randn(M, d)
        x = mb.moespec_block_norm(moe, h, w_pre=w_norm[0], eps=1e-6)[1]
        for l in range(L):
            qkv[l] = (x @ w_qkv[l]).view(M, H + 2 * Hk, D)
            q, kt, vt = qkv[l, :, :H], qkv[l, :, H:H + Hk], qkv[l, :, H + Hk:]
            o, _ = mb.moespec_tree_attention(att, q, kt, vt, kc[l], vc[l], cache_len, lse=lse[l], **batch)
            check = Batch.__new__(Batch)
            check.dtype, check.D, check.lens, check.trees, check.off = dtype, D, lens, trees, off
            check.check(o, lse[l], A.attention(f64(q), f64(kt), f64(vt), f64(kc[l]), f64(vc[l]), lens, off, sees,
                                               float(np.float32(D ** -0.5))))
            y = o.view(M, H * D) @ w_out[l]
            r, x2 = mb.moespec_block_norm(moe, y, h, post_norm=True, scale=0.5, w_pre=w_norm[2 * l + 1], eps=1e-6)
            wr, _, z = A.block_norm(f64(y), f64(h), True, None, None, False, 0.5, f64(w_norm[2 * l + 1]), 1e-6)
            tol = HALF_STEP[dtype] * np.abs(wr) * (1 + 2.0 ** -6) + 40 * 2.0 ** -24 * (z + np.abs(wr))
            assert np.all(np.abs(f64(r) - wr) <= tol)
            ws = mb.alloc_workspace(moe, M)
            y2 = mb.moespec_layer_forward(moe, W_d[l], x2, 4, mb.SUBSTITUTE, ws)
            ref = O.layer_forward(x2.float().cpu().numpy(), oracle_weights(W[l]), 2, cfg.renorm, 4, O.SUBSTITUTE)
            assert_out_close(out_to_numpy(y2), ref["out"], dtype, scale_aware=True)
            h, x = mb.moespec_block_norm(moe, y2, r, w_pre=w_norm[2 * l + 2], eps=1e-6)
        # acceptance: a path from a root of every tree downwards
        paths = []
        for s, m in enumerate(sees):
            leaf = int(rng.integers(trees[s]))
            paths.append([int(j) for j in np.flatnonzero(m[leaf])][:6])
        path = np.zeros((S, 6), dtype=np.int32)
        accepted = np.zeros(M, dtype=np.float32)
        for s, p in enumerate(paths):
            path[s, :len(p)] = p
            accepted[off[s] + np.array(p)] = 1.0
        rw = torch.from_numpy(accepted).cuda()
        for l in range(L):
            q, kt = qkv[l, :, :H], qkv[l, :, H:H + Hk]
            before = cw[l].clone()
            mb.moespec_cache_weights(att, q, kt, kc[l], cache_len, lse[l], cache_w=cw[l], tree_w=tree_w[l], cache_w_in=cw[l],
                                     decay=0.9, row_weight=rw, **batch)
            want, tw, acw, atw = A.weights(f64(q), f64(kt), f64(kc[l]), lens, off, sees, float(np.float32(D ** -0.5)),
                                           f64(lse[l]), accepted.astype(np.float64), f64(before), float(np.float32(0.9)))
            for s, n in enumerate(lens):  # scores of a few units: 2^-14 is far above what fp32 leaves, far below an error of indexing
                assert np.all(np.abs(f64(cw[l, s, :, :n]) - want[s, :, :n]) <= 2.0 ** -14 * acw[s, :, :n])
            assert np.all(np.abs(f64(tree_w[l]) - tw) <= 2.0 ** -14 * atw + 1e-30)
        new_len = mb.moespec_cache_commit(att, qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:], i32(path), i32([len(p) for p in paths]), kc, vc,
                                          cache_len, tree_w=tree_w, cache_w=cw, tree_off=batch["tree_off"], max_tree=top,
                                          n_layers=L)
        for l in range(L):
            for s, p in enumerate(paths):
                rows = torch.tensor([int(off[s]) + j for j in p], device="cuda")
                for g in range(Hk):
                    k, v = hand[l][s][g]
                    hand[l][s][g] = (torch.cat([k, qkv[l, rows, H + g]]), torch.cat([v, qkv[l, rows, H + Hk + g]]))
                    assert torch.equal(cw[l, s, g, lens[s]:lens[s] + len(p)], tree_w[l, rows, g])
        lens = [n + len(p) for n, p in zip(lens, paths)]
        assert new_len.tolist() == lens
        cache_len = new_len
        if max(lens) > budget:
            evictions += 1
            small = mb.moespec_cache_evict(att, kc, vc, cw, cache_len, budget, recent, n_layers=L)
            for l in range(L):
                for s, n in enumerate(lens):
                    for g in range(Hk):
                        keep = A.kept_entries(cw[l, s, g].cpu().numpy(), n, budget, recent)
                        at = torch.from_numpy(keep).cuda()
                        hand[l][s][g] = tuple(t[at] for t in hand[l][s][g])
            lens = [min(n, budget) for n in lens]
            assert small["new_len"].tolist() == lens
            kc[..., :budget, :], vc[..., :budget, :], cw[..., :budget] = small["k"], small["v"], small["w"]
            cache_len = small["new_len"]
        for l in range(L):
            for s, n in enumerate(lens):
                for g in range(Hk):
                    assert torch.equal(kc[l, s, g, :n], hand[l][s][g][0]) and torch.equal(vc[l, s, g, :n], hand[l][s][g][1])
    assert evictions >= 2
