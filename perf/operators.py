"""The operators around the budgeted MoE layer of a verification step whose speed is tracked: the other half of a transformer
layer that verifies a draft tree, over a cache of keys and values that is itself held to a budget.

  attention  tree attention (TreeAttentionCall): every drafted token sees the cache and its ancestors in the tree
  weights    attention weight that every cached key received, summed over tokens and heads (CacheWeightsCall)
  commit     keys and values of the accepted path appended to the cache of every layer (CacheCommitCall)
  evict      cache cut to its budget: the latest entries and those with the most weight (CacheEvictCall)
  norm       residual + scale * gate * norm(block output), and the next block's normed input (BlockNormCall)

Keys and queries are N(0, 1) with queries scaled to give scores a standard deviation of 2; trees are random (every token's
parent is one of the 8 tokens in front of it); accumulated weights are log-normal with a share of exact zeros.
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


# ---- the cases

def _attention(name, dtype, n_seq, tree, heads, kv_heads, head_dim, length, masked, ragged=False, fused=False, op="attention"):
    return dict(name=name, op=op, dtype=dtype, n_seq=n_seq, tree=tree, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                length=length, masked=masked, ragged=ragged, fused=fused)


def listed():
    return [
        # one token over a short cache: what an undrafted decoding step asks, all latency
        _attention("attn_token", "bf16", 1, 1, 32, 4, 128, 1021, False),
        # sixteen requests at once, trees of up to 31 tokens, long caches of different lengths, q, k, v out of one projection
        _attention("attn_tree_batch", "bf16", 16, 31, 32, 8, 128, 16381, True, ragged=True, fused=True),
        # the largest tree over the longest cache: bound by arithmetic
        _attention("attn_tree_long", "bf16", 1, 511, 32, 4, 128, 65521, True),
        # a small model verified at full precision
        _attention("attn_f32", "f32", 2, 63, 8, 8, 64, 2039, True, ragged=True),
        # the benchmark's tree, hidden size 2048 as 16 heads
        _attention("weights_tree63", "bf16", 1, 63, 16, 16, 128, 4093, True, op="weights"),
        # four requests, wide trees, long caches
        _attention("weights_batch", "bf16", 4, 127, 32, 4, 128, 32749, True, ragged=True, fused=True, op="weights"),
        # one layer of a small fp32 model, four tokens accepted
        dict(name="commit_f32", op="commit", dtype="f32", n_layers=1, n_seq=1, tree=15, path=4, kv_heads=8, head_dim=64,
             length=500),
        # a whole model at the end of a step: 48 layers, eight requests, up to eight tokens accepted
        dict(name="commit_layers", op="commit", dtype="bf16", n_layers=48, n_seq=8, tree=63, path=8, kv_heads=4,
             head_dim=128, length=1009),
        # one layer, half of the cache goes
        dict(name="evict_layer", op="evict", dtype="bf16", n_layers=1, n_seq=1, kv_heads=16, head_dim=128, length=4093,
             budget=2048, recent=64),
        # four layers of four requests, long prompts cut to an eighth
        dict(name="evict_long", op="evict", dtype="bf16", n_layers=4, n_seq=4, kv_heads=8, head_dim=128, length=32749,
             budget=4096, recent=256),
        # one token
        dict(name="norm_token", op="norm", dtype="bf16", tokens=1, d=2048, gate="token", sigmoid=True, post=True),
        # four trees of 511 tokens, a gate for every element
        dict(name="norm_trees", op="norm", dtype="bf16", tokens=2044, d=4096, gate="element", sigmoid=False, post=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "weights", "commit", "evict", "norm"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    while True:
        if op in ("attention", "weights"):
            heads, kv_heads = rng.choice([(32, 4), (32, 8), (16, 16), (8, 8), (12, 2), (20, 4), (7, 1), (64, 8)])
            c = dict(op=op, dtype=dtype, n_seq=_log(rng, 1, 16), tree=_log(rng, 1, 511), heads=heads, kv_heads=kv_heads,
                     head_dim=rng.choice([64, 96, 128, 128, 192, 256]), length=_log(rng, 30, 65536),
                     masked=rng.random() < 0.8, ragged=rng.random() < 0.5, fused=rng.random() < 0.5)
            cells = c["n_seq"] * c["tree"] * heads * c["length"]
            kept = c["n_seq"] * kv_heads * c["length"] * c["head_dim"]
            if cells * c["head_dim"] <= (1.3e11 if dtype == "bf16" else 2e10) and kept <= (1 << 27):
                return c
        elif op == "commit":
            c = dict(op=op, dtype=dtype, n_layers=_log(rng, 1, 48), n_seq=_log(rng, 1, 8), tree=_log(rng, 1, 255),
                     path=_log(rng, 1, 12), kv_heads=rng.choice([1, 2, 4, 8]), head_dim=rng.choice([64, 96, 128, 256]),
                     length=_log(rng, 16, 1000))
            if c["n_layers"] * c["n_seq"] * c["kv_heads"] * c["length"] * c["head_dim"] <= (1 << 27):
                return c
        elif op == "evict":
            length = _log(rng, 64, 65536)
            budget = max(8, int(length * rng.uniform(0.05, 0.9)))
            c = dict(op=op, dtype=dtype, n_layers=_log(rng, 1, 8), n_seq=_log(rng, 1, 4), kv_heads=rng.choice([1, 4, 8, 16]),
                     head_dim=rng.choice([64, 96, 128, 256]), length=length, budget=budget,
                     recent=int(budget * rng.uniform(0.0, 0.5)))
            if c["n_layers"] * c["n_seq"] * c["kv_heads"] * length * c["head_dim"] <= (1 << 27):
                return c
        else:
            return dict(op=op, dtype=dtype, tokens=_log(rng, 1, 2000), d=32 * _log(rng, 4, 128), sigmoid=rng.random() < 0.5,
                        gate=rng.choice(["none", "channel", "token", "element"]), post=rng.random() < 0.7)


def _of_sequences(c, most):
    """Sizes of the sequences of a batch: all alike, or falling to half of the first one's."""
    n = c["n_seq"]
    return [max(1, most - (s * most) // (2 * n)) if c.get("ragged") else most for s in range(n)]


def work(c):
    b = _BYTES[c["dtype"]]
    if c["op"] in ("attention", "weights"):
        trees, lens = _of_sequences(c, c["tree"]), _of_sequences(c, c["length"])
        H, Hk, D, M = c["heads"], c["kv_heads"], c["head_dim"], sum(trees)
        seen = sum(t * n for t, n in zip(trees, lens)) + M  # every token also sees itself at least
        keys, q = (sum(lens) + M) * Hk * D * b, M * H * D * b
        mask = 4 * M * ((c["tree"] + 31) // 32) if c["masked"] else 0
        if c["op"] == "attention":
            return {"bytes": 2 * keys + 2 * q + 4 * M * H + mask, "flops": 4 * D * H * seen}
        return {"bytes": keys + q + 4 * M * H + 4 * (2 * sum(lens) + M) * Hk + 4 * M + mask, "flops": 2 * D * H * seen}
    if c["op"] == "commit":
        rows = c["n_layers"] * sum(_accepted(c)) * c["kv_heads"]
        return {"bytes": rows * (4 * c["head_dim"] * b + 8), "flops": 0}
    if c["op"] == "evict":
        heads = c["n_layers"] * c["n_seq"] * c["kv_heads"]
        kept = min(c["length"], c["budget"])
        return {"bytes": heads * (4 * c["length"] + kept * (4 * c["head_dim"] * b + 8)), "flops": 0}
    per = {"none": 0, "channel": c["d"], "token": c["tokens"], "element": c["tokens"] * c["d"]}[c["gate"]]
    return {"bytes": (4 * c["tokens"] * c["d"] + per + 2 * c["d"]) * b, "flops": 8 * c["tokens"] * c["d"]}


def _accepted(c):
    """Length of the accepted path of every sequence: 1 .. path."""
    return [1 + (5 * s + c["path"] - 1) % c["path"] for s in range(c["n_seq"])]


# ---- inputs

def _tree_words(sizes, most, gen):
    """Packed ancestor sets [M, ceil(most / 32)] of random trees: bit j of a token's row is set if it sees token j."""
    rows = []
    for n in sizes:
        back = torch.randint(1, 9, (n,), generator=gen).tolist()
        seen = [0] * n
        for t in range(n):
            seen[t] = (seen[t - back[t]] if t >= back[t] else 0) | (1 << t)
        rows += seen
    words = [[(r >> (32 * w)) & 0xFFFFFFFF for w in range((most + 31) // 32)] for r in rows]
    return torch.tensor(words, dtype=torch.int64).to(torch.int32)


def _randn(shape, dtype, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def prepare(c, seed):
    dev, host = torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    dt = _TORCH[c["dtype"]]
    on = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    s = dict(op=c["op"], case=c)
    if c["op"] in ("attention", "weights"):
        H, Hk, D, S = c["heads"], c["kv_heads"], c["head_dim"], c["n_seq"]
        trees, lens = _of_sequences(c, c["tree"]), _of_sequences(c, c["length"])
        M, cap = sum(trees), c["length"] + 11
        if c["fused"]:  # q, k and v of a token lie in one row, as one projection leaves them
            qkv = _randn((M, H + 2 * Hk, D), dt, dev)
            qkv[:, :H] *= 2.0
            s["q"], s["k_tree"], s["v_tree"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:
            s["q"], s["k_tree"], s["v_tree"] = (_randn((M, H, D), dt, dev, 2.0), _randn((M, Hk, D), dt, dev),
                                                _randn((M, Hk, D), dt, dev))
        s["k_cache"] = _randn((S, Hk, cap, D), dt, dev)
        s["v_cache"] = _randn((S, Hk, cap, D), dt, dev)
        s["tree_off"] = on([sum(trees[:i]) for i in range(S + 1)])
        s["cache_len"], s["max_tree"], s["max_len"] = on(lens), c["tree"], c["length"]
        s["tree_mask"] = _tree_words(trees, c["tree"], host).cuda() if c["masked"] else None
        if c["op"] == "attention":
            s["out"] = torch.zeros((M, H, D), dtype=dt, device="cuda")
            s["lse"] = torch.zeros((M, H), dtype=torch.float32, device="cuda")
        else:
            s["lse"] = _plain_attention(s, want_out=False)["lse"]
            s["row_weight"] = torch.rand((M,), generator=dev, device="cuda")
            s["decay"] = 0.875
            s["cache_w"] = torch.rand((S, Hk, cap), generator=dev, device="cuda")
            s["cache_w_out"] = torch.zeros((S, Hk, cap), device="cuda")
            s["tree_w"] = torch.zeros((M, Hk), device="cuda")
        return s
    if c["op"] in ("commit", "evict"):
        Hk, D, S, L, cap = c["kv_heads"], c["head_dim"], c["n_seq"], c["n_layers"], c["length"] + 23
        s["k_cache"] = _randn((L, S, Hk, cap, D), dt, dev)
        s["v_cache"] = _randn((L, S, Hk, cap, D), dt, dev)
        s["cache_w"] = torch.randn((L, S, Hk, cap), generator=dev, device="cuda").mul_(2.0).exp_()
        s["cache_w"] *= torch.rand((L, S, Hk, cap), generator=dev, device="cuda") > 0.1
        s["cache_len"] = on([max(1, c["length"] - 7 * i) for i in range(S)])
        s["new_len"] = torch.zeros(S, dtype=torch.int32, device="cuda")
    if c["op"] == "commit":
        T, n = c["tree"], _accepted(c)
        s["k_tree"], s["v_tree"] = _randn((L, S * T, Hk, D), dt, dev), _randn((L, S * T, Hk, D), dt, dev)
        s["tree_w"] = torch.rand((L, S * T, Hk), generator=dev, device="cuda")
        s["tree_off"], s["max_tree"] = on([T * i for i in range(S + 1)]), T
        s["path"] = torch.randint(0, T, (S, c["path"]), generator=host).sort(dim=1).values.to(torch.int32).cuda()
        s["n_path"] = on(n)
    elif c["op"] == "evict":
        B = c["budget"]
        s["budget"], s["recent"] = B, c["recent"]
        s["k_out"], s["v_out"] = (torch.zeros((L, S, Hk, B + 64, D), dtype=dt, device="cuda") for _ in range(2))
        s["w_out"] = torch.zeros((L, S, Hk, B + 64), device="cuda")
        s["kept"] = torch.zeros((L, S, Hk, B), dtype=torch.int32, device="cuda")
    elif c["op"] == "norm":
        M, d = c["tokens"], c["d"]
        shape = {"none": None, "channel": (d,), "token": (M,), "element": (M, d)}[c["gate"]]
        s["y"], s["residual"] = _randn((M, d), dt, dev, 0.5), _randn((M, d), dt, dev, 3.0)
        s["gate"] = None if shape is None else _randn(shape, dt, dev)
        s["w_post"] = (1.0 + _randn((d,), torch.float32, dev, 0.1)).to(dt) if c["post"] else None
        s["w_pre"] = (1.0 + _randn((d,), torch.float32, dev, 0.1)).to(dt)
        s["scale"], s["eps"] = 0.7, 1e-6
        s["r"], s["x"] = (torch.zeros((M, d), dtype=dt, device="cuda") for _ in range(2))
    return s


# ---- the plain forms

def _visible(s, n_keys):
    """[S, T, n_keys + T] truth values: the cached keys of the sequence, then the tokens of its tree."""
    S, T = s["cache_len"].numel(), s["max_tree"]
    at = torch.arange(T, device="cuda")
    sizes = s["tree_off"][1:] - s["tree_off"][:-1]
    cached = torch.arange(n_keys, device="cuda") < s["cache_len"][:, None, None]
    if s["tree_mask"] is None:
        tree = (at[None, :] <= at[:, None]).expand(S, T, T)
    else:
        words = s["tree_mask"][_token_rows(s)]  # [S, T, W]
        tree = ((words[..., None] >> torch.arange(32, device="cuda")) & 1).flatten(2)[..., :T] != 0
    tree = tree & (at < sizes[:, None, None])
    return torch.cat([cached.expand(S, T, n_keys), tree], dim=2)


def _token_rows(s):
    """[S, T] row of every token of every tree; rows past a tree's end repeat the last one."""
    T = torch.arange(s["max_tree"], device="cuda")
    return torch.minimum(s["tree_off"][:-1, None] + T, s["tree_off"][1:, None] - 1).long()


def _plain_scores(s):
    """Scores [S, Hk, T, G, keys] in 32 bits, -inf where a token does not see a key."""
    rows, n = _token_rows(s), s["max_len"]
    S, T = rows.shape
    Hk, D = s["k_cache"].shape[1], s["k_cache"].shape[3]
    q = s["q"][rows].float().reshape(S, T, Hk, -1, D).permute(0, 2, 1, 3, 4).reshape(S, Hk, -1, D)
    k = torch.cat([s["k_cache"][:, :, :n].float(), s["k_tree"][rows].float().transpose(1, 2)], dim=2)
    a = (q @ k.transpose(2, 3)).mul_(D ** -0.5).reshape(S, Hk, T, -1, n + T)
    return a.masked_fill_(~_visible(s, n)[:, None, :, None], -math.inf)


def _to_rows(s, v):
    """[S, Hk, T, G, ...] of the trees -> [M, H, ...]."""
    S, Hk, T, G = v.shape[:4]
    M = s["q"].shape[0]
    v = v.transpose(1, 2).reshape(S, T, Hk * G, *v.shape[4:])
    at = torch.arange(M, device="cuda")
    seq = (at[:, None] >= s["tree_off"][None, 1:]).sum(dim=1)
    return v[seq, at - s["tree_off"][seq]]


def _plain_attention(s, want_out=True):
    a = _plain_scores(s)
    top = a.amax(dim=4, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = a.sub_(top).exp_()
    total = p.sum(dim=4, keepdim=True)
    res = dict(lse=_to_rows(s, (top + total.log())[..., 0]))
    if want_out:
        S, Hk, T, G, n = p.shape
        v = torch.cat([s["v_cache"][:, :, :s["max_len"]].float(), s["v_tree"][_token_rows(s)].float().transpose(1, 2)], dim=2)
        o = (p.reshape(S, Hk, T * G, n) @ v).reshape(S, Hk, T, G, -1) / torch.where(total == 0, 1.0, total)
        res["out"] = _to_rows(s, o).to(s["q"].dtype)
    return res


def _plain_weights(s):
    rows, n = _token_rows(s), s["max_len"]
    S, T = rows.shape
    a = _plain_scores(s)
    Hk, G = a.shape[1], a.shape[3]
    inside = (torch.arange(T, device="cuda") < (s["tree_off"][1:] - s["tree_off"][:-1])[:, None]).float()
    lse = s["lse"][rows].reshape(S, T, Hk, G).permute(0, 2, 1, 3)
    p = a.sub_(lse[..., None]).exp_().mul_((s["row_weight"][rows] * inside)[:, None, :, None, None])
    w = p.sum(dim=(2, 3))
    used = torch.arange(n, device="cuda") < s["cache_len"][:, None, None]
    s["cache_w_out"][:, :, :n] = torch.where(used, s["decay"] * s["cache_w"][:, :, :n] + w[..., :n], s["cache_w_out"][:, :, :n])
    return dict(cache_w=s["cache_w_out"], tree_w=_tree_columns(s, w[..., n:]))


def _tree_columns(s, w):
    """[S, Hk, T] of the trees' own keys -> [M, Hk]."""
    M = s["q"].shape[0]
    at = torch.arange(M, device="cuda")
    seq = (at[:, None] >= s["tree_off"][None, 1:]).sum(dim=1)
    return w[seq, :, at - s["tree_off"][seq]]


def _plain_commit(s):
    S, P = s["path"].shape
    seq, at = torch.arange(S, device="cuda")[:, None], torch.arange(P, device="cuda")
    src, dst = s["tree_off"][:-1, None] + s["path"], s["cache_len"][:, None] + at
    taken = (at < s["n_path"][:, None])
    for cache, tree in ((s["k_cache"], s["k_tree"]), (s["v_cache"], s["v_tree"]), (s["cache_w"], s["tree_w"])):
        new = tree[:, src].movedim(0, 2)  # [S, P, layers, Hk, ...], as the indexing of the cache gives it
        old = cache[:, seq, :, dst]
        cache[:, seq, :, dst] = torch.where(taken.reshape(S, P, *[1] * (new.dim() - 2)), new, old)
    torch.add(s["cache_len"], s["n_path"], out=s["new_len"])
    return dict(k=s["k_cache"], v=s["v_cache"], w=s["cache_w"], new_len=s["new_len"])


def _plain_evict(s):
    B, cap, D = s["budget"], s["cache_w"].shape[3], s["k_cache"].shape[4]
    n = s["cache_len"][None, :, None, None]
    at = torch.arange(cap, device="cuda")
    rank = torch.where(at >= n - s["recent"], math.inf, s["cache_w"])
    rank = torch.where(at >= n, -math.inf, rank)
    order = rank.sort(dim=3, descending=True, stable=True).indices[..., :B]
    inside = torch.arange(B, device="cuda") < torch.clamp(n, max=B)
    order = torch.where(inside, order, cap).sort(dim=3).values
    safe = order.clamp(max=cap - 1)
    rows = safe[..., None].expand(*safe.shape, D)
    for out, cache in ((s["k_out"], s["k_cache"]), (s["v_out"], s["v_cache"])):
        out[..., :B, :] = torch.where(inside[..., None], cache.gather(3, rows), out[..., :B, :])
    s["w_out"][..., :B] = torch.where(inside, s["cache_w"].gather(3, safe), s["w_out"][..., :B])
    s["kept"].copy_(torch.where(inside, order, -1))
    torch.clamp(s["cache_len"], max=B, out=s["new_len"])
    return dict(k=s["k_out"], v=s["v_out"], w=s["w_out"], kept=s["kept"], new_len=s["new_len"])


def _plain_norm(s):
    y = s["y"].float()
    if s["w_post"] is not None:
        y = y * torch.rsqrt((y * y).mean(dim=1, keepdim=True) + s["eps"]) * s["w_post"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        g = 1.0 / (1.0 + torch.exp(-g)) if s["case"]["sigmoid"] else g
        y = y * (g[:, None] if s["case"]["gate"] == "token" else g)
    r = s["residual"].float() + s["scale"] * y
    x = r * torch.rsqrt((r * r).mean(dim=1, keepdim=True) + s["eps"]) * s["w_pre"].float()
    return dict(r=r.to(s["y"].dtype), x=x.to(s["y"].dtype))


_PLAIN = dict(attention=_plain_attention, weights=_plain_weights, commit=_plain_commit, evict=_plain_evict, norm=_plain_norm)


# ---- the framework's calls

def _call(s):
    """The call object that a program keeps next to its buffers (arguments marshalled once), and the outputs."""
    from paper_2602_16052_amd import binding as mb

    c = s["case"]
    code = mb.BF16 if c["dtype"] == "bf16" else mb.F32
    if c["op"] == "norm":
        d = mb.LayerDesc(c["d"], 1, 1, c["d"], code, False)
        kind = dict(none=mb.BLOCK_GATE_NONE, channel=mb.BLOCK_GATE_CHANNEL, token=mb.BLOCK_GATE_TOKEN,
                    element=mb.BLOCK_GATE_ELEMENT)[c["gate"]]
        return (mb.BlockNormCall(d, s["y"], s["residual"], s["r"], s["x"], post_norm=c["post"], w_post=s["w_post"],
                                 gate=s["gate"], gate_kind=kind, gate_sigmoid=c["sigmoid"], scale=s["scale"],
                                 w_pre=s["w_pre"], eps=s["eps"]), dict(r=s["r"], x=s["x"]))
    heads = c.get("heads", c["kv_heads"])
    d = mb.AttnDesc(heads, c["kv_heads"], c["head_dim"], s["k_cache"].shape[-2], code)
    if c["op"] == "attention":
        ws = mb.alloc_attn_workspace(d, c["n_seq"], s["q"].shape[0], s["max_tree"], s["max_len"])
        return (mb.TreeAttentionCall(d, s["q"], s["k_tree"], s["v_tree"], s["k_cache"], s["v_cache"], s["cache_len"], ws,
                                     s["out"], lse=s["lse"], tree_off=s["tree_off"], tree_mask=s["tree_mask"],
                                     max_tree=s["max_tree"], max_len=s["max_len"]), dict(lse=s["lse"], out=s["out"]))
    if c["op"] == "weights":
        ws = mb.alloc_attn_workspace(d, c["n_seq"], s["q"].shape[0], s["max_tree"], s["max_len"])
        return (mb.CacheWeightsCall(d, s["q"], s["k_tree"], s["k_cache"], s["cache_len"], s["lse"], ws, s["cache_w_out"],
                                    s["tree_w"], cache_w_in=s["cache_w"], decay=s["decay"], row_weight=s["row_weight"],
                                    tree_off=s["tree_off"], tree_mask=s["tree_mask"], max_tree=s["max_tree"],
                                    max_len=s["max_len"]), dict(cache_w=s["cache_w_out"], tree_w=s["tree_w"]))
    if c["op"] == "commit":
        return (mb.CacheCommitCall(d, s["k_tree"], s["v_tree"], s["path"], s["n_path"], s["k_cache"], s["v_cache"],
                                   s["cache_len"], new_len=s["new_len"], tree_w=s["tree_w"], cache_w=s["cache_w"],
                                   tree_off=s["tree_off"], max_tree=s["max_tree"], n_layers=c["n_layers"]),
                dict(k=s["k_cache"], v=s["v_cache"], w=s["cache_w"], new_len=s["new_len"]))
    ws = mb.alloc_evict_workspace(d, c["n_layers"], c["n_seq"], s["budget"])
    return (mb.CacheEvictCall(d, s["k_cache"], s["v_cache"], s["cache_w"], s["cache_len"], s["budget"], s["recent"],
                              s["k_out"], s["v_out"], s["w_out"], ws, kept=s["kept"], new_len=s["new_len"],
                              n_layers=c["n_layers"]),
            dict(k=s["k_out"], v=s["v_out"], w=s["w_out"], kept=s["kept"], new_len=s["new_len"]))


def run(state):
    if not own:
        return _PLAIN[state["op"]](state)
    if "call" not in state:
        state["call"], state["outputs"] = _call(state)
    state["call"]()
    return state["outputs"]


# ---- from the definitions, in 64 bits

def exact(c, seed):
    if c["op"] in ("commit", "evict"):
        return None  # copies and whole numbers
    s = prepare(c, seed)
    if c["op"] == "norm":
        unit = lambda v: v / (v.pow(2).sum(1, keepdim=True) / v.shape[1] + s["eps"]).sqrt()  # noqa: E731
        y, r = s["y"].double(), s["residual"].double()
        if c["post"]:
            y = unit(y) * s["w_post"].double()
        g = torch.ones((), dtype=torch.float64, device="cuda") if s["gate"] is None else s["gate"].double()
        if c["gate"] != "none" and c["sigmoid"]:
            g = torch.sigmoid(g)
        r = r + s["scale"] * (g.unsqueeze(1) if c["gate"] == "token" else g) * y
        return dict(r=r, x=unit(r) * s["w_pre"].double())
    H, Hk, D = c["heads"], c["kv_heads"], c["head_dim"]
    off, lens = s["tree_off"].tolist(), s["cache_len"].tolist()
    M, G = off[-1], H // Hk
    lse = torch.zeros((M, H), dtype=torch.float64, device="cuda")
    out = torch.zeros((M, H, D), dtype=torch.float64, device="cuda") if c["op"] == "attention" else None
    if c["op"] == "weights":
        cache_w = torch.zeros_like(s["cache_w"], dtype=torch.float64)
        tree_w = torch.zeros((M, Hk), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        rows = slice(off[b], off[b + 1])
        T = off[b + 1] - off[b]
        sees = torch.tril(torch.ones((T, T), dtype=torch.bool, device="cuda"))
        if s["tree_mask"] is not None:
            j = torch.arange(T, device="cuda")
            sees = s["tree_mask"][rows][:, j // 32].bitwise_right_shift((j % 32).int()).bitwise_and(1).bool()
        hidden = torch.zeros((T, n + T), dtype=torch.bool, device="cuda")
        hidden[:, n:] = ~sees
        for h in range(H):
            k = torch.cat([s["k_cache"][b, h // G, :n], s["k_tree"][rows, h // G]]).double()
            a = s["q"][rows, h].double().mm(k.t().contiguous()) / math.sqrt(D)
            a.masked_fill_(hidden, -math.inf)
            if c["op"] == "attention":
                v = torch.cat([s["v_cache"][b, h // G, :n], s["v_tree"][rows, h // G]]).double()
                lse[rows, h] = torch.logsumexp(a, dim=1)
                out[rows, h] = torch.softmax(a, dim=1).mm(v)
            else:
                p = torch.exp(a - s["lse"][rows, h].double().unsqueeze(1)) * s["row_weight"][rows].double().unsqueeze(1)
                cache_w[b, h // G, :n] += p[:, :n].sum(0)
                tree_w[rows, h // G] += p[:, n:].sum(0)
        if c["op"] == "weights":
            cache_w[b, :, :n] += s["decay"] * s["cache_w"][b, :, :n].double()
    return dict(lse=lse, out=out) if c["op"] == "attention" else dict(cache_w=cache_w, tree_w=tree_w)
