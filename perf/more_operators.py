"""Operators of a serving step around the budgeted MoE layer whose speed is tracked: queries and keys made ready for attention, a
paged cache held in 8 bits, single tokens that attend over it, and the draft's verification.

  rope    queries and keys normed for each head and rotated to their place in the tree (HeadRopeCall)
  cache   keys and values quantised into pages, and the written entries read back (PagedWriteCall, PagedReadCall)
  paged   one new token of every sequence over its pages (PagedAttentionCall)
  verify  accepted path and next token from the target's logits and given random numbers (DraftVerifyCall)

Keys, values and queries are N(0, 1) (queries scaled to give scores a standard deviation of 2); pages of a sequence lie anywhere in
the pool; target logits are N(0, 2.5) with the drafted tokens raised to probabilities around 0.5; sampled drafts are drawn from logits
that are the target's plus noise.
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_HEADS = [(32, 4), (32, 8), (16, 16), (8, 8), (12, 2), (20, 4), (7, 1), (64, 8)]


# ---- the cases

def _paged(name, dtype, code, n_seq, heads, kv_heads, head_dim, length, page, ragged=False):
    return dict(name=name, op="paged", dtype=dtype, code=code, n_seq=n_seq, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                length=length, page=page, ragged=ragged)


def listed():
    return [
        # one token of a fresh chain, place 1021: what every layer of an undrafted decoding step asks, all latency
        dict(name="rope_token", op="rope", dtype="bf16", n_seq=1, tree=1, heads=32, kv_heads=4, head_dim=128, rot=128,
             interleaved=False, norm=True, masked=False, start=1021),
        # four of the largest trees, q, k and v out of one projection, places far into a long context
        dict(name="rope_trees", op="rope", dtype="bf16", n_seq=4, tree=511, heads=32, kv_heads=8, head_dim=128, rot=128,
             interleaved=False, norm=True, masked=True, start=1000003),
        # the end of a verification step in all 48 layers: up to eight accepted tokens of eight requests
        dict(name="cache_step", op="cache", dtype="bf16", code="i8", n_layers=48, n_seq=8, tree=63, path=8, kv_heads=4,
             head_dim=128, page=16, start=119),
        # four prompts of a layer written whole, and read back
        dict(name="cache_prompt", op="cache", dtype="bf16", code="e4m3", n_layers=1, n_seq=4, tree=8190, path=0, kv_heads=8,
             head_dim=128, page=64, start=0),
        # one token over a short cache: latency
        _paged("paged_token", "bf16", "plain", 1, 32, 4, 128, 1021, 16),
        # a batch of requests of different lengths, pages as wide as the layer
        _paged("paged_batch", "bf16", "plain", 64, 32, 8, 128, 8189, 32, ragged=True),
        # many requests over pages of 8-bit integers, 16 query heads to a KV head
        _paged("paged_i8", "bf16", "i8", 48, 64, 4, 128, 16381, 64, ragged=True),
        # a single request over a very long context in 8-bit floats
        _paged("paged_e4m3_long", "bf16", "e4m3", 1, 32, 4, 128, 131071, 128),
        # a small model at full precision
        _paged("paged_f32", "f32", "plain", 4, 8, 8, 64, 2039, 16, ragged=True),
        # four drafted tokens of one request, each drawn from the drafter's distribution, small vocabulary
        dict(name="verify_chain", op="verify", dtype="f32", n_seq=1, tree=5, vocab=32003, pad=1, sampled=True, path=6),
        # the benchmark's tree over a large vocabulary, drafts without a distribution of their own
        dict(name="verify_tree", op="verify", dtype="bf16", n_seq=1, tree=63, vocab=131071, pad=1, sampled=False, path=16),
        # sixteen requests with the benchmark's tree
        dict(name="verify_batch", op="verify", dtype="bf16", n_seq=16, tree=63, vocab=50001, pad=7, sampled=False, path=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["paged", "paged", "paged", "rope", "cache", "verify"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    code = rng.choice(["plain", "i8", "e4m3"])
    while True:
        heads, kv_heads = rng.choice(_HEADS)
        head_dim = rng.choice([64, 96, 128, 128, 192, 256])
        page = rng.choice([16, 32, 64, 128, 256])
        if op == "paged":
            c = dict(op=op, dtype=dtype, code=code, n_seq=_log(rng, 1, 128), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                     length=_log(rng, 1, 131072), page=page, ragged=rng.random() < 0.6)
            if c["n_seq"] * kv_heads * c["length"] * head_dim <= 4e8 and c["n_seq"] * heads * c["length"] <= 5e7:
                return c
        elif op == "rope":
            c = dict(op=op, dtype=dtype, n_seq=_log(rng, 1, 16), tree=_log(rng, 1, 511), heads=heads, kv_heads=kv_heads,
                     head_dim=head_dim, rot=16 * rng.randint(1, head_dim // 16), interleaved=rng.random() < 0.4,
                     norm=rng.random() < 0.7, masked=rng.random() < 0.6, start=_log(rng, 1, 1 << 20))
            if c["n_seq"] * c["tree"] * (heads + kv_heads) * head_dim <= 10_000_000:
                return c
        elif op == "cache":
            path = _log(rng, 1, 12) if rng.random() < 0.6 else 0
            c = dict(op=op, dtype=dtype, code=code, n_layers=_log(rng, 1, 48), n_seq=_log(rng, 1, 8),
                     tree=max(path, _log(rng, 1, 255 if path else 8000)), path=path, kv_heads=kv_heads, head_dim=head_dim, page=page,
                     start=_log(rng, 1, 300) if path else 0)
            if c["n_layers"] * c["n_seq"] * (c["tree"] + c["start"]) * kv_heads * head_dim <= 30_000_000:
                return c
        else:
            sampled = rng.random() < 0.4
            c = dict(op=op, dtype=dtype, n_seq=_log(rng, 1, 16), tree=_log(rng, 2, 12 if sampled else 127), vocab=_log(rng, 1000, 160000),
                     pad=rng.choice([0, 1, 3, 8]), sampled=sampled, path=rng.choice([4, 8, 16]))
            if c["n_seq"] * c["tree"] * c["vocab"] * (2 if sampled else 1) <= 50_000_000:
                return c


def _lengths(c):
    """Entries of every sequence: all alike, or falling to half of the first one's."""
    n = c["n_seq"]
    return [max(1, c["length"] - (s * c["length"]) // (2 * n)) if c["ragged"] else c["length"] for s in range(n)]


def _written(c):
    """Entries that every sequence writes: the accepted path, or a whole prompt."""
    if c["path"] == 0:
        return [max(1, c["tree"] - (s * c["tree"]) // (2 * c["n_seq"])) for s in range(c["n_seq"])]
    return [1 + (5 * s + c["path"] - 1) % c["path"] for s in range(c["n_seq"])]


def _row_bytes(c):
    """Bytes of one row of keys or values in a page."""
    return c["head_dim"] * _BYTES[c["dtype"]] if c["code"] == "plain" else c["head_dim"] + 4


def work(c):
    b = _BYTES[c["dtype"]]
    if c["op"] == "rope":
        n = c["n_seq"] * c["tree"] * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        words = c["n_seq"] * c["tree"] * ((c["tree"] + 31) // 32) if c["masked"] else 0
        return {"bytes": 2 * n * b + 4 * words, "flops": 8 * n}
    if c["op"] == "cache":  # source and pages written, the same pages and the layer's own form read back
        rows = 2 * c["n_layers"] * sum(_written(c)) * c["kv_heads"]
        return {"bytes": rows * (2 * c["head_dim"] * b + 2 * _row_bytes(c)), "flops": 4 * rows * c["head_dim"]}
    if c["op"] == "paged":
        n = sum(_lengths(c))
        return {"bytes": 2 * n * c["kv_heads"] * _row_bytes(c) + c["n_seq"] * c["heads"] * (2 * c["head_dim"] * b + 4),
                "flops": 4 * n * c["heads"] * c["head_dim"]}
    # every row of logits: which ones lie on the path is known when they have been looked at
    n = c["n_seq"] * c["tree"] * c["vocab"] * (2 if c["sampled"] else 1)
    return {"bytes": n * b, "flops": 4 * n}


# ---- inputs

def _tree_words(n_seq, n, gen):
    """Packed ancestor sets [n_seq * n, ceil(n / 32)] of random trees (every token's parent is one of the 8 in front of it; token
    0 is the root of all): bit j of a token's row is set if it sees token j."""
    rows = []
    for _ in range(n_seq):
        back = torch.randint(1, 9, (n,), generator=gen).tolist()
        seen = [0] * n
        for t in range(n):
            seen[t] = (seen[max(t - back[t], 0)] if t else 0) | (1 << t)
        rows += seen
    words = [[(r >> (32 * w)) & 0xFFFFFFFF for w in range((n + 31) // 32)] for r in rows]
    return torch.tensor(words, dtype=torch.int64).to(torch.int32)


def _randn(shape, dtype, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _table(entries, page, gen):
    """Page table [n_seq, pages of the longest] and the number of pages: those of a sequence lie anywhere in the pool, unused places
    of the table hold -1."""
    need = [(n + page - 1) // page for n in entries]
    pool = sum(need) + 3
    order = torch.randperm(pool, generator=gen).tolist()
    at, rows = 0, []
    for n in need:
        rows.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    return _i32(rows), pool


def _codes(x, code):
    """(codes, scales) of rows x [..., D] in 8 bits: integers of amax / 127, or e4m3 with the smallest power of two that amax fits."""
    amax = x.float().abs().amax(dim=-1)
    if code == "i8":
        inv = torch.clamp(127.0 / amax, max=torch.finfo(torch.float32).max)
        return torch.round(x.double() * inv.double()[..., None]).to(torch.int8), amax / 127.0
    mantissa, exponent = torch.frexp(amax / 448.0)  # amax / 448 = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = torch.clamp(torch.where(mantissa == 0.5, exponent - 1, exponent), min=-126)
    scale = torch.ldexp(torch.ones_like(amax), torch.where(amax == 0, -126, e))
    return (x.float() / scale[..., None]).to(torch.float8_e4m3fn), scale


def prepare(c, seed):
    dev, host = torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    dt = _TORCH[c["dtype"]]
    s = dict(op=c["op"], case=c)
    S = c["n_seq"]
    if c["op"] == "rope":
        H, Hk, D, T = c["heads"], c["kv_heads"], c["head_dim"], c["tree"]
        M = S * T
        qkv = _randn((M, H + 2 * Hk, D), dt, dev, 3.0)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + Hk]
        s["w_q"], s["w_k"] = ((1.0 + _randn((D,), torch.float32, dev, 0.2)).to(dt) if c["norm"] else None for _ in range(2))
        s["freq"] = torch.tensor([1e6 ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)], dtype=torch.float32).cuda()
        s["tree_off"], s["max_tree"] = _i32([T * i for i in range(S + 1)]), T
        s["tree_mask"] = _tree_words(S, T, host).cuda() if c["masked"] else None
        s["cache_len"], s["eps"] = _i32([max(0, c["start"] - 97 * i) for i in range(S)]), 1e-6
        s["q_out"], s["k_out"] = (torch.zeros((M, n, D), dtype=dt, device="cuda") for n in (H, Hk))
    elif c["op"] == "cache":
        Hk, D, L, T, n = c["kv_heads"], c["head_dim"], c["n_layers"], c["tree"], _written(c)
        s["k_tree"], s["v_tree"] = (_randn((L, S * T, Hk, D), dt, dev) for _ in range(2))
        starts = [max(0, c["start"] - 7 * i) for i in range(S)]
        s["cache_len"], s["tree_off"], s["max_tree"] = _i32(starts), _i32([T * i for i in range(S + 1)]), T
        s["page_table"], pool = _table([a + b for a, b in zip(starts, n)], c["page"], host)
        if c["path"]:
            s["path"] = torch.randint(0, T, (S, c["path"]), generator=host).sort(dim=1).values.to(torch.int32).cuda()
        else:
            s["path"] = torch.arange(T, dtype=torch.int32, device="cuda").expand(S, T).contiguous()
        s["n_path"] = _i32(n)
        s["new_len"] = torch.zeros(S, dtype=torch.int32, device="cuda")
        held = dict(plain=dt, i8=torch.int8, e4m3=torch.float8_e4m3fn)[c["code"]]
        s["k_pages"], s["v_pages"] = (torch.zeros((L, pool, Hk, c["page"], D), dtype=held, device="cuda") for _ in range(2))
        s["k_scale"], s["v_scale"] = (None if c["code"] == "plain" else torch.zeros((L, pool, Hk, c["page"]), device="cuda")
                                      for _ in range(2))
        s["max_len"] = max(a + b for a, b in zip(starts, n))
        s["k"], s["v"] = (torch.zeros((L, S, Hk, s["max_len"] + 3, D), dtype=dt, device="cuda") for _ in range(2))
    elif c["op"] == "paged":
        H, Hk, D, lens = c["heads"], c["kv_heads"], c["head_dim"], _lengths(c)
        s["page_table"], pool = _table(lens, c["page"], host)
        for x in ("k", "v"):
            if c["code"] == "plain":
                s[x + "_pages"], s[x + "_scale"] = _randn((1, pool, Hk, c["page"], D), dt, dev), None
            else:
                wide = _randn((1, pool, Hk, c["page"], D), dt, dev)
                parts = [_codes(p, c["code"]) for p in wide.split(max(1, (1 << 27) // (Hk * c["page"] * D)), dim=1)]
                s[x + "_pages"], s[x + "_scale"] = (torch.cat(v, dim=1) for v in zip(*parts))
        s["q"] = _randn((S, H, D), dt, dev, 2.0)
        s["cache_len"], s["max_len"] = _i32(lens), c["length"]
        s["out"], s["lse"] = torch.zeros((S, H, D), dtype=dt, device="cuda"), torch.zeros((S, H), device="cuda")
    else:
        _prepare_verify(s, c, dt, dev, host)
    return s


def _prepare_verify(s, c, dt, dev, host):
    S, T, V = c["n_seq"], c["tree"], c["vocab"]
    M = S * T
    rows = torch.arange(M, device="cuda")
    logits = torch.randn((M, V + c["pad"]), generator=dev, device="cuda").mul_(2.5)
    s["tree_off"], s["max_tree"] = _i32([T * i for i in range(S + 1)]), T
    if c["sampled"]:
        s["tree_mask"] = None
        # a share of mass on a few tokens, so that drafter and target often agree
        top = torch.randint(0, V, (M, 4), generator=dev, device="cuda")
        logits.scatter_(1, top, math.log(V) + 2.5 + torch.rand((M, 4), generator=dev, device="cuda"))
        drafts = (logits + torch.randn(logits.shape, generator=dev, device="cuda").mul_(0.7)).to(dt)
        drawn = torch.multinomial(torch.softmax(drafts[:, :V].float(), dim=1), 1, generator=dev)[:, 0]
        s["draft_logits"] = drafts[:, :V]
        s["tokens"] = drawn.roll(1).to(torch.int32)  # token t was drawn from the row of the one in front of it
    else:
        words = _tree_words(S, T, host)
        s["tree_mask"], s["draft_logits"] = words.cuda(), None
        s["tokens"] = torch.randint(0, V, (M,), generator=dev, device="cuda").to(torch.int32)
        parent = rows.view(S, T)[:, :1] + _parents(s, S, T)
        raised = math.log(V) + 3.1 + torch.empty((M,), device="cuda").uniform_(-1.0, 2.5, generator=dev)
        logits[parent.reshape(-1), s["tokens"].long()] = raised
    s["logits"] = logits.to(dt)[:, :V]
    s["temperature"] = torch.tensor([[1.0, 0.8, 0.0, 0.6][i % 4] for i in range(S)]).cuda()
    s["u_accept"] = torch.rand((M,), generator=dev, device="cuda", dtype=torch.float64)
    s["u_sample"] = torch.rand((S,), generator=dev, device="cuda", dtype=torch.float64)
    s["path"] = torch.zeros((S, c["path"]), dtype=torch.int32, device="cuda")
    s["n_path"], s["next_token"] = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    s["accepted"] = torch.zeros(M, device="cuda")


# ---- the plain forms

def _bits(s, S, T):
    """[S, T, T] truth values: token t of a tree sees token j."""
    at = torch.arange(T, device="cuda")
    if s["tree_mask"] is None:
        return (at[None, :] <= at[:, None]).expand(S, T, T)
    words = s["tree_mask"].view(S, T, -1)
    return ((words[..., None] >> torch.arange(32, device="cuda")) & 1).flatten(2)[..., :T] != 0


def _parents(s, S, T):
    """[S, T] place of every token's parent: the last token in front of it that it sees (the root: 0)."""
    at = torch.arange(T, device="cuda")
    return torch.where(_bits(s, S, T) & (at[None, :] < at[:, None]), at, 0).amax(dim=2)


def _plain_rope(s):
    c, eps = s["case"], s["eps"]
    S, T, R = c["n_seq"], c["tree"], c["rot"]
    place = (s["cache_len"][:, None] + _bits(s, S, T).sum(dim=2) - 1).reshape(-1)
    angle = place.double()[:, None] * s["freq"].double()  # 64 bits: places times frequencies lose their fraction in 32
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    res = []
    for x, w, out in ((s["q"], s["w_q"], s["q_out"]), (s["k"], s["w_k"], s["k_out"])):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(dim=2, keepdim=True) + eps) * w.float()
        head, rest = x[..., :R], x[..., R:]
        if c["interleaved"]:
            a, b = head[..., 0::2], head[..., 1::2]
            head = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).flatten(2)
        else:
            a, b = head[..., :R // 2], head[..., R // 2:]
            head = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
        res.append(out.copy_(torch.cat([head, rest], dim=2)))
    return dict(q=res[0], k=res[1])


def _plain_cache(s):
    c = s["case"]
    S, P, page = c["n_seq"], s["path"].shape[1], c["page"]
    i = torch.arange(P, device="cuda")
    i = torch.where(i < s["n_path"][:, None], i, 0).reshape(-1)  # places behind the path's end: its first entry once more
    seq = torch.arange(S, device="cuda").repeat_interleave(P, output_size=S * P)
    entry = s["cache_len"][seq] + i
    src = s["tree_off"][seq] + s["path"][seq, i]
    where, slot = s["page_table"][seq, entry // page].long(), entry % page
    for x in ("k", "v"):
        rows, pages, scales = s[x + "_tree"][:, src], s[x + "_pages"], s[x + "_scale"]
        if c["code"] == "plain":
            pages[:, where, :, slot] = rows.transpose(0, 1)
            back = pages[:, where, :, slot]
        else:
            codes, scale = _codes(rows, c["code"])
            raw = pages.view(torch.int8)
            raw[:, where, :, slot] = codes.view(torch.int8).transpose(0, 1)
            scales[:, where, :, slot] = scale.transpose(0, 1)
            back = raw[:, where, :, slot].view(pages.dtype).float() * scales[:, where, :, slot][..., None]
        s[x][:, seq, :, entry] = back.to(s[x].dtype)
    torch.add(s["cache_len"], s["n_path"], out=s["new_len"])
    return dict(k=s["k"], v=s["v"], new_len=s["new_len"])


def _plain_paged(s):
    c, n = s["case"], s["max_len"]
    S, H, D = s["q"].shape
    Hk, table = c["kv_heads"], s["page_table"].long().clamp(min=0)

    def dense(x):
        pages = s[x + "_pages"][0].view(torch.int8)[table] if c["code"] != "plain" else s[x + "_pages"][0][table]
        pages = pages.view(s[x + "_pages"].dtype).transpose(1, 2).flatten(2, 3)[:, :, :n].float()  # [S, Hk, n, D]
        return pages if c["code"] == "plain" else pages.mul_(s[x + "_scale"][0][table].transpose(1, 2).flatten(2)[:, :, :n, None])

    q = s["q"].float().reshape(S, Hk, H // Hk, D)
    a = (q @ dense("k").transpose(2, 3)).mul_(D ** -0.5)
    a = a.masked_fill_((torch.arange(n, device="cuda") >= s["cache_len"][:, None])[:, None, None], -math.inf)
    top = a.amax(dim=3, keepdim=True)
    p = a.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    s["out"].copy_((p @ dense("v")).div_(total).reshape(S, H, D))
    s["lse"].copy_((top + total.log()).reshape(S, H))
    return dict(out=s["out"], lse=s["lse"])


def _plain_verify(s):
    """In 64 bits throughout: acceptance and the draw are decisions, and have to fall the same way for every order of the sums."""
    c = s["case"]
    S, T, V, P = c["n_seq"], c["tree"], c["vocab"], c["path"]
    at = torch.arange(T, device="cuda")
    tokens, greedy = s["tokens"].long().view(S, T), s["temperature"] <= 0
    inverse = 1.0 / torch.where(greedy, 1.0, s["temperature"]).double()

    def probabilities(x):
        x = x.double().view(S, T, V)
        w = ((x - x.amax(dim=2, keepdim=True)) * inverse[:, None, None]).exp_()
        return w.div_(w.sum(dim=2, keepdim=True))

    p, best = probabilities(s["logits"]), s["logits"].view(S, T, V).argmax(dim=2)
    bits, parent = _bits(s, S, T), _parents(s, S, T)
    seq = torch.arange(S, device="cuda")[:, None]
    mine = p[seq, parent, tokens]
    # older[t, j]: j is a child of the same parent, in front of t
    older = (parent[:, :, None] == parent[:, None, :]) & (at[None, :] < at[:, None]) & (at > 0)
    same = older & (tokens[:, :, None] == tokens[:, None, :])
    repeated = same.any(dim=2)
    u = s["u_accept"].view(S, T)
    if c["sampled"]:
        q = probabilities(s["draft_logits"])
        accept = u * q[seq, parent, tokens] < mine
    else:
        gone = torch.where(older & ~repeated[:, None, :], mine[:, None, :], 0.0).sum(dim=2)
        accept = (u * (1.0 - gone) < mine) & ~repeated
    accept = torch.where(greedy[:, None], (tokens == best[seq, parent]) & ~repeated, accept)
    chosen = (accept & ~(older & accept[:, None, :]).any(dim=2)) | (at == 0)
    whole = (~bits | chosen[:, None, :]).all(dim=2)  # the token and all that it comes from
    depth = bits.sum(dim=2)
    on = whole & (depth <= P)
    last = torch.where(on, at, 0).amax(dim=1)
    s["n_path"].copy_(on.sum(dim=1))
    s["path"].fill_(-1).scatter_(1, torch.where(on, depth - 1, 0), torch.where(on, at, 0).to(torch.int32))
    s["accepted"].copy_(on.reshape(-1))
    child = (parent == last[:, None]) & (at > 0)
    beyond = child & whole  # where the path is cut: the token that comes next on it
    w = p[seq[:, 0], last]
    if c["sampled"]:
        rest = torch.clamp(w - q[seq[:, 0], last], min=0.0)
        w = torch.where(child.any(dim=1, keepdim=True) & (rest.sum(dim=1, keepdim=True) > 0), rest, w)
    else:
        keep = torch.ones_like(w).scatter_reduce_(1, tokens, torch.where(child, 0.0, 1.0).double(), "amin")
        rest = w * keep
        w = torch.where(rest.sum(dim=1, keepdim=True) > 0, rest, w)
    total = w.cumsum(dim=1)
    past = total > (s["u_sample"] * total[:, -1])[:, None]
    drawn = torch.where(past.any(dim=1), past.to(torch.int8).argmax(dim=1), V - 1 - (w > 0).to(torch.int8).flip(1).argmax(dim=1))
    token = torch.where(greedy, best[seq[:, 0], last], drawn)
    cut = torch.where(beyond, tokens, 0).amax(dim=1)
    s["next_token"].copy_(torch.where(beyond.any(dim=1), cut, token))
    return {k: s[k] for k in ("path", "n_path", "next_token", "accepted")}


_PLAIN = dict(rope=_plain_rope, cache=_plain_cache, paged=_plain_paged, verify=_plain_verify)


# ---- the framework's calls

def _calls(s):
    """The call objects that a program keeps next to its buffers (arguments marshalled once), and the outputs."""
    from paper_2602_16052_amd import binding as mb

    c = s["case"]
    code = mb.BF16 if c["dtype"] == "bf16" else mb.F32
    if c["op"] == "verify":
        d = mb.VerifyDesc(c["vocab"], code)
        ws = mb.alloc_verify_workspace(d, c["n_seq"], s["logits"].shape[0], c["sampled"])
        return ([mb.DraftVerifyCall(d, s["logits"], s["tokens"], s["u_accept"], s["u_sample"], s["path"], s["n_path"],
                                    s["next_token"], ws, draft_logits=s["draft_logits"], temperature=s["temperature"],
                                    accepted=s["accepted"], tree_off=s["tree_off"], tree_mask=s["tree_mask"],
                                    max_tree=s["max_tree"])],
                {k: s[k] for k in ("path", "n_path", "next_token", "accepted")})
    capacity = s["k"].shape[-2] if c["op"] == "cache" else 1
    d = mb.AttnDesc(c.get("heads", c["kv_heads"]), c["kv_heads"], c["head_dim"], capacity, code)
    if c["op"] == "rope":
        return ([mb.HeadRopeCall(d, s["q"], s["k"], s["q_out"], s["k_out"], s["freq"], rot_dim=c["rot"],
                                 interleaved=c["interleaved"], norm=c["norm"], w_q=s["w_q"], w_k=s["w_k"], eps=s["eps"],
                                 cache_len=s["cache_len"], tree_off=s["tree_off"], tree_mask=s["tree_mask"],
                                 max_tree=s["max_tree"])], dict(q=s["q_out"], k=s["k_out"]))
    kind = dict(plain=mb.CACHE_PLAIN, i8=mb.CACHE_I8, e4m3=mb.CACHE_E4M3)[c["code"]]
    cache = mb.PagedCache(kind, s["k_pages"], s["v_pages"], s["page_table"], s["k_scale"], s["v_scale"])
    if c["op"] == "cache":
        return ([mb.PagedWriteCall(d, cache, s["k_tree"], s["v_tree"], s["cache_len"], path=s["path"], n_path=s["n_path"],
                                   new_len=s["new_len"], tree_off=s["tree_off"], max_tree=s["max_tree"]),
                 mb.PagedReadCall(d, cache, s["new_len"], s["k"], s["v"], first=s["cache_len"], max_len=s["max_len"])],
                dict(k=s["k"], v=s["v"], new_len=s["new_len"]))
    ws = mb.alloc_paged_attention_workspace(d, cache, c["n_seq"], s["max_len"])
    return ([mb.PagedAttentionCall(d, cache, s["q"], s["cache_len"], ws, s["out"], lse=s["lse"], max_len=s["max_len"])],
            dict(out=s["out"], lse=s["lse"]))


def run(state):
    if not own:
        return _PLAIN[state["op"]](state)
    if "calls" not in state:
        state["calls"], state["outputs"] = _calls(state)
    for call in state["calls"]:
        call()
    return state["outputs"]


# ---- from the definitions, in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    return dict(rope=_exact_rope, cache=_exact_cache, paged=_exact_paged, verify=_exact_verify)[c["op"]](s, c)


def _exact_verify(s, c):
    """The walk down every tree, token by token."""
    S, T, V, P = c["n_seq"], c["tree"], c["vocab"], c["path"]
    tokens, u, u_sample = s["tokens"].tolist(), s["u_accept"].tolist(), s["u_sample"].tolist()
    sees = [1 << t | (1 << t) - 1 for t in range(T)] * S
    if s["tree_mask"] is not None:
        sees = [sum((w & 0xFFFFFFFF) << (32 * i) for i, w in enumerate(r)) for r in s["tree_mask"].tolist()]
    paths, lengths, following, accepted = [], [], [], torch.zeros(S * T)
    for b, heat in enumerate(s["temperature"].tolist()):
        children = [[] for _ in range(T)]
        for t in range(1, T):
            children[(sees[b * T + t] & ((1 << t) - 1)).bit_length() - 1].append(t)
        path, token = [0], None
        while token is None:
            row = s["logits"][b * T + path[-1]]
            mass = torch.softmax(row.double() / heat, dim=0) if heat > 0 else (row == row.max()).double()
            if heat <= 0:
                mass = torch.zeros_like(mass).index_fill_(0, mass.argmax()[None], 1.0)
            step = None
            for t in children[path[-1]]:
                x, rest = tokens[b * T + t], mass.clone()
                proposal = torch.zeros_like(mass).index_fill_(0, torch.tensor([x], device="cuda"), 1.0)
                if c["sampled"] and heat > 0:
                    proposal = torch.softmax(s["draft_logits"][b * T + path[-1]].double() / heat, dim=0)
                if (u[b * T + t] if heat > 0 else 0.0) * float(proposal[x]) < float(mass[x]):
                    step = t
                    break
                rest = (mass - proposal).clamp_(min=0.0)
                mass = rest / rest.sum() if float(rest.sum()) > 0 else mass
            if step is not None and len(path) < P:
                path.append(step)
            elif step is not None:
                token = tokens[b * T + step]
            else:
                total = mass.cumsum(0)
                token = int((total > u_sample[b] * total[-1]).to(torch.int8).argmax())
        accepted[[b * T + t for t in path]] = 1.0
        paths.append(path + [-1] * (P - len(path)))
        lengths.append(len(path))
        following.append(token)
    return dict(path=torch.tensor(paths), n_path=torch.tensor(lengths), next_token=torch.tensor(following), accepted=accepted.double())


def _exact_rope(s, c):
    S, T, R = c["n_seq"], c["tree"], c["rot"]
    if s["tree_mask"] is None:
        depth = torch.arange(T).repeat(S, 1)
    else:
        depth = torch.tensor([sum(bin(w & 0xFFFFFFFF).count("1") for w in r) - 1 for r in s["tree_mask"].tolist()]).view(S, T)
    place = (s["cache_len"].cpu()[:, None] + depth).reshape(-1).cuda().double()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(place, s["freq"].double()))[:, None]
    res = {}
    for x in ("q", "k"):
        v = s[x].double()
        if c["norm"]:
            v = v / (v.pow(2).sum(2, keepdim=True) / c["head_dim"] + s["eps"]).sqrt() * s["w_" + x].double()
        v = v.clone()
        first, second = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(v[..., first], v[..., second]) * turn
        v[..., first], v[..., second] = z.real, z.imag
        res[x] = v
    return res


def _exact_cache(s, c):
    """Values that the codes stand for, from the rule of the codes."""
    out, new_len = {}, s["cache_len"] + s["n_path"]
    for x in ("k", "v"):
        dense = torch.zeros(s[x].shape, dtype=torch.float64, device="cuda")
        for b in range(c["n_seq"]):
            n, at = int(s["n_path"][b]), int(s["cache_len"][b])
            rows = s[x + "_tree"][:, b * c["tree"] + s["path"][b, :n].long()].double()
            if c["code"] != "plain":
                most = rows.abs().max(dim=3, keepdim=True).values
                if c["code"] == "i8":  # scale and its inverse are stored in 32 bits
                    rows = torch.round(rows * (127.0 / most).float().double()) * (most / 127.0).float().double()
                else:
                    scale = torch.exp2(torch.ceil(torch.log2(most / 448.0)))
                    y = rows / scale
                    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=1e-30))), min=-6.0) - 3.0)
                    rows = torch.round(y / step) * step * scale
            dense[:, b, :, at:at + n] = rows.transpose(1, 2)
        out[x] = dense
    return dict(out, new_len=new_len)


def _exact_paged(s, c):
    H, Hk, D, page = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(c)):
        ids = s["page_table"][b, :(n + page - 1) // page].tolist()
        for g in range(Hk):
            rows = {}
            for x in ("k", "v"):
                v = torch.stack([s[x + "_pages"][0, i, g].to(torch.float32) for i in ids]).double().view(-1, D)[:n]
                if c["code"] != "plain":
                    v = v * torch.stack([s[x + "_scale"][0, i, g] for i in ids]).double().view(-1, 1)[:n]
                rows[x] = v
            heads = slice(g * (H // Hk), (g + 1) * (H // Hk))
            a = s["q"][b, heads].double().mm(rows["k"].t().contiguous()) / math.sqrt(D)
            out[b, heads] = torch.softmax(a, dim=1).mm(rows["v"])
            lse[b, heads] = torch.logsumexp(a, dim=1)
    return dict(out=out, lse=lse)
