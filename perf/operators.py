"""Workloads of the paged key/value cache: attention of a chunk of new tokens over it (one token a sequence, chunks of a
chunked prefill, mixed batches), appending tokens, forking and compacting, and the span decode step over it.

A case gives ranges; which length each sequence of a case has, and which page each part of it lies in, follows from the case's
``mix`` alone, the tensors' values from the seed.  Pages of a sequence are scattered over the pool, as they are after a while
of serving.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


def _attention(name, seqs, ctx, new, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", page=64, token_major=False, window=0,
               mix=1):
    """`ctx`, `new`: (lowest, highest) of a sequence's tokens and of those of them that are new (its queries)."""
    return {"name": name, "kind": "attention", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0],
            "new_hi": new[1], "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page,
            "token_major": token_major, "window": window, "mix": mix}


def _append(name, seqs, ctx, new, kv_heads=8, head_dim=128, dtype="bf16", page=64, token_major=False, mix=1):
    return dict(_attention(name, seqs, ctx, new, kv_heads, kv_heads, head_dim, dtype, page, token_major, 0, mix), kind="append")


def _fork(name, parents, children, ctx, kv_heads=8, head_dim=128, dtype="bf16", page=64, mix=1):
    """`children` new sequences, each a copy of one of the `parents`; the children of the step before are released."""
    return dict(_attention(name, parents, ctx, (1, 1), kv_heads, kv_heads, head_dim, dtype, page, False, 0, mix), kind="fork",
                children=children)


def _compact(name, seqs, ctx, kv_heads=8, head_dim=128, dtype="bf16", page=64, mix=1):
    """Every second sequence has ended; what the others hold moves to the front of the pool."""
    return dict(_attention(name, seqs, ctx, (1, 1), kv_heads, kv_heads, head_dim, dtype, page, False, 0, mix), kind="compact")


def _span(name, seqs, ctx, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", page=64, top_k=8, span_len=0, mix=1):
    return dict(_attention(name, seqs, ctx, (1, 1), q_heads, kv_heads, head_dim, dtype, page, False, 0, mix), kind="span",
                top_k=top_k, span_len=span_len)


def listed():
    return [
        # a few short dialogues: the smallest call, latency counts; 64 dimensions a head, small pages
        _attention("step_b4_short", 4, (17, 700), (1, 1), q_heads=8, kv_heads=2, head_dim=64, page=16),
        # one step of a serving loop: 32 sequences of a thousand to 65536 tokens, one new token each
        _attention("step_b32", 32, (1000, 65536), (1, 1)),
        # an ordinary chunk of a chunked prefill, odd lengths
        _attention("chunk_2k_at_30k", 1, (30011, 30011), (1999, 1999)),
        # the largest: a chunk of 8192 tokens that ends at 65536, the flagship's length and heads
        _attention("chunk_8k_at_64k", 1, (65536, 65536), (8192, 8192)),
        # prompts, parts of prompts and single tokens of 16 sequences in one call, token-major pages, the paper's window
        _attention("mixed_b16_window", 16, (200, 9000), (1, 600), token_major=True, page=32, window=1088),
        # fp32 arithmetic: the ends of two prompts
        _attention("chunk_f32", 2, (2500, 3001), (200, 333), q_heads=8, kv_heads=2, head_dim=64, dtype="f32", page=16),
        # the new keys and values of a serving step, and of three prompts' chunks
        _append("append_b48", 48, (300, 12000), (1, 1)),
        _append("append_32k", 3, (30000, 40000), (5000, 16384)),
        # 48 continuations of 6 prompts (parallel sampling), those of the step before released
        _fork("fork_6_to_48", 6, 48, (700, 9000)),
        # a pool of about 1 GB of which half has ended
        _compact("compact_64", 64, (500, 20000)),
        # the span decode step: 16 sequences of 8 to 130 thousand tokens, base span length by the paper's rule ceil(sqrt(i))
        _span("span_step_b16", 16, (8000, 130000)),
        # and the million-token decode configuration
        _span("span_step_1m", 1, (1048576, 1048576), kv_heads=4, top_k=16, span_len=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = _drawn(rng)
    del c["name"]
    return c


def _drawn(rng):
    kind = rng.choice(["step", "step", "chunk", "chunk", "mixed", "f32", "append", "fork", "compact", "span", "span"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 4), (16, 4), (8, 2), (16, 1), (12, 4), (8, 8)])
    page = rng.choice([16, 32, 64, 64, 128])
    mix, head_dim = rng.randrange(1, 1000), rng.choice([64, 128, 128, 128])
    more = dict(kv_heads=kv_heads, head_dim=head_dim, page=page, mix=mix)
    if kind == "step":
        seqs = _log_int(rng, 1, 96)
        hi = _log_int(rng, 100, 2097152 // (kv_heads * seqs))
        return _attention("", seqs, (max(1, hi // rng.choice([1, 8, 40])), hi), (1, rng.choice([1, 1, 3])), q_heads=q_heads,
                          token_major=rng.choice([False, True]), window=rng.choice([0, 0, 0, 1088]), **more)
    if kind == "chunk":
        seqs = rng.choice([1, 1, 2])
        new, ctx = _log_int(rng, 20, 4096 // seqs), _log_int(rng, 4096, 65536)
        return _attention("", seqs, (ctx // rng.choice([1, 2]), ctx), (max(1, new // 2), new), q_heads=q_heads,
                          token_major=rng.choice([False, True]), window=rng.choice([0, 0, 0, 1088]), **more)
    if kind == "mixed":
        seqs, hi = rng.randrange(4, 20), _log_int(rng, 1000, 12000)
        return _attention("", seqs, (hi // 30, hi), (1, _log_int(rng, 20, 800)), q_heads=q_heads,
                          token_major=rng.choice([False, True]), window=rng.choice([0, 0, 1088]), **more)
    if kind == "f32":
        q_heads, more["kv_heads"] = rng.choice([(8, 2), (4, 4), (6, 2)])
        hi = _log_int(rng, 300, 8000)
        return _attention("", rng.randrange(1, 4), (hi // 2, hi), (1, _log_int(rng, 1, 600)), q_heads=q_heads, dtype="f32", **more)
    if kind == "append":
        new = rng.choice([1, _log_int(rng, 10, 8192)])
        seqs = _log_int(rng, 1, 96) if new == 1 else rng.randrange(1, 5)
        hi = max(new, _log_int(rng, 500, 20000))
        return _append("", seqs, (max(1, hi // 20), hi), (1, new), token_major=rng.choice([False, True]),
                       dtype=rng.choice(["bf16", "bf16", "f32"]), **more)
    if kind == "fork":
        parents = rng.randrange(1, 9)
        return _fork("", parents, parents * rng.randrange(2, 12), (100, _log_int(rng, 500, 12000)), **more)
    if kind == "compact":
        seqs = rng.randrange(4, 64)
        return _compact("", seqs, (50, _log_int(rng, 500, 65536 * 8 // (kv_heads * seqs))), **more)
    seqs = _log_int(rng, 1, 24)
    hi = _log_int(rng, 3000, 1048576 * 8 // (kv_heads * max(4, seqs)))
    return _span("", seqs, (hi // rng.choice([1, 3, 12]), hi), q_heads=q_heads, top_k=rng.choice([4, 8, 16]),
                 span_len=rng.choice([0, 0, math.isqrt(hi)]), **more)


# ---- what a case means --------------------------------------------------------------------------------


def _plan(c):
    """Lengths and pages of a case's sequences: (tokens, new tokens) per sequence, the page table, pages of the pool."""
    rs = np.random.RandomState(c["mix"])
    n = c["seqs"]

    def spread(lo, hi):
        return np.rint(np.exp(rs.uniform(math.log(lo), math.log(hi), n))).astype(np.int64)

    ctx = spread(c["ctx_lo"], c["ctx_hi"])
    new = np.minimum(spread(c["new_lo"], c["new_hi"]), ctx)
    P = c["page"]
    held = -(-ctx // P)
    width = int(held.max()) + 1
    slots = n + c.get("children", 0)
    n_pages = int(held.sum()) + 2 * c.get("children", 0) + 5
    order = rs.permutation(n_pages)
    table = np.full((slots, width), -1, dtype=np.int32)
    at = 0
    for s in range(n):
        table[s, : held[s]] = order[at : at + held[s]]
        at += held[s]
    return ctx, new, table, n_pages


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _on_grid(t):
    """Rounds to multiples of 1/64 in place: every sum of products of two such tensors is then exact in fp32 in any order, so
    that a selection by score does not depend on the order of summation."""
    return t.mul_(64).round_().mul_(1 / 64)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, P, D, Hkv, Hq = DTYPES[c["dtype"]], c["page"], c["head_dim"], c["kv_heads"], c["q_heads"]
    ctx, new, table, n_pages = _plan(c)
    n = len(ctx)
    if c["token_major"]:
        k, v = (_normal((n_pages, P, Hkv, D), dt, gen).transpose(1, 2) for _ in range(2))
    else:
        k, v = (_normal((n_pages, Hkv, P, D), dt, gen) for _ in range(2))
    held = ctx - new if c["kind"] == "append" else ctx   # an append finds the sequence as it was before
    if c["kind"] == "append":
        for s in range(n):
            table[s, -(-held[s] // P):] = -1
    slots, width = table.shape
    ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages)
    lengths = np.zeros(slots, dtype=np.int32)
    lengths[:n] = held
    # the cache's bookkeeping is one buffer, so that a program can keep and restore it with one copy
    ints = torch.cat([_ints(table).reshape(-1), _ints(lengths), _ints(ref)])
    at = slots * width
    s = {"c": c, "k": k, "v": v, "ints0": ints, "ints": ints.clone(), "width": width}
    s["table"] = s["ints"][:at].view(slots, width)
    s["n_tokens"], s["ref"] = s["ints"][at : at + slots], s["ints"][at + slots :]
    cu = np.concatenate([[0], np.cumsum(new)])
    s["cu"], s["n_new"], s["max_new"], s["max_ctx"] = _ints(cu), int(cu[-1]), int(new.max()), int(ctx.max())
    T = s["n_new"]
    if c["kind"] == "attention":
        s["q"] = _normal((T, Hq, D), dt, gen)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(T, Hq, dtype=torch.float32, device=DEV)
    elif c["kind"] == "append":
        s["k_new"], s["v_new"] = _normal((T, Hkv, D), dt, gen), _normal((T, Hkv, D), dt, gen)
    elif c["kind"] == "fork":
        s["src"] = _ints(np.arange(c["children"]) % n)
        s["dst"] = _ints(n + np.arange(c["children"]))
    elif c["kind"] == "compact":
        s["ended"] = _ints(np.arange(0, n, 2))
    else:
        _on_grid(k)
        s["q_s"], s["q"] = _on_grid(_normal((n, Hq, D), dt, gen)), _normal((n, Hq, D), dt, gen)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(n, Hq, dtype=torch.float32, device=DEV)
        s["anchor"] = torch.empty(n, Hq, c["top_k"], dtype=torch.int32, device=DEV)
        s["score"] = torch.empty(n, Hq, c["top_k"], dtype=torch.float32, device=DEV)
    if own:
        import paper_2601_18401_b200 as sla

        s["sla"] = sla
        s["cache"] = sla.make_cache(k, v, s["table"], s["n_tokens"], s["ref"])
        s["params"] = sla.make_params(c.get("top_k", 1), c.get("span_len", 0), head_dim=D) if c["kind"] == "span" else None
        s["h"] = sla.Handle(0, sla.sla_paged_workspace_bytes(s["cache"], Hq, n, T, params=s["params"]))
    return s


def run(s):
    c = s["c"]
    if not own:
        return _plain(s)
    sla, h, cache = s["sla"], s["h"], s["cache"]
    if c["kind"] == "attention":
        return sla.sla_paged_attention(h, s["q"], cache, s["cu"], max_new=s["max_new"], window=c["window"], out=s["out"], lse=s["lse"])
    if c["kind"] == "span":
        return sla.sla_paged_decode_step(h, s["q_s"], s["q"], cache, s["params"], max_tokens=s["max_ctx"], out=s["out"],
                                         lse=s["lse"], out_anchor=s["anchor"], out_score=s["score"])
    if c["kind"] == "fork":   # releases what it makes: it finds the same cache every time
        sla.sla_cache_release(h, cache, s["dst"])
        pairs = sla.sla_cache_fork(h, cache, s["src"], s["dst"])
        return s["k"], s["v"], s["ints"], pairs
    s["ints"].copy_(s["ints0"])
    if c["kind"] == "append":
        first = sla.sla_cache_extend(h, cache, s["cu"])
        sla.sla_cache_append(h, cache, s["cu"], first, s["k_new"], s["v_new"])
        return s["k"], s["v"], s["ints"], first
    sla.sla_cache_release(h, cache, s["ended"])
    moves = sla.sla_cache_compact(h, cache)
    return s["k"], s["v"], s["ints"], moves


# ---- the plain forms ----------------------------------------------------------------------------------


def _plain(s):
    kind = s["c"]["kind"]
    if kind == "attention":
        return _plain_attention(s)
    if kind == "span":
        return _plain_span(s)
    if kind != "fork":
        s["ints"].copy_(s["ints0"])
    return {"append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[kind](s)


def _plain_attention(s):
    c, q = s["c"], s["q"]
    P, D, Hkv, Hq = c["page"], c["head_dim"], c["kv_heads"], c["q_heads"]
    G, n = Hq // Hkv, c["seqs"]
    new = s["cu"][1:] - s["cu"][:-1]
    r = torch.arange(s["max_new"], device=DEV)
    rows = (s["cu"][:-1, None] + r).clamp(max=s["n_new"] - 1)                       # [n, R]
    pos = (s["n_tokens"] - new)[:, None] + r                                          # [n, R]
    pages = s["table"][:, : -(-s["max_ctx"] // P)].clamp(min=0).long()                # [n, pages]
    j = torch.arange(pages.shape[1] * P, device=DEV)
    seen = j <= pos[:, :, None]                                                       # [n, R, keys]
    if c["window"]:
        seen &= j > pos[:, :, None] - c["window"]
    live = r < new[:, None]                                                           # rows that exist
    b, at = torch.arange(n, device=DEV)[:, None].expand_as(rows)[live], r.expand_as(rows)[live]
    out, lse = s["out"], s["lse"]
    heads = max(1, (1 << 30) // (n * G * len(r) * len(j)))                            # KV heads a pass, by the memory of S
    for g in range(0, Hkv, heads):
        kf = s["k"][:, g : g + heads][pages].transpose(1, 2).reshape(n, -1, len(j), D).float()
        vf = s["v"][:, g : g + heads][pages].transpose(1, 2).reshape(n, -1, len(j), D).float()
        m_heads = kf.shape[1]
        qf = q[rows][:, :, g * G : g * G + m_heads * G].float().reshape(n, len(r), m_heads, G, D).permute(0, 2, 3, 1, 4)
        S = (qf.reshape(n, m_heads, -1, D) @ kf.transpose(-1, -2)).mul_(D ** -0.5).view(n, m_heads, G, len(r), len(j))
        S.masked_fill_(~seen[:, None, None], NEG)
        m = S.amax(-1, keepdim=True)
        S.sub_(m.clamp(min=-3e38)).exp_()
        total = S.sum(-1, keepdim=True)
        o = (S.view(n, m_heads, -1, len(j)) @ vf).view(n, m_heads, G, len(r), D) / total.clamp(min=1e-30)
        o = o.permute(0, 3, 1, 2, 4).reshape(n, len(r), -1, D)
        z = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n, len(r), -1)
        out[:, g * G : g * G + m_heads * G] = o[b, at].to(out.dtype)
        lse[:, g * G : g * G + m_heads * G] = z[b, at]
    return out, lse


def _free_pages(ref):
    """Pages by (in use, index): the free ones first, in ascending order."""
    return torch.sort((ref > 0).int(), stable=True)[1].int()


def _plain_append(s):
    P, table, lengths, ref = s["c"]["page"], s["table"], s["n_tokens"], s["ref"]
    new = s["cu"][1:] - s["cu"][:-1]
    first = lengths.clone()
    have, want = (first + P - 1) // P, (first + new + P - 1) // P
    before = torch.cumsum(want - have, 0) - (want - have)
    free = _free_pages(ref)
    col = torch.arange(s["width"], device=DEV)
    fresh = (col >= have[:, None]) & (col < want[:, None])
    table.copy_(torch.where(fresh, free[(before[:, None] + col - have[:, None]).clamp(0, len(free) - 1).long()], table))
    taken = torch.arange(len(free), device=DEV) < (want - have).sum()
    ref.index_put_((free.long(),), taken.int(), accumulate=True)
    lengths.add_(new)
    x = torch.repeat_interleave(torch.arange(len(new), device=DEV), new.long(), output_size=s["n_new"])
    pos = first[x] + torch.arange(s["n_new"], device=DEV) - s["cu"][:-1][x]
    page = table[x, (pos // P).long()].long()
    s["k"][page, :, pos % P] = s["k_new"]
    s["v"][page, :, pos % P] = s["v_new"]
    return s["k"], s["v"], s["ints"], first.int()


def _plain_release(s, seq):
    rows = s["table"][seq]
    s["ref"].index_put_((rows.clamp(min=0).reshape(-1).long(),), -(rows >= 0).int().reshape(-1), accumulate=True)
    s["table"][seq] = -1
    s["n_tokens"][seq] = 0


def _plain_fork(s):
    P, table, lengths, ref, src, dst = s["c"]["page"], s["table"], s["n_tokens"], s["ref"], s["src"].long(), s["dst"].long()
    _plain_release(s, dst)
    n = lengths[src]
    full, part = n // P, (n % P > 0).int()
    free = _free_pages(ref)[(torch.cumsum(part, 0) - part).long()]
    col = torch.arange(s["width"], device=DEV)
    shared = col < full[:, None]
    rows = torch.where(shared, table[src], -1)
    last = (col == full[:, None]) & (part[:, None] > 0)
    old = torch.where(part > 0, table[src].gather(1, full[:, None].long()).squeeze(1), -1)
    table[dst] = torch.where(last, free[:, None], rows)
    lengths[dst] = n
    ref.index_put_((rows.clamp(min=0).reshape(-1).long(),), shared.int().reshape(-1), accumulate=True)
    ref.index_put_((free.long(),), part, accumulate=True)
    to = torch.where(part > 0, free, -1)
    # a sequence without a partly filled page copies its first page onto itself
    a, b = torch.where(part > 0, old, table[src, 0]).long(), torch.where(part > 0, free, table[src, 0]).long()
    s["k"][b], s["v"][b] = s["k"][a], s["v"][a]
    return s["k"], s["v"], s["ints"], torch.stack([old, to]).int()


def _plain_compact(s):
    table, ref = s["table"], s["ref"]
    _plain_release(s, s["ended"].long())
    n, live = len(ref), ref > 0
    count = live.sum()
    idx = torch.arange(n, device=DEV)
    movers, holes = live & (idx >= count), ~live & (idx < count)
    n_moves = movers.sum()
    src = torch.sort((~movers).int(), stable=True)[1]
    dst = torch.sort((~holes).int(), stable=True)[1]
    on = idx < n_moves
    to = idx.clone()
    to[src] = torch.where(on, dst, src)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    moved = torch.where(on, ref[src], 0)
    ref.mul_((idx < count).int())
    ref.index_put_((dst,), moved, accumulate=True)
    most = int(n_moves)   # the pages that move are copied, not the pool
    s["k"][dst[:most]], s["v"][dst[:most]] = s["k"][src[:most]], s["v"][src[:most]]
    return s["k"], s["v"], s["ints"], torch.stack([torch.where(on, src, -1), torch.where(on, dst, -1)]).int()


def _plain_span(s):
    c = s["c"]
    P, D, Hkv, Hq, K, n = c["page"], c["head_dim"], c["kv_heads"], c["q_heads"], c["top_k"], c["seqs"]
    G, table, lengths = Hq // Hkv, s["table"], s["n_tokens"].long()
    b = torch.arange(n, device=DEV)

    # anchors n_tokens - (t+1)^2 of the last position and their scores
    t = lengths[:, None] - (torch.arange(math.isqrt(s["max_ctx"]), device=DEV) + 1) ** 2
    page = table[b[:, None], t.clamp(min=0) // P].long()
    kf = s["k"][page, :, t.clamp(min=0) % P].float()                                 # [n, anchors, Hkv, D]
    S = torch.einsum("ngxd,nagd->ngxa", s["q_s"].float().view(n, Hkv, G, D), kf).reshape(n, Hq, -1)
    S.masked_fill_((t < 0)[:, None], NEG)
    score, order = torch.sort(S, dim=-1, descending=True, stable=True)
    score, order = score[..., :K], order[..., :K]
    got = score > NEG
    anchor = torch.where(got, t[b[:, None, None], order], -1)
    # spans [t - 2 l, t] in ascending order, each cut where the one before ends
    i = lengths - 1
    root = torch.sqrt(i.double()).long()
    ell = torch.full_like(i, c["span_len"]) if c["span_len"] else root + (root * root < i)
    hi = torch.sort(anchor, dim=-1)[0]
    lo = torch.where(hi >= 0, (hi - 2 * ell[:, None, None]).clamp(min=0), 0)
    ends = torch.cat([torch.full_like(hi[..., :1], -1), hi[..., :-1]], -1)           # the spans' ends ascend with their starts
    lo = torch.maximum(lo, ends + 1)
    longest = 2 * (c["span_len"] or math.isqrt(s["max_ctx"]) + 1) + 1
    j = lo[..., None] + torch.arange(longest, device=DEV)                             # [n, Hq, K, tokens]
    seen = (j <= hi[..., None]).reshape(n, Hq, -1)
    j = j.clamp(max=s["max_ctx"] - 1).reshape(n, Hq, -1)
    group = (torch.arange(Hq, device=DEV) // G)[:, None]
    out, lse = s["out"], s["lse"]
    step = max(1, (1 << 29) // (Hq * K * longest * D))                                # sequences a pass, by the memory of K
    for x in range(0, n, step):
        jj, ok = j[x : x + step], seen[x : x + step]
        page = table[b[x : x + step, None, None], jj // P].clamp(min=0).long()
        kf, vf = (p[page, group, jj % P].float() for p in (s["k"], s["v"]))
        L = (kf * s["q"][x : x + step, :, None].float()).sum(-1).mul_(D ** -0.5).masked_fill_(~ok, NEG)
        m = L.amax(-1, keepdim=True)
        p = (L - m).exp()
        total = p.sum(-1, keepdim=True)
        out[x : x + step] = ((p[..., None] * vf).sum(-2) / total).to(out.dtype)
        lse[x : x + step] = (m + total.log()).squeeze(-1)
    s["anchor"].copy_(anchor)
    s["score"].copy_(score)
    return out, lse, s["anchor"], s["score"]


# ---- the definitions in 64 bits ------------------------------------------------------------------------


def exact(case, seed):
    c, s = case, prepare(case, seed)
    D, Hkv, G, P = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["page"]
    ctx, new, _, _ = _plan(c)
    if c["kind"] in ("fork", "compact"):
        return None   # copies of whole pages: no computed numbers
    table = s["table"].cpu().numpy()

    def tokens(pool, x, g, n):
        """The first n rows of KV head g of sequence x."""
        pages = torch.from_numpy(table[x, : -(-n // P)].astype(np.int64)).to(DEV)
        return pool[pages, g].reshape(-1, D)[:n].double()

    def attend(q, k, v, seen=None):
        z = q @ k.T / math.sqrt(D)
        if seen is not None:
            z = torch.where(seen, z, NEG)
        lse = torch.logsumexp(z, -1)
        return torch.exp(z - lse[:, None]) @ v, lse

    if c["kind"] == "append":
        k, v = s["k"].clone(), s["v"].clone()
        free = [p for p in range(k.shape[0]) if s["ref"][p].item() == 0] if k.shape[0] <= 4096 else None
        if free is None:
            return None
        at = 0
        for x in range(c["seqs"]):
            n0, r0 = int(ctx[x] - new[x]), int(s["cu"][x])
            row = [int(p) for p in table[x] if p >= 0]
            while len(row) * P < ctx[x]:
                row.append(free[at])
                at += 1
            done = 0
            while done < new[x]:
                page, off = row[(n0 + done) // P], (n0 + done) % P
                m = min(P - off, int(new[x]) - done)
                k[page, :, off : off + m] = s["k_new"][r0 + done : r0 + done + m].transpose(0, 1)
                v[page, :, off : off + m] = s["v_new"][r0 + done : r0 + done + m].transpose(0, 1)
                done += m
        return k.double(), v.double(), None, None
    if c["kind"] == "attention":
        out = torch.zeros(s["n_new"], c["q_heads"], D, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s["n_new"], c["q_heads"], dtype=torch.float64, device=DEV)
        for x in range(c["seqs"]):
            n, r0 = int(ctx[x]), int(s["cu"][x])
            for g in range(Hkv):
                k, v = tokens(s["k"], x, g, n), tokens(s["v"], x, g, n)
                for a in range(0, int(new[x]), 1024):
                    e = min(a + 1024, int(new[x]))
                    p = n - int(new[x]) + torch.arange(a, e, device=DEV)[:, None]
                    j = torch.arange(n, device=DEV)
                    seen = (j <= p) & (j > p - c["window"]) if c["window"] else j <= p
                    for h in range(g * G, g * G + G):
                        out[r0 + a : r0 + e, h], lse[r0 + a : r0 + e, h] = attend(s["q"][r0 + a : r0 + e, h].double(), k, v, seen)
        return out, lse
    out = torch.zeros(c["seqs"], c["q_heads"], D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["seqs"], c["q_heads"], dtype=torch.float64, device=DEV)
    score = torch.full((c["seqs"], c["q_heads"], c["top_k"]), NEG, dtype=torch.float64, device=DEV)
    for x in range(c["seqs"]):
        n = int(ctx[x])
        ell = c["span_len"] or math.isqrt(n - 1) + (math.isqrt(n - 1) ** 2 < n - 1)
        at = torch.tensor([n - (a + 1) ** 2 for a in range(math.isqrt(n))], device=DEV)
        for g in range(Hkv):
            k, v = tokens(s["k"], x, g, n), tokens(s["v"], x, g, n)
            for h in range(g * G, g * G + G):
                z, order = torch.sort(k[at] @ s["q_s"][x, h].double(), descending=True, stable=True)
                m = min(c["top_k"], len(at))
                score[x, h, :m] = z[:m]
                seen = torch.zeros(n, dtype=torch.bool, device=DEV)
                for t in at[order[:m]].tolist():
                    seen[max(0, t - 2 * ell) : t + 1] = True
                o, l = attend(s["q"][x, h : h + 1].double(), k[seen], v[seen])
                out[x, h], lse[x, h] = o[0], l[0]
    return out, lse, None, score


# ---- the work ------------------------------------------------------------------------------------------


def _union(n, ell, draws):
    """Expected number of keys in the union of `draws` spans [t - 2 ell, t] whose anchors are drawn evenly from those of n - 1."""
    t = n - np.arange(1, math.isqrt(n) + 1, dtype=np.int64) ** 2
    at = np.concatenate([np.maximum(t - 2 * ell, 0), t + 1])
    order = np.argsort(at, kind="stable")
    cover = np.cumsum(np.concatenate([np.ones(t.size), -np.ones(t.size)])[order])[:-1]
    return float((np.diff(at[order]) * (1 - (1 - cover / t.size) ** min(draws, t.size))).sum())


def work(case):
    """Bytes: each input read once (of the cache what the queries see), each output written once.  Operations: the products of
    queries and keys, and of weights and values."""
    c = case
    ctx, new, table, n_pages = _plan(c)
    es, P, D, Hkv, Hq = (4 if c["dtype"] == "f32" else 2), c["page"], c["head_dim"], c["kv_heads"], c["q_heads"]
    row, T = Hkv * D * es, int(new.sum())
    if c["kind"] == "attention":
        first = ctx - new
        w = c["window"] or int(ctx.max()) + 1
        keys = np.minimum(ctx, new + w - 1)
        pairs = sum(int(np.minimum(np.arange(f + 1, n + 1), w).sum()) for f, n in zip(first, ctx))
        return {"bytes": int(2 * row * keys.sum() + T * Hq * (2 * D * es + 4) + 4 * (keys // P + 1).sum()),
                "flops": 4 * D * Hq * pairs}
    if c["kind"] == "span":
        total = flops = 0.0
        G = Hq // Hkv
        for n in ctx.tolist():
            ell = c["span_len"] or math.isqrt(n - 1) + (math.isqrt(n - 1) ** 2 < n - 1)
            total += Hkv * D * es * (math.isqrt(n) + 2 * _union(n, ell, c["top_k"] * G))
            flops += Hq * D * (2 * math.isqrt(n) + 4 * _union(n, ell, c["top_k"]))
        return {"bytes": int(total) + len(ctx) * Hq * (3 * D * es + 4 + 8 * c["top_k"]), "flops": int(flops)}
    ints = 4 * (table.size + table.shape[0] + n_pages)
    if c["kind"] == "append":
        return {"bytes": 4 * T * row + 2 * ints, "flops": 0}
    if c["kind"] == "fork":
        part = sum(1 for x in range(c["children"]) if ctx[x % len(ctx)] % P)
        return {"bytes": 4 * part * P * row + 4 * ints, "flops": 0}
    ref = np.bincount(table[1::2][table[1::2] >= 0].ravel(), minlength=n_pages)
    moves = int((ref[int((ref > 0).sum()):] > 0).sum())
    return {"bytes": 4 * moves * P * row + 4 * ints, "flops": 0}
