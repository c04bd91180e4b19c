"""Workloads of the paged key/value cache in four bits: new tokens quantised as they are written, sequences read back into dense
tensors, and attention of new tokens over the cache (one token a sequence, a few, chunks of a prefill, mixed batches).

A value x of a key or value is held as c s: s per token, KV head and group of 32 dimensions is the smallest number of five significant
bits (and at least 2^-40) with 7.5 s >= max |x|, c = x / s rounded to a whole number (halves away from zero), -7 .. 7.  A page's plane of one head has the
codes of its tokens, head_dim / 2 bytes each, and behind them their scales, head_dim / 32 bf16 each.

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


def _attention(name, seqs, ctx, new, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", page=64, window=0, mix=1):
    """`ctx`, `new`: (lowest, highest) of a sequence's tokens and of those of them that are new (its queries)."""
    return {"name": name, "kind": "attention", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0],
            "new_hi": new[1], "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page,
            "window": window, "mix": mix}


def _write(name, seqs, ctx, new, kv_heads=8, head_dim=128, dtype="bf16", page=64, mix=1):
    """Room for the new tokens, their keys and values into it, and what the cache then holds of them read back."""
    return dict(_attention(name, seqs, ctx, new, kv_heads, kv_heads, head_dim, dtype, page, 0, mix), kind="write")


def _read(name, seqs, ctx, rows, kv_heads=8, head_dim=128, dtype="bf16", page=64, head_major=False, mix=1):
    """`rows`: how many of its last tokens are read of each sequence.  head_major: into [heads, rows, head_dim], as dense
    attention over one sequence takes them."""
    return dict(_attention(name, seqs, ctx, rows, kv_heads, kv_heads, head_dim, dtype, page, 0, mix), kind="read",
                head_major=head_major)


def listed():
    return [
        # a few short dialogues: the smallest call, latency counts; 64 dimensions a head, small pages
        _attention("step_b4_short", 4, (17, 700), (1, 1), q_heads=8, kv_heads=2, head_dim=64, page=16),
        # one step of a serving loop: 32 sequences of a thousand to 65536 tokens, one new token each
        _attention("step_b32", 32, (1000, 65536), (1, 1)),
        # a step that checks up to four guessed tokens of each sequence
        _attention("verify_b16", 16, (500, 30000), (1, 4)),
        # an ordinary chunk of a chunked prefill, odd lengths
        _attention("chunk_2k_at_30k", 1, (30011, 30011), (1999, 1999)),
        # the largest: a chunk of 8192 tokens that ends at 65536, the flagship's length and heads
        _attention("chunk_8k_at_64k", 1, (65536, 65536), (8192, 8192)),
        # whole prompts, 64 dimensions a head
        _attention("prompts_d64", 4, (1800, 2100), (2100, 2100), head_dim=64),
        # prompts, parts of prompts and single tokens of 16 sequences in one call, the paper's window
        _attention("mixed_b16_window", 16, (200, 9000), (1, 600), page=32, window=1088),
        # queries in fp32: the ends of two prompts
        _attention("chunk_f32", 2, (2500, 3001), (200, 333), q_heads=8, kv_heads=2, head_dim=64, dtype="f32", page=16),
        # the new keys and values of a serving step, and of three prompts' chunks
        _write("write_b48", 48, (300, 12000), (1, 1)),
        _write("write_32k", 3, (30000, 40000), (5000, 16384)),
        # a whole context for dense or span attention over it
        _read("read_64k", 1, (65536, 65536), (65536, 65536), head_major=True),
        # ends of ragged sequences, in fp32
        _read("read_b24_f32", 24, (500, 9000), (77, 2000), head_dim=64, dtype="f32", page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = _drawn(rng)
    del c["name"]
    return c


def _drawn(rng):
    kind = rng.choice(["step", "step", "step", "verify", "chunk", "chunk", "mixed", "prompts", "f32", "write", "write", "read"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 4), (16, 4), (8, 2), (16, 1), (12, 4), (8, 8)])
    page = rng.choice([16, 32, 64, 64, 128])
    mix, head_dim = rng.randrange(1, 1000), rng.choice([64, 128, 128, 128])
    more = dict(kv_heads=kv_heads, head_dim=head_dim, page=page, mix=mix)
    if kind in ("step", "verify"):
        seqs = _log_int(rng, 1, 96)
        hi = _log_int(rng, 100, 2097152 // (kv_heads * seqs))
        return _attention("", seqs, (max(1, hi // rng.choice([1, 8, 40])), hi), (1, 1 if kind == "step" else rng.choice([2, 3, 4])),
                          q_heads=q_heads, window=rng.choice([0, 0, 0, 1088]), **more)
    if kind == "chunk":
        seqs = rng.choice([1, 1, 2])
        new, ctx = _log_int(rng, 20, 4096 // seqs), _log_int(rng, 4096, 65536)
        return _attention("", seqs, (ctx // rng.choice([1, 2]), ctx), (max(1, new // 2), new), q_heads=q_heads,
                          window=rng.choice([0, 0, 0, 1088]), **more)
    if kind == "mixed":
        seqs, hi = rng.randrange(4, 20), _log_int(rng, 1000, 12000)
        return _attention("", seqs, (hi // 30, hi), (1, _log_int(rng, 20, 800)), q_heads=q_heads, window=rng.choice([0, 0, 1088]), **more)
    if kind == "prompts":
        seqs, hi = rng.randrange(1, 7), _log_int(rng, 200, 4000)
        return _attention("", seqs, (max(1, hi // 2), hi), (hi, hi), q_heads=q_heads, **more)
    if kind == "f32":
        q_heads, more["kv_heads"] = rng.choice([(8, 2), (4, 4), (6, 2)])
        hi = _log_int(rng, 300, 8000)
        return _attention("", rng.randrange(1, 4), (hi // 2, hi), (1, _log_int(rng, 1, 600)), q_heads=q_heads, dtype="f32", **more)
    more["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    if kind == "write":
        new = rng.choice([1, _log_int(rng, 10, 8192)])
        seqs = _log_int(rng, 1, 96) if new == 1 else rng.randrange(1, 5)
        hi = max(new, _log_int(rng, 500, 20000))
        return _write("", seqs, (max(1, hi // 20), hi), (1, new), **more)
    seqs = _log_int(rng, 1, 32)
    hi = _log_int(rng, 100, 65536 // seqs + 100)
    return _read("", seqs, (max(1, hi // 4), hi), (max(1, hi // 50), hi), head_major=rng.choice([False, True]), **more)


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
    n_pages = int(held.sum()) + 5
    order = rs.permutation(n_pages)
    table = np.full((n, int(held.max()) + 1), -1, dtype=np.int32)
    at = 0
    for s in range(n):
        table[s, : held[s]] = order[at : at + held[s]]
        at += held[s]
    return ctx, new, table, n_pages


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _tokens(shape, dtype, gen, spread):
    """Keys or values of tokens: the dimensions of a head differ in size (keys' more), as a model's do."""
    size = torch.exp(spread * _normal(shape[-1:], torch.float32, gen))
    return (_normal(shape, torch.float32, gen) * size).to(dtype)


# ---- the format ----------------------------------------------------------------------------------------

# Dimension d = 32 g + 8 c + 2 i + h of a row lies in the 16-bit unit (g, c, h) as its code i: sign and magnitude in these bits.
_SIGN, _MAGNITUDE = (15, 14, 7, 6), (0, 3, 8, 11)


def _quantise(x):
    """x [.., D] -> codes [.., D] (whole numbers) and scales [.., D / 32], in 64 bits."""
    g = x.double().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    m, e = torch.frexp(a * (2 / 15))
    quantum = torch.ldexp(torch.ones_like(a), e - 5)
    s = torch.floor(m * 32) * quantum
    s = torch.where(7.5 * (s - quantum) >= a, s - quantum, s)          # (2 / 15 is rounded)
    s = torch.where(7.5 * s < a, s + quantum, s)
    s = s.clamp(min=2.0 ** -40)
    return (torch.floor(g.abs() / s[..., None] + 0.5).clamp(max=7) * torch.sign(g)).flatten(-2), s


def _pack(codes, s, values):
    """Codes [.., P, D] and scales [.., P, D / 32] -> planes uint8 [.., P D / 2 + P D / 16]."""
    u = codes.int().unflatten(-1, (-1, 4, 4, 2))                       # g, c, i, h
    unit = sum((u[..., i, :].abs() << _MAGNITUDE[i]) | ((u[..., i, :] < 0).int() << _SIGN[i]) for i in range(4))   # g, c, h
    unit = unit.movedim(-3, -1) if values else unit.transpose(-3, -2)  # values c, h, g; keys c, g, h
    unit = torch.where(unit >= 32768, unit - 65536, unit).to(torch.int16)
    rows = unit.flatten(-3).contiguous().view(torch.uint8).flatten(-2)
    return torch.cat([rows, s.to(torch.bfloat16).contiguous().view(torch.uint8).flatten(-2)], -1)


def _unpack(planes, P, D, values):
    """Planes [.., bytes] -> the values they stand for, fp32 [.., P, D]."""
    n = D // 32
    unit = planes[..., : P * D // 2].contiguous().view(torch.int16).int().unflatten(-1, (P, 4, 2, n) if values else (P, 4, n, 2))
    unit = unit.movedim(-1, -3) if values else unit.transpose(-3, -2)  # g, c, h
    code = torch.stack([((unit >> _MAGNITUDE[i]) & 7) * (1 - 2 * ((unit >> _SIGN[i]) & 1)) for i in range(4)], -2)   # g, c, i, h
    s = planes[..., P * D // 2 :].contiguous().view(torch.bfloat16).unflatten(-1, (P, n)).float()
    return (code.flatten(-3) * s[..., None]).flatten(-2)


def _plane_bytes(c):
    return c["page"] * (c["head_dim"] // 2 + c["head_dim"] // 16)


def _pool(c, n_pages, gen, values):
    pool = torch.empty(n_pages, c["kv_heads"], _plane_bytes(c), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (c["kv_heads"] * c["page"] * c["head_dim"]))
    spread = 0.2 if values else 0.8
    size = torch.exp(spread * _normal((c["kv_heads"], 1, c["head_dim"]), torch.float32, gen))
    for p in range(0, n_pages, step):
        m = min(step, n_pages - p)
        x = (_normal((m, c["kv_heads"], c["page"], c["head_dim"]), torch.float32, gen) * size).to(torch.bfloat16)
        pool[p : p + m] = _pack(*_quantise(x), values)
    return pool


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, P, D, Hkv, Hq = DTYPES[c["dtype"]], c["page"], c["head_dim"], c["kv_heads"], c["q_heads"]
    ctx, new, table, n_pages = _plan(c)
    n = len(ctx)
    k, v = _pool(c, n_pages, gen, False), _pool(c, n_pages, gen, True)
    held = ctx - new if c["kind"] == "write" else ctx   # a write finds the sequence as it was before
    if c["kind"] == "write":
        for s in range(n):
            table[s, -(-held[s] // P):] = -1
    slots, width = table.shape
    ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages)
    # the cache's bookkeeping is one buffer, so that a program can keep and restore it with one copy
    ints = torch.cat([_ints(table).reshape(-1), _ints(held), _ints(ref)])
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
    else:
        shape = (Hkv, T, D) if c.get("head_major") else (T, Hkv, D)
        s["k_out"], s["v_out"] = (torch.empty(shape, dtype=dt, device=DEV) for _ in range(2))
        if c.get("head_major"):
            s["k_out"], s["v_out"] = s["k_out"].transpose(0, 1), s["v_out"].transpose(0, 1)
        if c["kind"] == "write":
            s["k_new"], s["v_new"] = _tokens((T, Hkv, D), dt, gen, 0.8), _tokens((T, Hkv, D), dt, gen, 0.2)
        else:
            s["first"] = _ints(ctx - new)
    if own:
        import paper_2601_18401_b200 as sla

        s["sla"] = sla
        s["cache"] = sla.make_cache_q4(k, v, s["table"], s["n_tokens"], s["ref"], page_tokens=P, head_dim=D, dtype=dt)
        s["h"] = sla.Handle(0, sla.sla_paged_workspace_bytes(s["cache"], Hq, n, T))
    return s


def run(s):
    c = s["c"]
    if not own:
        return {"attention": _plain_attention, "write": _plain_write, "read": _plain_read}[c["kind"]](s)
    sla, h, cache = s["sla"], s["h"], s["cache"]
    if c["kind"] == "attention":
        return sla.sla_paged_attention(h, s["q"], cache, s["cu"], max_new=s["max_new"], window=c["window"], out=s["out"], lse=s["lse"])
    if c["kind"] == "read":
        return sla.sla_cache_read(h, cache, s["cu"], s["first"], k_out=s["k_out"], v_out=s["v_out"])
    s["ints"].copy_(s["ints0"])
    first = sla.sla_cache_extend(h, cache, s["cu"])
    sla.sla_cache_append(h, cache, s["cu"], first, s["k_new"], s["v_new"])
    k, v = sla.sla_cache_read(h, cache, s["cu"], first, k_out=s["k_out"], v_out=s["v_out"])
    return k, v, s["ints"], first


# ---- the plain forms ----------------------------------------------------------------------------------


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
    heads = max(1, (1 << 30) // (n * G * max(len(r), 8) * len(j)))                    # KV heads a pass, by the memory of S
    for g in range(0, Hkv, heads):
        kf, vf = (_unpack(s[name][:, g : g + heads][pages], P, D, name == "v").transpose(1, 2).reshape(n, -1, len(j), D) for name in "kv")
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


def _places(s, first):
    """Page and row in it of every row of the call."""
    P = s["c"]["page"]
    new = s["cu"][1:] - s["cu"][:-1]
    x = torch.repeat_interleave(torch.arange(len(new), device=DEV), new.long(), output_size=s["n_new"])
    pos = first[x] + torch.arange(s["n_new"], device=DEV) - s["cu"][:-1][x]
    return s["table"][x, (pos // P).long()].long(), (pos % P).long()


def _row_bytes(c, at):
    """Where the row `at` of a plane has its codes and its scales: indices [rows, bytes]."""
    P, D = c["page"], c["head_dim"]
    codes, scales = torch.arange(D // 2, device=DEV), torch.arange(D // 16, device=DEV)
    return torch.cat([at[:, None] * (D // 2) + codes, P * (D // 2) + at[:, None] * (D // 16) + scales], 1)


def _plain_read(s, first=None):
    c = s["c"]
    page, at = _places(s, s["first"] if first is None else first)
    where = _row_bytes(c, at)[:, None, :]
    heads = torch.arange(c["kv_heads"], device=DEV)[None, :, None]
    step = 16384
    for a in range(0, len(page), step):
        for name in "kv":
            rows = s[name][page[a : a + step, None, None], heads, where[a : a + step]]          # [rows, heads, bytes]
            s[name + "_out"][a : a + step] = _unpack(rows, 1, c["head_dim"], name == "v").squeeze(-2).to(s[name + "_out"].dtype)
    return s["k_out"], s["v_out"]


def _plain_write(s):
    c, table, lengths, ref = s["c"], s["table"], s["n_tokens"], s["ref"]
    s["ints"].copy_(s["ints0"])
    P = c["page"]
    new = s["cu"][1:] - s["cu"][:-1]
    first = lengths.clone()
    have, want = (first + P - 1) // P, (first + new + P - 1) // P
    before = torch.cumsum(want - have, 0) - (want - have)
    free = torch.sort((ref > 0).int(), stable=True)[1].int()      # the free pages first, in ascending order
    col = torch.arange(s["width"], device=DEV)
    fresh = (col >= have[:, None]) & (col < want[:, None])
    table.copy_(torch.where(fresh, free[(before[:, None] + col - have[:, None]).clamp(0, len(free) - 1).long()], table))
    taken = torch.arange(len(free), device=DEV) < (want - have).sum()
    ref.index_put_((free.long(),), taken.int(), accumulate=True)
    lengths.add_(new)
    page, at = _places(s, first)
    where = _row_bytes(c, at)[:, None, :]
    heads = torch.arange(c["kv_heads"], device=DEV)[None, :, None]
    step = 16384
    for a in range(0, len(page), step):
        for name in "kv":
            codes, scales = _quantise(s[name + "_new"][a : a + step])
            s[name][page[a : a + step, None, None], heads, where[a : a + step]] = _pack(codes[..., None, :], scales[..., None, :], name == "v")
    _plain_read(s, first)
    return s["k_out"], s["v_out"], s["ints"], first.int()


# ---- the definitions in 64 bits ------------------------------------------------------------------------


def _held(x):
    """What the cache holds of x [.., D], in 64 bits: scales looked up among all of five bits, codes counted by the borders passed."""
    numbers = torch.tensor([m * 2.0 ** e for e in range(-44, 36) for m in range(16, 32)], dtype=torch.float64, device=DEV)
    g = x.double().unflatten(-1, (-1, 32))
    s = numbers[torch.searchsorted(7.5 * numbers, g.abs().amax(-1))][..., None]
    code = torch.zeros_like(g)
    for j in range(7):
        code += g.abs() >= (j + 0.5) * s
    return (torch.sign(g) * code * s).flatten(-2)


def _planes_to_values(planes, P, D, values):
    """[pages, bytes] -> [pages * P, D] in 64 bits, unit by unit through a table of the four codes of each 16-bit word."""
    bits = np.arange(65536)
    four = np.stack([(bits >> m & 7) * np.where(bits >> b & 1, -1.0, 1.0) for m, b in ((0, 15), (3, 14), (8, 7), (11, 6))], 1)
    four = torch.from_numpy(four).to(DEV)
    n = D // 32
    word = planes[:, : P * D // 2].reshape(-1, P, D // 4, 2).int()
    word = four[(word[..., 0] + 256 * word[..., 1]).long()]                        # [pages, P, units, 4]
    scale = planes[:, P * D // 2 :].contiguous().view(torch.bfloat16).reshape(-1, P, n).double()
    out = torch.empty(planes.shape[0], P, D, dtype=torch.float64, device=DEV)
    for d in range(D):
        g, c, i, h = d // 32, d // 8 % 4, d // 2 % 4, d % 2
        out[..., d] = word[:, :, (2 * c + h) * n + g if values else (c * n + g) * 2 + h, i] * scale[..., g]
    return out.reshape(-1, D)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    D, Hkv, G, P = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["page"]
    ctx, new, _, _ = _plan(c)
    if c["kind"] == "write":
        return _held(s["k_new"]), _held(s["v_new"]), None, None
    table = s["table"].cpu().numpy()

    def tokens(name, x, g, lo, hi):
        """Rows lo .. hi - 1 of KV head g of sequence x."""
        pages = torch.from_numpy(table[x, lo // P : -(-hi // P)].astype(np.int64)).to(DEV)
        return _planes_to_values(s[name][pages, g], P, D, name == "v")[lo - lo // P * P :][: hi - lo]

    if c["kind"] == "read":
        k, v = (torch.empty_like(s["k_out"], dtype=torch.float64) for _ in range(2))
        for x in range(c["seqs"]):
            r0 = int(s["cu"][x])
            for g in range(Hkv):
                for name, out in (("k", k), ("v", v)):
                    out[r0 : r0 + int(new[x]), g] = tokens(name, x, g, int(ctx[x] - new[x]), int(ctx[x]))
        return k, v
    out = torch.zeros(s["n_new"], c["q_heads"], D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["n_new"], c["q_heads"], dtype=torch.float64, device=DEV)
    for x in range(c["seqs"]):
        n, r0 = int(ctx[x]), int(s["cu"][x])
        for g in range(Hkv):
            k, v = tokens("k", x, g, 0, n), tokens("v", x, g, 0, n)
            for a in range(0, int(new[x]), 1024):
                e = min(a + 1024, int(new[x]))
                p = n - int(new[x]) + torch.arange(a, e, device=DEV)[:, None]
                j = torch.arange(n, device=DEV)
                seen = (j <= p) & (j > p - c["window"]) if c["window"] else j <= p
                for h in range(g * G, g * G + G):
                    z = torch.where(seen, s["q"][r0 + a : r0 + e, h].double() @ k.T / math.sqrt(D), NEG)
                    lse[r0 + a : r0 + e, h] = torch.logsumexp(z, -1)
                    out[r0 + a : r0 + e, h] = torch.exp(z - lse[r0 + a : r0 + e, h, None]) @ v
    return out, lse


# ---- the work ------------------------------------------------------------------------------------------


def work(case):
    """Bytes: each input read once (of the cache what the queries see), each output written once.  Operations: the products of
    queries and keys, and of weights and values."""
    c = case
    ctx, new, table, n_pages = _plan(c)
    es, P, D, Hkv, Hq = (4 if c["dtype"] == "f32" else 2), c["page"], c["head_dim"], c["kv_heads"], c["q_heads"]
    row, T = Hkv * (D // 2 + D // 16), int(new.sum())
    if c["kind"] == "read":
        return {"bytes": 2 * T * (row + Hkv * D * es) + 4 * int((new // P + 1).sum()), "flops": 0}
    if c["kind"] == "write":   # the new tokens in, their codes out and in again, their values out
        return {"bytes": 2 * T * (2 * row + 2 * Hkv * D * es) + 8 * (table.size + table.shape[0] + n_pages), "flops": 0}
    first = ctx - new
    w = c["window"] or int(ctx.max()) + 1
    keys = np.minimum(ctx, new + w - 1)
    pairs = sum(int(np.minimum(np.arange(f + 1, n + 1), w).sum()) for f, n in zip(first, ctx))
    return {"bytes": int(2 * row * keys.sum() + T * Hq * (2 * D * es + 4) + 4 * (keys // P + 1).sum()), "flops": 4 * D * Hq * pairs}
