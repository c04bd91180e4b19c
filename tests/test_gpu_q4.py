"""The paged cache in four bits on the device: rounding as tokens are written, reading back, bookkeeping, and attention over it, against
64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_util as U
import q4_util as Q

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def sla():
    import paper_2601_18401_b200 as sla_pkg
    return sla_pkg


@pytest.fixture(scope="module")
def handle(sla):
    h = sla.Handle(0, 1 << 30)
    yield h
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


def planes(sla, n_pages, hkv, page, d, gap=0):
    """k, v of planes whose every byte is 255: scales that are NaN."""
    size = sla.q4_plane_bytes(page, d)
    return [torch.full((n_pages, hkv * (size + gap) + gap), 255, dtype=torch.uint8, device="cuda:0")[:, : hkv * (size + gap)]
            .unflatten(-1, (hkv, size + gap))[..., :size] for _ in range(2)]


def cu_of(new):
    return U.device_ints(np.concatenate([[0], np.cumsum(new)]))


# ---- writing and reading back -------------------------------------------------------------------------------------------------------


def empty_cache(sla, n_pages=40, hkv=2, page=16, d=64, slots=6, width=20, dtype=BF16, gap=0):
    k, v = planes(sla, n_pages, hkv, page, d, gap)
    ints = [U.device_ints(np.full((slots, width), -1)), U.device_ints(np.zeros(slots)), U.device_ints(np.zeros(n_pages))]
    return sla.make_cache_q4(k, v, *ints, page_tokens=page, head_dim=d, dtype=dtype), k, v, ints[0]


def normal(shape, dtype, seed, spread=1.0):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    x = torch.empty(shape, device="cuda:0").normal_(generator=g)
    return (x * torch.exp(spread * torch.empty(shape[-1:], device="cuda:0").normal_(generator=g))).to(dtype)


@pytest.mark.parametrize("dtype,d,hkv,page,gap", [(BF16, 64, 2, 16, 0), (BF16, 128, 8, 64, 16), (F32, 128, 3, 32, 0), (F32, 64, 1, 256, 32), (BF16, 128, 1, 128, 0),
                                                  (BF16, 64, 40, 16, 0)])
def test_what_is_written_and_read_back(sla, handle, dtype, d, hkv, page, gap):
    """Every byte of every plane, twice over, and every value read back; sequences that were refused and rows of none stay as they are."""
    c, k, v, table = empty_cache(sla, hkv=hkv, page=page, d=d, dtype=dtype, gap=gap, width=7)
    want = [t.clone() for t in (k, v)]
    held = {s: 0 for s in range(6)}
    for step, (seq, new) in enumerate([([0, 3, 5], [33, 1, 40]), ([3, 0, 1], [1, 1, 0]), ([5, 2], [30, 17]), ([0, 1, 3], [1, 1, 1])]):
        T = sum(new)
        big = normal((T + 3, hkv + 1, d), dtype, 10 + step)
        kn, vn = big[:T, :hkv], normal((T + 3, hkv + 1, d), dtype, 20 + step)[:T, 1:]
        cu = cu_of(new)
        first = sla.sla_cache_extend(handle, c, cu, seq=U.device_ints(seq))
        assert first.tolist() == [held[s] for s in seq]
        sla.sla_cache_append(handle, c, cu, first, kn, vn, seq=U.device_ints(seq))
        tab, at = table.cpu().numpy(), 0
        for s, m in zip(seq, new):
            for r in range(m):
                p, t = int(tab[s, (held[s] + r) // page]), (held[s] + r) % page
                for pool, x, values in ((want[0], kn, False), (want[1], vn, True)):
                    row = Q.pack(*(y[:, None] for y in Q.quantise(x[at])), values)      # [hkv, bytes of a row]
                    pool[p, :, t * d // 2 : (t + 1) * d // 2] = row[:, : d // 2]
                    pool[p, :, page * d // 2 + t * d // 16 : page * d // 2 + (t + 1) * d // 16] = row[:, d // 2 :]
                at += 1
            held[s] += m
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
        ko, vo = sla.sla_cache_read(handle, c, cu, first, seq=U.device_ints(seq), n_new=T)
        assert torch.equal(ko.double(), Q.held(kn)) and torch.equal(vo.double(), Q.held(vn))
    # whole sequences head by head into a larger tensor, a refused one left out
    n = [held[0], 5, held[5]]
    out = torch.full((2, hkv + 1, sum(n) + 4, d), 7.0, dtype=dtype, device="cuda:0")
    ko, vo = (o[:hkv, : sum(n)].transpose(0, 1) for o in out)
    sla.sla_cache_read(handle, c, cu_of(n), U.device_ints([0, -1, 0]), seq=U.device_ints([0, 2, 5]), k_out=ko, v_out=vo)
    tab = table.cpu().numpy()
    for o, pool, values in ((out[0], k, False), (out[1], v, True)):
        at = 0
        for s, m in ((0, n[0]), (None, 5), (5, n[2])):
            if s is None:
                assert (o[:, at : at + m] == 7).all()
            else:
                pages = torch.from_numpy(tab[s, : -(-m // page)].astype(np.int64)).cuda()
                assert torch.equal(o[:hkv, at : at + m].double(), Q.unpack(pool[pages], page, d, values).transpose(0, 1).flatten(1, 2)[:, :m])
            at += m
        assert (o[hkv] == 7).all() and (o[:, at:] == 7).all()


def test_every_bf16_and_the_values_next_to_the_borders(sla, handle):
    """Groups with every finite bf16 as their largest; every code's border hit exactly, from a bit above and a bit below, in both types."""
    rows = []
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(BF16) if hasattr(torch, "uint16") else torch.arange(-32768, 32768, dtype=torch.int16).view(BF16)
    rows.append(every.float().view(-1, 1).expand(-1, 32) * torch.linspace(0, 1, 32).round(decimals=3))
    rows[0][:, 31] = every.float()
    m = torch.arange(16, 32, dtype=torch.float64)
    s = (m[:, None] * 2.0 ** torch.arange(-44, 36, 3, dtype=torch.float64)).reshape(-1)
    borders = (torch.arange(8, dtype=torch.float64) + 0.5) * s[:, None]                      # [.., 8], exact in fp32
    x = torch.cat([borders, -borders, borders * (1 + 2.0 ** -23), borders * (1 - 2.0 ** -24)], 1)
    x[:, 16 + 7] = borders[:, 7]                                                            # nothing above 7.5 s: the scale is s
    rows.append(x.float())
    rows.append(rows[1].to(BF16).float().clamp(max=3e38))
    x = torch.cat([r.reshape(-1, 32) for r in rows])
    x = torch.cat([x, torch.zeros((-len(x)) % 4, 32)])
    for dtype in (BF16, F32):
        new = x.to(dtype).view(-1, 1, 128).cuda()
        T = len(new)
        c, k, v, table = empty_cache(sla, n_pages=-(-T // 256), hkv=1, page=256, d=128, slots=1, width=-(-T // 256), dtype=dtype)
        cu = U.device_ints([0, T])
        first = sla.sla_cache_extend(handle, c, cu)
        sla.sla_cache_append(handle, c, cu, first, new, new)
        want = Q.held(new)
        nan = torch.isnan(want)
        for got in sla.sla_cache_read(handle, c, cu, n_new=T):
            assert torch.equal(torch.isnan(got), nan) and torch.equal(got.double()[~nan], want[~nan])


def test_groups_that_are_not_finite_or_too_large(sla, handle):
    """One such value makes its group NaN and no other.  (2^42 / 7.5 is below 2^40, 2^43 / 7.5 is not.)"""
    x = torch.ones(6, 2, 128, dtype=F32, device="cuda:0")
    x[0, 0, 3], x[1, 1, 64], x[2, 0, 127], x[3, 1, 40], x[4, 0, 0], x[5, 1, 100] = math.nan, math.inf, -math.inf, 2e38, -2.0 ** 42, 2.0 ** 43
    c, *_ = empty_cache(sla, hkv=2, d=128, dtype=F32)
    cu = U.device_ints([0, 6, 6, 6, 6, 6, 6])
    sla.sla_cache_append(handle, c, cu, sla.sla_cache_extend(handle, c, cu), x, x)
    bad = torch.zeros(6, 2, 4, dtype=torch.bool, device="cuda:0")
    bad[0, 0, 0] = bad[1, 1, 2] = bad[2, 0, 3] = bad[3, 1, 1] = bad[5, 1, 3] = True
    want = Q.held(x)
    for got in sla.sla_cache_read(handle, c, cu, n_new=6):
        assert torch.equal(torch.isnan(got).unflatten(-1, (4, 32)), bad[..., None].expand(-1, -1, -1, 32))
        assert torch.equal(got.double().nan_to_num(5.0), want.nan_to_num(5.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("token_major", [False, True])
def test_reading_other_caches(sla, handle, dtype, token_major):
    """sla_cache_read on caches in bf16 and fp32: the rows as they are."""
    hkv, page, d, n = 3, 32, 128, [70, 0, 33, 5]
    k, v = U.make_pools(12, hkv, page, d, dtype, token_major, 8)
    table = np.full((4, 4), -1)
    table[0, :3], table[2, :2], table[3, 0] = [7, 2, 11], [0, 5], 9
    c = sla.make_cache(k, v, U.device_ints(table), U.device_ints(n), U.device_ints(np.bincount(table[table >= 0], minlength=12)))
    lo, m = [3, 0, 31, 4], [67, 0, 2, 1]
    ko, vo = sla.sla_cache_read(handle, c, cu_of(m), U.device_ints(lo), n_new=70)
    for o, pool in ((ko, k), (vo, v)):
        at = 0
        for s in range(4):
            rows = torch.stack([pool[int(table[s, p // page]), :, p % page] for p in range(lo[s], lo[s] + m[s])]) if m[s] else o[:0]
            assert torch.equal(o[at : at + m[s]], rows)
            at += m[s]
    one, _ = sla.sla_cache_read(handle, c, None, U.device_ints([69, 0]), seq=U.device_ints([0, 2]))
    assert torch.equal(one[0], k[11, :, 5]) and torch.equal(one[1], k[0, :, 0])


@pytest.mark.parametrize("four", [False, True])
def test_positions_that_are_not_there_are_flagged_and_left(sla, four):
    h = sla.Handle(0, 1 << 26)
    if four:
        c, k, v, table = empty_cache(sla)
    else:
        k, v = U.make_pools(40, 2, 16, 64, BF16)
        table = U.device_ints(np.full((6, 20), -1))
        c = sla.make_cache(k, v, table, U.device_ints(np.zeros(6)), U.device_ints(np.zeros(40)))
    cu = U.device_ints([0, 20, 50])
    x = normal((50, 2, 64), BF16, 1)
    sla.sla_cache_append(h, c, cu, sla.sla_cache_extend(h, c, cu), x, x)
    want = Q.held(x).to(BF16) if four else x
    out = torch.full((44, 2, 64), 7.0, dtype=BF16, device="cuda:0")
    spare = out.clone()
    sla.sla_cache_read(h, c, U.device_ints([0, 12, 44]), U.device_ints([10, 0]), k_out=out, v_out=spare)
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    assert torch.equal(out[:10], want[10:20]) and (out[10:12] == 7).all() and torch.equal(out[12:42], want[20:]) and (out[42:] == 7).all()
    for bad_seq, bad_table in (([0, 9], None), ([0, 1], 10 ** 6), ([0, 1], -1)):
        if bad_table is not None:
            table[1, 0] = bad_table
        sla.sla_cache_read(h, c, cu, seq=U.device_ints(bad_seq), n_new=50)
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    sla.sla_cache_append(h, c, cu, U.device_ints([0, 0]), x, x)                    # into the page that is not there
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    sla.sla_cache_append(h, c, U.device_ints([0, 10 ** 6, -5]), U.device_ints([0, 0]), x, x)
    torch.cuda.synchronize()
    sla.sla_poll_status(h)
    h.close()


@pytest.mark.parametrize("gap", [0, 48])
def test_pages_are_forked_compacted_and_copied_whole(sla, handle, gap):
    """The bookkeeping against its model, and the planes' bytes with it."""
    c, k, v, table = empty_cache(sla, n_pages=30, hkv=3, page=32, d=64, width=6, gap=gap)
    m = U.Model(30, 32, 6, 6)
    cu = cu_of([40, 64, 100])
    x, y = normal((204, 3, 64), BF16, 1), normal((204, 3, 64), BF16, 2)
    sla.sla_cache_append(handle, c, cu, sla.sla_cache_extend(handle, c, cu, seq=U.device_ints([0, 1, 2])), x, y, seq=U.device_ints([0, 1, 2]))
    m.extend([0, 1, 2], [40, 64, 100])
    pairs = sla.sla_cache_fork(handle, c, U.device_ints([0, 2, 1]), U.device_ints([3, 4, 5]))
    want = m.fork([0, 2, 1], [3, 4, 5])
    assert np.array_equal(pairs.cpu().numpy(), want)
    sla.sla_cache_release(handle, c, U.device_ints([0, 1]))
    m.release([0, 1])
    before = k.clone(), v.clone()
    pairs = sla.sla_cache_compact(handle, c)
    want = m.compact()
    assert np.array_equal(pairs.cpu().numpy(), want) and np.array_equal(table.cpu().numpy(), m.table)
    moved = {int(b): int(a) for a, b in want.T if a >= 0}
    assert moved
    src = torch.tensor([moved.get(p, p) for p in range(30)], device="cuda:0")
    assert torch.equal(k, before[0][src]) and torch.equal(v, before[1][src])
    sla.sla_cache_copy(handle, c, U.device_ints([[1, -1], [29, 3]]))
    assert torch.equal(k[29], k[1]) and torch.equal(v[29], v[1])
    for slot, rows in ((3, slice(0, 40)), (4, slice(104, 204)), (5, slice(40, 104))):
        count = rows.stop - rows.start
        ko, vo = sla.sla_cache_read(handle, c, U.device_ints([0, count]), seq=U.device_ints([slot]), n_new=count)
        assert torch.equal(ko.double(), Q.held(x[rows])) and torch.equal(vo.double(), Q.held(y[rows]))


# ---- attention ------------------------------------------------------------------------------------------------------------------------


def build(sla, n, new, *, hkv=2, G=4, d=128, dtype=BF16, page=16, gap=0, seed=3, spare=3, size=1.0):
    """A cache of sequences of n tokens, their pages scattered; what no sequence owns has scales that are NaN."""
    rs = np.random.RandomState(seed)
    held = [-(-int(x) // page) for x in n]
    n_pages = sum(held) + spare
    k, v = planes(sla, n_pages, hkv, page, d, gap)
    order = rs.permutation(n_pages)
    table = np.full((len(n), max(held + [1]) + 1), -1, dtype=np.int32)
    at = 0
    for x, c in enumerate(held):
        table[x, :c] = order[at:at + c]
        at += c
    cache = sla.make_cache_q4(k, v, U.device_ints(table), U.device_ints(n), U.device_ints(np.bincount(table[table >= 0], minlength=n_pages)),
                              page_tokens=page, head_dim=d, dtype=dtype)
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, hkv * G, len(n), max(sum(n), 1)))
    if sum(n):
        kn, vn = (normal((sum(n), hkv, d), dtype, seed + e, 0.4) * size for e in (1, 2))
        sla.sla_cache_append(h, cache, cu_of(n), U.device_ints(np.zeros(len(n))), kn, vn)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()
    q = normal((int(sum(new)), hkv * G, d), dtype, seed + 7, 0.1)
    return cache, k, v, table, q, cu_of(new)


def reference(q, k, v, table, n, new, G, window, scale, page):
    """attention_reference over the values that the planes stand for.

    A bound beside U.tolerances: codes of bf16 calls are 2^-133 as large as they are in their products and weights 2^78 times as large, so that
    a sum in fp32, which is cut at 2^-149 with each of its 16 keys or fewer, is off by 2^-149 2^(133 - 78) = 2^-94 each time.  (Where the keys of
    large weight have codes of zero in a dimension, the result there is as small.)  The weights' rounding, 2^-8 of sum p |v|, makes 2^-94 of 2^-86."""
    d = q.shape[-1]
    kk, vv = Q.unpack(k, page, d, False), Q.unpack(v, page, d, True)
    out, lse, mag, dot, keys = U.attention_reference(q, kk, vv, table, n, new, G, window, scale, page)
    return out, lse, mag + keys[:, None, None] * 2.0 ** -86 if q.dtype == BF16 else mag, dot, keys


def run(sla, handle, n, new, window=0, scale=None, max_new=None, prep=None, **kw):
    cache, k, v, table, q, cu = build(sla, n, new, **kw)
    if prep:
        prep(k, v, table, q)
    out, lse = sla.sla_paged_attention(handle, q, cache, cu, window=window, softmax_scale=scale, max_new=max(new) if max_new is None else max_new)
    torch.cuda.synchronize()
    s = 1 / math.sqrt(q.shape[-1]) if scale is None else scale
    ref = reference(q, k, v, table, n, new, kw.get("G", 4), window, s, kw.get("page", 16))
    U.check_attention(out, lse, ref, q.dtype)
    return out, lse, ref


SINGLE = ([1, 2, 15, 16, 17, 0, 63, 64, 65, 700], [1] * 10)       # one token each, an empty sequence among them
CHUNKS = ([40, 5, 0, 129, 300, 64, 513], [40, 0, 0, 1, 77, 64, 200])   # whole prompts, ends of prompts, nothing new
TYPES = [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("lens", [SINGLE, CHUNKS], ids=["single", "chunks"])
def test_attention_types(sla, handle, dtype, d, lens):
    run(sla, handle, *lens, dtype=dtype, d=d)


@pytest.mark.parametrize("hkv,G", [(1, 1), (3, 2), (2, 3), (1, 5), (2, 7), (1, 8), (1, 12), (2, 16)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_groups(sla, handle, hkv, G, dtype):
    run(sla, handle, *SINGLE, hkv=hkv, G=G, dtype=dtype)
    run(sla, handle, *CHUNKS, hkv=hkv, G=G, dtype=dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("gap", [0, 16])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_pages_and_strides(sla, handle, page, gap, d):
    run(sla, handle, *SINGLE, page=page, gap=gap, d=d)
    run(sla, handle, *CHUNKS, page=page, gap=gap, hkv=3, d=d)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 129, 400, 5000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_window(sla, handle, window, dtype):
    run(sla, handle, *SINGLE, window=window, dtype=dtype)
    run(sla, handle, *CHUNKS, window=window, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_keys(sla, handle, dtype):
    """Sequences shorter than their new tokens: the first rows see nothing."""
    out, lse, _ = run(sla, handle, [3, 0, 20, 1], [5, 4, 20, 3], dtype=dtype)
    assert (out[:2] == 0).all() and (out[5:9] == 0).all()
    run(sla, handle, [3, 0, 20, 1], [5, 4, 20, 3], dtype=dtype, window=2 ** 31 - 1)
    run(sla, handle, [0, 0], [1, 1], dtype=dtype)
    run(sla, handle, [0, 7], [1, 0], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G", [4, 16])
def test_long_sequences_are_cut_and_joined(sla, handle, dtype, G):
    run(sla, handle, [20000, 33, 9001], [1, 1, 1], G=G, dtype=dtype, page=64)
    run(sla, handle, [20000, 33, 9001], [3, 2, 1], G=G, dtype=dtype, page=64)
    run(sla, handle, [6000], [70], G=G, dtype=dtype, page=64)
    run(sla, handle, [6000, 4000], [70, 130], G=G, dtype=dtype, page=32, window=900)
    run(sla, handle, [20011, 17000], [150, 40], G=G, dtype=dtype, page=64, window=16900)


FEW = [(1, 16), (1, 9), (2, 8), (2, 3), (3, 5), (4, 4), (4, 2), (5, 3), (7, 2), (8, 2)]   # heads of a group x new tokens <= 16


@pytest.mark.parametrize("G,new", FEW)
@pytest.mark.parametrize("dtype,d", TYPES)
def test_few_new_tokens(sla, handle, G, new, dtype, d):
    """Ragged counts, none, fewer keys than tokens, a long sequence; and the same through the kernel of chunks."""
    n = [1, 2, 15, 16, 17, 0, 63, 64, 65, 700, 3, 40, 9001]
    c = [(i * 5 + 2) % (new + 1) for i in range(len(n))]
    c[2] = c[5] = c[10] = c[-1] = new
    for window in (0, 1, 7, 100):
        out, lse, _ = run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=window, max_new=new)
    one, one_lse, _ = run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=100, max_new=400)
    assert torch.allclose(out.float(), one.float(), atol=0.02) and torch.equal(lse.isinf(), one_lse.isinf())


@pytest.mark.parametrize("G,new", [(1, 2), (1, 3), (1, 4), (2, 2), (1, 7), (2, 4)])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_few_rows(sla, handle, G, new, dtype, d):
    """Heads of a group x new tokens <= 8, four and fewer among them; with groups that are NaN where only some rows look."""
    n = [1, 2, 31, 32, 33, 0, 64, 700, 9001]
    c = [(i * 5 + 2) % (new + 1) for i in range(len(n))]
    c[1] = c[2] = c[5] = c[-1] = new
    for window in (0, 1, 31, 100):
        def prep(k, v, table, q):
            at = n[-1] - new // 2 - 1
            spoil(v, int(table[-1, at // 16]), 1, at % 16, 16, d, 5)
            spoil(v, int(table[7, 43]), 0, 8, 16, d, d - 1)
        run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=window, max_new=new)
        run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=window, max_new=new, prep=prep)


def spoil(pool, page_of, g, t, page, d, dim):
    """The scale of dimension `dim` of row t of a plane becomes NaN."""
    at = page * d // 2 + t * (d // 16) + dim // 32 * 2
    pool[page_of, g, at], pool[page_of, g, at + 1] = 0xC0, 0x7F


@pytest.mark.parametrize("G,new", [(1, 16), (2, 3), (4, 4), (8, 2), (4, 1), (12, 1), (4, 70), (16, 9), (1, 200)])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_groups_that_are_nan_reach_the_rows_that_see_them(sla, handle, G, new, dtype, d):
    """At positions that only some of the new tokens see, at either end of the window: the groups' dimensions of those rows, no others."""
    n = [400, 300]
    for window in (0, 40):
        for back in {0, new // 2, new - 1}:
            for at in (n[0] - 1 - back, n[0] - window - back):
                if at >= n[0]:
                    continue

                def prep(k, v, table, q):
                    spoil(v, int(table[0, at // 16]), 1, at % 16, 16, d, 5)
                    spoil(v, int(table[0, at // 16]), 0, at % 16, 16, d, d - 1)
                run(sla, handle, n, [new, min(new, 2)], dtype=dtype, d=d, G=G, window=window, prep=prep)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("new", [1, 3, 20, 200])
def test_cut_units_and_groups_that_are_nan(sla, handle, dtype, d, new):
    n = 4000 + 37 * new
    for window in (0, 2500):
        for at in (n - 1, n - new, n - 1 - new // 2, n - window - new // 2, n - 130):
            if at >= n:
                continue

            def prep(k, v, table, q):
                spoil(v, int(table[0, at // 16]), 1, at % 16, 16, d, d - 3)
                spoil(v, int(table[1, 10]), 0, 3, 16, d, 2)
            run(sla, handle, [n, 350], [new, new], dtype=dtype, d=d, window=window, prep=prep)


@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 2), (BF16, 150), (F32, 1), (F32, 150)])
def test_keys_that_are_nan(sla, handle, dtype, new):
    n, at = [400, 300], 399 if new == 1 else 398 if new == 2 else 330
    cache, k, v, table, q, cu = build(sla, n, [new, new], dtype=dtype)
    clean, clean_lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=new)
    spoil(k, int(table[0, at // 16]), 1, at % 16, 16, 128, 5)
    out, lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=new)
    sees = n[0] - new + torch.arange(new, device=out.device) >= at
    assert torch.equal(out[:new][~sees], clean[:new][~sees]) and torch.equal(out[new:], clean[new:])
    assert torch.equal(out[:, :4], clean[:, :4]) and torch.equal(lse[:, :4], clean_lse[:, :4])
    assert torch.isnan(out[:new][sees][:, 4:]).all() and torch.isnan(lse[:new][sees][:, 4:]).all()


@pytest.mark.parametrize("dtype,new", [(BF16, [1, 1]), (BF16, [3, 2]), (BF16, [60, 1]), (F32, [60, 1])])
def test_scales_of_the_softmax(sla, handle, dtype, new):
    for scale in (3.0, 0.0, -0.5):
        run(sla, handle, [500, 31], new, dtype=dtype, scale=scale)


@pytest.mark.parametrize("dtype,new", [(BF16, [1, 1]), (BF16, [60, 1]), (F32, [3, 1])])
@pytest.mark.parametrize("size", [2.0 ** -18, 2.0 ** 18, 2.0 ** 35])
def test_small_and_large_keys_and_values(sla, handle, dtype, new, size):
    """Keys and values of other sizes, the softmax's scale to match."""
    run(sla, handle, [500, 31], new, dtype=dtype, size=size, scale=128 ** -0.5 / size)


@pytest.mark.parametrize("power", [-60, -30, 30, 60])
@pytest.mark.parametrize("new", [[1, 1], [60, 1]])
def test_small_and_large_queries(sla, handle, power, new):
    def prep(k, v, table, q):
        q.mul_(2.0 ** power)
    run(sla, handle, [500, 31], new, scale=128 ** -0.5 * 2.0 ** -power, prep=prep)


@pytest.mark.parametrize("power,scale", [(100, None), (113, None), (120, None), (124, None), (-110, 2.0 ** 63)])
@pytest.mark.parametrize("new,G", [([1, 1], 2), ([1, 1], 4), ([1, 1], 8), ([3, 1], 4), ([60, 1], 4)])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_next_to_the_ends_of_bf16(sla, handle, power, scale, new, G, d):
    """Every finite query has its answer, whatever kernel the call runs on.  Powers of two move no rounding but at the small end: fp32 sums of
    products, which may be 2^-48 as large as they are, end at 2^-149, 2^-38 of a logit under the largest scale, beside which 2^-20 is allowed."""
    def prep(k, v, table, q):
        q.clamp_(-7.5, 7.5).mul_(2.0 ** power)
    run(sla, handle, [500, 31], new, G=G, d=d, scale=d ** -0.5 * 2.0 ** -power if scale is None else scale, prep=prep)


@pytest.mark.parametrize("power,scale", [(60, 2.0 ** 63), (124, 1.0), (124, -1.0), (126, 2.0 ** 63), (0, 2.0 ** 63)])
@pytest.mark.parametrize("new", [[1, 1], [3, 1], [60, 1]])
def test_keys_of_zero_under_large_queries_and_scales(sla, handle, power, scale, new):
    """Logits that are zero stay zero, whatever they are multiplied by: every key weighs the same."""
    def prep(k, v, table, q):
        k[:, :, : 16 * 64] = 0                                    # codes
        q.clamp_(-2, 2).mul_(2.0 ** (power - 1))
    run(sla, handle, [500, 31], new, scale=scale, prep=prep)


@pytest.mark.parametrize("power", [20, 60, 100, 125])
@pytest.mark.parametrize("new", [[1, 1], [3, 1], [60, 1]])
def test_a_large_dimension_whose_codes_are_zero(sla, handle, power, new):
    """The others decide, however much smaller they are.  (Sums of codes' products, 2^-133 as large as they are beside a query of 2^125, end at
    2^-149: 2^-16 times a key's scale, here about 1/2, and the softmax's, 2^-3.5, each of the 6 to 24 times that something is added, 2^-16 in
    all.  The bound allows 2^-16 of the sum of the products' magnitudes, which are about 100 2^-3.5 here.)"""
    def prep(k, v, table, q):
        b = k[:, :, : 16 * 64].unflatten(-1, (16, 4, 4, 4))       # row, piece of eight, group, bytes
        b[:, :, :, :, 0] = 0
        q[..., 5] = 2.0 ** power
    run(sla, handle, [500, 31], new, prep=prep)


@pytest.mark.parametrize("dtype,new", [(BF16, [1, 1]), (BF16, [3, 1]), (BF16, [60, 1]), (F32, [1, 1]), (F32, [60, 1])])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 35])
def test_logits_next_to_the_largest_allowed(sla, handle, dtype, new, size):
    """Logits up to 2^23, of either sign: results lie among the values, whatever these are, and the sums' logarithms are right.  (D 2^-23 of the
    sum of a logit's magnitudes, as everywhere; logits times log2 e are rounded to 2 each, a maximum, a weight's exponent and the logarithm
    at the end: 8 in all.)"""
    n = [500, 31]
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, size=size)
    ref = reference(q, k, v, table, n, new, 4, 0, 1.0, 16)
    scale = 2.0 ** 23 / ref[3].max().item()                    # (no logit passes the sum of its products' magnitudes)
    out, lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=max(new), softmax_scale=scale)
    ref = reference(q, k, v, table, n, new, 4, 0, scale, 16)
    assert torch.isfinite(out).all()
    assert out.double().abs().max() <= Q.unpack(v, 16, 128, True).nan_to_num(0).abs().max() * (1 + 2.0 ** -8)
    assert ((lse.double() - ref[1]).abs() <= 128 * 2.0 ** -23 * ref[3] + 8).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_queries_slots_and_shared_pages(sla, handle, dtype):
    n, new = [100, 64, 250], [3, 1, 40]
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype)
    table[1] = table[2]                     # slot 1 shares slot 2's first pages
    cache.tensors[2].copy_(U.device_ints(table))
    for order, most in (([2, 0, 1], 40), ([0, 1], 3)):
        rows = torch.cat([torch.arange(int(cu[s]), int(cu[s + 1])) for s in order])
        big = torch.zeros(len(rows), 3, 8, 128, dtype=dtype, device="cuda:0")
        big[:, 1] = q[rows.cuda()]
        out = torch.full_like(big, 7.0)
        o, lse = sla.sla_paged_attention(handle, big[:, 1], cache, cu_of([new[s] for s in order]), seq=U.device_ints(order), max_new=most, out=out[:, 1])
        ref = reference(big[:, 1], k, v, table[order], [n[s] for s in order], [new[s] for s in order], 4, 0, 128 ** -0.5, 16)
        U.check_attention(o, lse, ref, dtype)
        assert (out[:, 0] == 7).all() and (out[:, 2] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 12])
def test_queries_with_tokens_inside_heads(sla, handle, dtype, G):
    for n, new in (SINGLE, CHUNKS, ([300, 41], [300, 41])):
        cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, G=G)
        big = torch.full((q.shape[1], q.shape[0], 136), 7.0, dtype=dtype, device="cuda:0")[..., 8:]   # rows at any 16 bytes
        q = big.copy_(q.transpose(0, 1)).transpose(0, 1)
        out, lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=max(new))
        assert out.stride() == q.stride()
        U.check_attention(out, lse, reference(q, k, v, table, n, new, G, 0, 128 ** -0.5, 16), dtype)


@pytest.mark.parametrize("dtype,n_seqs,new,G,d", [(F32, 300, 2, 8, 128), (BF16, 1010, 1, 16, 128), (BF16, 1030, 4, 4, 64), (BF16, 2500, 1, 2, 64)])
def test_many_sequences(sla, handle, dtype, n_seqs, new, G, d):
    rs = np.random.RandomState(n_seqs)
    n = rs.randint(0, 40, n_seqs)
    c = np.minimum(n, rs.randint(0, new + 1, n_seqs)) if new > 1 else np.ones(n_seqs, dtype=int)
    run(sla, handle, n.tolist(), c.tolist(), dtype=dtype, hkv=1, G=G, d=d, max_new=new)


@pytest.mark.parametrize("n_seqs,new,G,d", [(1030, 4, 4, 128), (2500, 1, 2, 64), (1025, 2, 2, 128)])
def test_many_sequences_in_fp32(sla, handle, n_seqs, new, G, d):
    test_many_sequences(sla, handle, F32, n_seqs, new, G, d)


def test_offsets_above_2_to_32(sla, handle):
    """Pools of more than 2^32 bytes: the pages of the sequences lie behind them."""
    n_pages, hkv, page, d = 120000, 8, 64, 128
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("not enough device memory")
    k, v = (torch.empty(n_pages, hkv, sla.q4_plane_bytes(page, d), dtype=torch.uint8, device="cuda:0") for _ in range(2))
    table = np.full((2, 4), -1, dtype=np.int32)
    table[0, :3], table[1, :1] = [119999, 119900, 40], [119950]
    n = [150, 40]
    cache = sla.make_cache_q4(k, v, U.device_ints(table), U.device_ints(n), U.device_ints(np.zeros(n_pages)), page_tokens=page, head_dim=d)
    kn, vn = normal((190, hkv, d), BF16, 1), normal((190, hkv, d), BF16, 2)
    sla.sla_cache_append(handle, cache, cu_of(n), U.device_ints([0, 0]), kn, vn)
    ko, vo = sla.sla_cache_read(handle, cache, cu_of(n), n_new=190)
    assert torch.equal(ko.double(), Q.held(kn)) and torch.equal(vo.double(), Q.held(vn))
    used, small = sorted(table[table >= 0].tolist()), np.full_like(table, -1)
    for i, p in enumerate(used):
        small[table == p] = i
    for new in ([1, 1], [100, 40]):
        q = normal((sum(new), 16, d), BF16, 3, 0.1)
        out, lse = sla.sla_paged_attention(handle, q, cache, cu_of(new), max_new=max(new))
        U.check_attention(out, lse, reference(q, k[used], v[used], small, n, new, 2, 0, d ** -0.5, page), BF16)
    sla.sla_cache_copy(handle, cache, U.device_ints([[119999], [119998]]))
    assert torch.equal(k[119998], k[119999]) and torch.equal(v[119998], v[119999])
    del k, v, cache
    torch.cuda.empty_cache()


def test_same_result_every_time_on_any_stream(sla, handle):
    for n, new in (([9000, 100, 4000], [1, 50, 300]), ([9000, 100, 4000], [1, 1, 1])):
        cache, k, v, table, q, cu = build(sla, n, new, page=64)
        a = sla.sla_paged_attention(handle, q, cache, cu, max_new=max(new))
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        for stream in (torch.cuda.current_stream(), st, torch.cuda.current_stream()):
            with torch.cuda.stream(stream):
                b = sla.sla_paged_attention(handle, q, cache, cu, max_new=max(new))
            stream.synchronize()
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_what_is_out_of_range_is_flagged_and_not_followed(sla):
    h = sla.Handle(0, 1 << 28)
    for new in ([1, 1], [3, 2], [40, 33]):
        cache, k, v, table, q, cu = build(sla, [100, 60], new)
        sla.sla_paged_attention(h, q, cache, cu, max_new=max(new), seq=U.device_ints([0, 9]))
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
        bad = table.copy()
        for page in (10 ** 6, -1):
            bad[0, 1] = page
            cache.tensors[2].copy_(U.device_ints(bad))
            sla.sla_paged_attention(h, q, cache, cu, max_new=max(new))
            assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
        cache.tensors[2].copy_(U.device_ints(np.where(table < 0, 0, table)))
        cache.tensors[3].copy_(U.device_ints([10 ** 6, 60]))
        sla.sla_paged_attention(h, q, cache, cu, max_new=max(new))
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
        cache.tensors[3].copy_(U.device_ints([100, 60]))
        sla.sla_paged_attention(h, q, cache, U.device_ints([0, 10 ** 6, -5]), max_new=max(new))
        torch.cuda.synchronize()
        sla.sla_poll_status(h)
    h.close()


@pytest.mark.parametrize("max_new", [1, 2, 3])
def test_more_new_tokens_than_max_new_are_flagged(sla, max_new):
    h = sla.Handle(0, 1 << 28)
    cache, k, v, table, q, cu = build(sla, [100, 60], [2 * max_new, 0])
    out = torch.full((q.shape[0] + 8, *q.shape[1:]), 7.0, dtype=BF16, device="cuda:0")
    sla.sla_paged_attention(h, q, cache, cu, max_new=max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) in (sla.SLA_OK, sla.SLA_ERR_DEVICE_INDEX)
    assert (out[q.shape[0]:] == 7).all()
    sla.sla_paged_attention(h, q, cache, cu, max_new=2 * max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G,max_new", [(1, 1), (1, 4), (4, 1), (4, 2), (4, 4), (2, 3), (8, 2), (16, 1)])
def test_more_few_new_tokens_than_max_new_are_always_flagged(sla, dtype, d, G, max_new):
    """On the kernels of few rows, four, eight and sixteen of them; the sequence of max_new tokens beside it has its results."""
    h = sla.Handle(0, 1 << 28)
    n, new = [100, 60, 10], [2 * max_new, max_new, 0]
    cache, k, v, table, q, cu = build(sla, n, new, G=G, dtype=dtype, d=d)
    out = torch.full((q.shape[0] + 8, *q.shape[1:]), 7.0, dtype=dtype, device="cuda:0")
    o, lse = sla.sla_paged_attention(h, q, cache, cu, max_new=max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    assert (out[q.shape[0]:] == 7).all()
    ref = reference(q, k, v, table, n, new, G, 0, d ** -0.5, 16)
    U.check_attention(o[2 * max_new:], lse[2 * max_new:], [t[2 * max_new:] for t in ref], dtype)
    h.close()


@pytest.mark.parametrize("dtype,d,hkv,G", [(BF16, 128, 8, 4), (BF16, 64, 2, 16), (BF16, 128, 2, 1), (F32, 64, 1, 16)])
@pytest.mark.parametrize("n_seqs,n_new", [(4, 4), (3, 40), (40, 300)])
def test_a_workspace_of_the_size_asked_for_is_enough(sla, dtype, d, hkv, G, n_seqs, n_new):
    new = [n_new // n_seqs] * n_seqs
    new[0] += n_new - sum(new)
    n = [30 + x for x in new]
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, d=d, hkv=hkv, G=G)
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, hkv * G, n_seqs, n_new))
    sla.sla_set_debug_canaries(h, True)
    for scale in (None, -0.1):
        ref = reference(q, k, v, table, n, new, G, 0, d ** -0.5 if scale is None else scale, 16)
        for bound in sorted({max(new), max(new) + 1, 16, 17, 64, 65, n_new, n_new + 1, 2 ** 31 - 1}):
            if bound >= max(new):
                U.check_attention(*sla.sla_paged_attention(h, q, cache, cu, max_new=bound, softmax_scale=scale), ref, dtype)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


def test_refusals(sla, handle):
    import ctypes as C
    cache, k, v, table, q, cu = build(sla, [30, 50], [1, 1])
    first, new = U.device_ints([0, 0]), normal((2, 2, 128), BF16, 1)
    with pytest.raises(sla.SlaError) as e:
        sla.sla_paged_decode_step(handle, q, q, cache, sla.make_params(4, 0))
    assert e.value.status == -2
    for bad in (dict(window=-1), dict(softmax_scale=math.nan), dict(max_new=0), dict(softmax_scale=2.0 ** 64), dict(softmax_scale=-math.inf)):
        with pytest.raises(sla.SlaError):
            sla.sla_paged_attention(handle, q, cache, cu, **bad)
    with pytest.raises(TypeError):
        sla.sla_paged_attention(handle, q.half(), cache, cu)
    for call in (lambda: sla.sla_paged_attention(handle, q.float(), cache, cu), lambda: sla.sla_cache_append(handle, cache, None, first, new.float(), new.float()),
                 lambda: sla.sla_cache_append(handle, cache, None, first[:1], new, new), lambda: sla.sla_cache_read(handle, cache, cu, first[:1], n_new=2),
                 lambda: sla.sla_cache_read(handle, cache, None, first, k_out=new, v_out=new.float())):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(2, 2, 2, 132, dtype=BF16, device="cuda:0")
    for ko, vo in ((wide[0, ..., 4:], wide[1, ..., 4:]), (wide[0, ..., :128], wide[1, ..., :128]),   # 8 bytes off; rows of 132
                   (new[:1].expand(2, 2, 128), new[:1].expand(2, 2, 128))):                          # rows that lie over one another
        with pytest.raises(sla.SlaError):
            sla.sla_cache_read(handle, cache, None, first, k_out=ko, v_out=vo)
    b = sla.sla_batch_t(2, 2, 1, 0, None, None)
    lib, ca, ba = sla.load_library(), C.addressof(cache), C.addressof(b)
    assert lib.sla_cache_read(handle.ptr, ca, ba, None, None, new.data_ptr(), 256, 128, None) == -1
    assert lib.sla_cache_read(handle.ptr, ca, ba, None, new.data_ptr(), new.data_ptr(), -8, 128, None) == -1
    assert lib.sla_cache_read(handle.ptr, ca, None, None, new.data_ptr(), new.data_ptr(), 256, 128, None) == -1
    for field, bad in (("stride_t", 64), ("stride_h", 16), ("stride_page", 100), ("page_tokens", 24)):
        was = getattr(cache, field)
        setattr(cache, field, bad)
        assert lib.sla_cache_read(handle.ptr, ca, ba, None, new.data_ptr(), new.data_ptr(), 256, 128, None) == -1, field
        assert lib.sla_cache_append(handle.ptr, ca, ba, first.data_ptr(), new.data_ptr(), new.data_ptr(), 256, 128, None) == -1, field
        setattr(cache, field, was)
    with pytest.raises(ValueError):
        from paper_2601_18401_b200.paged import PagedCache
        PagedCache(8, 2, 64, n_q_heads=8, n_kv_heads=2, four_bits=True, params=sla.make_params(4, 0))
    none = sla.sla_cache_read(handle, cache, U.device_ints([0, 0, 0]), first, n_new=0)
    assert none[0].shape == (0, 2, 128)


@pytest.mark.parametrize("four", [False, True])
def test_rows_read_that_would_lie_over_one_another(sla, handle, four):
    """Refused, and nothing is written; keys and values that share a tensor without meeting are read as any others."""
    d = 64
    if four:
        c, *_ = empty_cache(sla, d=d)
    else:
        k, v = U.make_pools(40, 2, 16, d, BF16)
        c = sla.make_cache(k, v, U.device_ints(np.full((6, 20), -1)), U.device_ints(np.zeros(6)), U.device_ints(np.zeros(40)))
    cu, x, y = U.device_ints([0, 5, 5, 5, 5, 5, 5]), normal((5, 2, d), BF16, 1), normal((5, 2, d), BF16, 2)
    sla.sla_cache_append(handle, c, cu, sla.sla_cache_extend(handle, c, cu), x, y)
    want = [Q.held(t) if four else t.double() for t in (x, y)]
    flat = torch.full((4000,), 7.0, dtype=BF16, device="cuda:0")

    def rows(at, s_t, s_h, T=5, H=2):
        return flat[at:].as_strided((T, H, d), (s_t, s_h, 1))
    for ko, vo in ((rows(0, 64, 64), rows(2000, 64, 64)),            # the second head of a row is the first of the next
                   (rows(0, 72, 136), rows(2000, 72, 136)),          # .. of the next but one, in part
                   (rows(0, 128, 64), rows(0, 128, 64)),             # keys and values in one place
                   (rows(0, 256, 64), rows(64, 256, 64)),            # values over the keys' second head
                   (rows(568, 128, 64), rows(0, 128, 64))):          # keys behind the values' start
        with pytest.raises(sla.SlaError) as e:
            sla.sla_cache_read(handle, c, cu, k_out=ko, v_out=vo)
        assert e.value.status == -1 and (flat == 7).all()
    for ko, vo in ((rows(0, 256, 64), rows(128, 256, 64)),           # token by token: keys, then values
                   (rows(0, 256, 128), rows(64, 256, 128)),          # head by head
                   (rows(0, 192, 128), rows(1600, 192, 128)),        # heads of one token between the next token's: 0, 128, 192, 320, ..
                   (rows(0, 64, 320), rows(640, 64, 320))):
        flat.fill_(7.0)
        for o, w in zip(sla.sla_cache_read(handle, c, cu, k_out=ko, v_out=vo), want):
            assert torch.equal(o.double(), w)
        assert (flat == 7).sum() == 4000 - 2 * 5 * 2 * d + sum((w == 7).sum() for w in want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,T,G", [((1 << 20) + 777, 2400, 16), (1 << 22, 1, 4), (1 << 21, 2, 8), (600000, 700, 1)])
def test_long_sums_of_values_of_one_sign(sla, d, n, T, G):
    """Hundreds of thousands of keys of like weight in a range.  Pages that are the same 64 again and again, so that a key's weight counts as
    often as a row sees its page.  Bounds as for bf16: each weight and the result rounded to 2^-9 of the value and more, 4096 sums in
    TMEM cut by 2^-23 each, the tiles' sums in fp32 2^-24 each."""
    page, n_pages = 256, 64
    k, v = planes(sla, n_pages, 1, page, d)
    width = -(-n // page)
    table = (np.arange(width) % n_pages).astype(np.int32)[None]
    ints = [U.device_ints(table), U.device_ints([n_pages * page]), U.device_ints(np.zeros(n_pages))]
    cache = sla.make_cache_q4(k, v, *ints, page_tokens=page, head_dim=d)
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, G, 1, n_pages * page))
    sla.sla_cache_append(h, cache, U.device_ints([0, n_pages * page]), U.device_ints([0]), normal((n_pages * page, 1, d), BF16, 1, 0.2),
                         normal((n_pages * page, 1, d), BF16, 2, 0.2).abs())
    ints[1].fill_(n)
    q = normal((T, G, d), BF16, 3, 0.1)
    sla.sla_set_debug_canaries(h, True)
    out, lse = sla.sla_paged_attention(h, q, cache, None if T == 1 else U.device_ints([0, T]))
    assert sla.sla_poll_status(h) == sla.SLA_OK
    kk, vv = (Q.unpack(t[:, 0], page, d, values).reshape(-1, d) for t, values in ((k, False), (v, True)))
    at = torch.arange(len(kk), device="cuda:0")
    tol = 2.0 ** -8 + 4096 * 2.0 ** -23 + 2 * (n / 128) * 2.0 ** -24
    for r in {0, T // 2, T - 1}:
        seen = n - T + r + 1
        times = (seen // len(kk) + (at < seen % len(kk))).double()
        z = q[r].double() @ kk.T * d ** -0.5
        w = torch.exp(z) * times
        want = (w @ vv) / w.sum(-1, keepdim=True)
        assert ((out[r].double() - want).abs() <= tol * want + 2.0 ** -40).all()
        assert ((lse[r].double() - w.sum(-1).log()).abs() <= tol).all()
    h.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 70000])
def test_groups_that_are_nan_in_long_ranges(sla, handle, d, window):
    """Segments of more tiles than one sum in TMEM has, a group that is NaN near the rows' own keys and at the window's beginning."""
    n, new = 300000, 300
    for at in (n - 100, n - 400, n - window - 100 if window else 70001):
        def prep(k, v, table, q):
            spoil(v, int(table[0, at // 64]), 1, at % 64, 64, d, 5)
        cache, k, v, table, q, cu = build(sla, [n], [new], d=d, page=64, G=2)
        clean, clean_lse = sla.sla_paged_attention(handle, q, cache, cu, window=window)
        prep(k, v, table, q)
        out, lse = sla.sla_paged_attention(handle, q, cache, cu, window=window)
        pos = torch.arange(n - new, n, device="cuda:0")
        sees = (pos >= at) & ((pos - at < window) if window else True)
        want = clean.clone()
        want[sees, 2:, :32] = math.nan
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(9.0), want.nan_to_num(9.0)) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("d", [64, 128])
def test_after_a_wait_that_ran_out_no_row_is_written(sla, d):
    h = sla.Handle(0, 1 << 28)
    cache, k, v, table, q, cu = build(sla, [9000, 4000, 2500], [70, 300, 129], d=d, page=64)
    want = sla.sla_paged_attention(h, q, cache, cu, max_new=300)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda:0")
    sla.sla_selftest_paged_expiry(h, True)
    sla.sla_paged_attention(h, q, cache, cu, max_new=300, out=out, lse=lse)
    sla.sla_selftest_paged_expiry(h, False)
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_TIMEOUT
    assert (out == 7).all() and (lse == 7).all()
    again = sla.sla_paged_attention(h, q, cache, cu, max_new=300)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    h.close()


def test_two_streams_at_once(sla):
    """Two handles over one cache, each on its own stream, at the same time."""
    n, new = [9000, 100, 4000], [40, 50, 300]
    cache, k, v, table, q, cu = build(sla, n, new, page=64)
    q1, cu1 = q[:3].contiguous(), cu_of([1, 1, 1])
    hs = [sla.Handle(0, sla.sla_paged_workspace_bytes(cache, 8, 3, 390)) for _ in range(2)]
    want = [sla.sla_paged_attention(hs[0], q, cache, cu, max_new=300), sla.sla_paged_attention(hs[0], q1, cache, cu1, max_new=1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for x, (qq, cc, m) in enumerate(((q, cu, 300), (q1, cu1, 1))):
            with torch.cuda.stream(streams[x]):
                got[x].append(sla.sla_paged_attention(hs[x], qq, cache, cc, max_new=m))
    torch.cuda.synchronize()
    for x in range(2):
        for o, l in got[x]:
            assert torch.equal(o, want[x][0]) and torch.equal(l, want[x][1])
        assert sla.sla_poll_status(hs[x]) == sla.SLA_OK
        hs[x].close()


def test_rows_that_no_sequence_has_stay_as_they_are(sla, handle):
    """Tensors with more rows than cu_new names: attention, reading and appending leave the rest alone."""
    cache, k, v, table, q, cu = build(sla, [300, 40], [70, 3])
    for new, most in (([70, 3], 70), ([1, 1], 1), ([3, 2], 3)):
        T = sum(new) + 9
        qq = normal((T, 8, 128), BF16, 5, 0.1)
        out, lse = torch.full_like(qq, 7.0), torch.full((T, 8), 7.0, device="cuda:0")
        sla.sla_paged_attention(handle, qq, cache, cu_of(new), max_new=max(most, -(-T // 2)), out=out, lse=lse)
        assert (out[T - 9:] == 7).all() and (lse[T - 9:] == 7).all() and not (out[: T - 9] == 7).all()
        ko = torch.full((T, 2, 128), 7.0, dtype=BF16, device="cuda:0")
        vo = ko.clone()
        sla.sla_cache_read(handle, cache, cu_of(new), k_out=ko, v_out=vo)
        assert (ko[T - 9:] == 7).all() and (vo[T - 9:] == 7).all()
        before = k.clone(), v.clone()
        sla.sla_cache_append(handle, cache, U.device_ints([0, 0, 0]), U.device_ints([5, 5]), ko, vo)
        assert torch.equal(k, before[0]) and torch.equal(v, before[1])


# ---- together -------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_serving_from_two_layers(sla, dtype):
    """Prompts in chunks, forks, steps of one token, an end, compaction, in two layers that share a table: every output against 64 bits
    over what the cache holds, which is what was appended, rounded."""
    from paper_2601_18401_b200.paged import PagedCache
    shape = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=32, dtype=dtype, max_new=300, four_bits=True)
    a = PagedCache(40, 6, 500, **shape)
    layers = [a, PagedCache(40, 6, 500, share=a, **shape)]
    rows = [{s: [torch.zeros(0, 2, 64, device="cuda:0", dtype=torch.float64)] * 2 for s in range(6)} for _ in layers]
    seed = iter(range(1000, 9000))

    def step(seq, new, refused=()):
        T = sum(new)
        cu = cu_of(new)
        first = a.extend(cu, seq=U.device_ints(seq))
        assert [x for x, f in enumerate(first.tolist()) if f < 0] == list(refused)
        for layer, held in zip(layers, rows):
            kn, vn, q = (normal((T, h, 64), dtype, next(seed), 0.3) for h in (2, 2, 8))
            layer.append(cu, first, kn, vn, seq=U.device_ints(seq))
            out, lse = layer.attend(q, cu, seq=U.device_ints(seq), max_new=max(new), first=first)
            at = 0
            n, pool = [], []
            for x, (s, c) in enumerate(zip(seq, new)):
                if x not in refused:
                    held[s] = [torch.cat([old, Q.held(t[at : at + c])]) for old, t in zip(held[s], (kn, vn))]
                    n.append(len(held[s][0]))
                    pool.append(held[s])
                else:
                    n.append(0)
                    pool.append(None)
                at += c
            width = max(max(n), 1)
            k, v = (torch.zeros(len(seq), 2, width, 64, dtype=torch.float64, device="cuda:0") for _ in range(2))
            for x, p in enumerate(pool):
                if p is not None:
                    k[x, :, : n[x]], v[x, :, : n[x]] = p[0].transpose(0, 1), p[1].transpose(0, 1)
            table = np.arange(len(seq), dtype=np.int32)[:, None]
            U.check_attention(out, lse, U.attention_reference(q, k, v, table, n, new, 4, 0, 64 ** -0.5, width), dtype)

    step([0, 1, 2], [100, 37, 160])
    step([0, 2], [61, 1])
    pairs = a.fork(U.device_ints([0, 0]), U.device_ints([3, 4]))
    layers[1].copy(pairs)
    for held in rows:
        held[3], held[4] = list(held[0]), list(held[0])
    for _ in range(3):
        step([4, 3, 0, 1], [1, 1, 1, 1])
    a.release(U.device_ints([0, 2]))
    pairs = a.compact()
    layers[1].copy(pairs)
    for held in rows:
        held[0] = held[2] = [torch.zeros(0, 2, 64, device="cuda:0", dtype=torch.float64)] * 2
    step([3, 4, 1], [2, 3, 1])
    step([5, 3], [290, 1])
    step([1, 2], [1, 280])
    step([4, 0], [1, 1])
    for layer, held in zip(layers, rows):
        for s in (1, 2, 3, 4, 5):
            n = len(held[s][0])
            ko, vo = layer.read(U.device_ints([0, n]), seq=U.device_ints([s]), n_new=n)
            assert torch.equal(ko.double(), held[s][0]) and torch.equal(vo.double(), held[s][1])
    assert a.poll() == sla.SLA_OK


@pytest.mark.parametrize("order", [(True, False), (False, True), (True, False, True)])
def test_layers_of_both_kinds_share_a_table(sla, order):
    """Whichever is the first: each gives what it gives alone, in calls as large as its max_new, and a poll of either sees what went wrong."""
    from paper_2601_18401_b200.paged import PagedCache
    new = [6000, 2190, 1, 1]
    cu, seq = cu_of(new), U.device_ints([2, 0, 1, 3])
    T = sum(new)
    kn, vn, q = (normal((T, h, 128), BF16, 40 + i, 0.3) for i, h in enumerate((8, 8, 32)))
    shape = dict(n_q_heads=32, n_kv_heads=8, max_batch=4, max_new=8192)

    def calls(c, first):
        c.append(cu, first, kn, vn, seq=seq)
        return [*c.attend(q, cu, seq=seq, max_new=6000, first=first), *c.attend(q[:4], seq=seq), *c.read(seq=seq, cu_new=U.device_ints([0, 9, 9, 9, 9]), n_new=9)]
    layers = []
    for four in order:
        layers.append(PagedCache(1100, 4, 1100 * 64, four_bits=four, share=layers[0] if layers else None, **shape))
    assert len({c.handle for c in layers}) == 1 + (order[0] and False in order)
    more = PagedCache(1100, 4, 1100 * 64, share=layers[0], **shape)   # (a handle that is large enough is used again)
    assert more.handle is layers[order.index(False)].handle and more.handles is layers[0].handles
    del more
    first = layers[0].extend(cu, seq=seq)
    got = [calls(c, first) for c in layers]
    for c in layers:
        assert c.poll() == sla.SLA_OK
    for four, outs in zip(order, got):
        alone = PagedCache(1100, 4, 1100 * 64, four_bits=four, **shape)
        for a, b in zip(outs, calls(alone, alone.extend(cu, seq=seq))):
            assert torch.equal(a, b)
        assert alone.poll() == sla.SLA_OK
        del alone
    for c in layers:                                   # what one layer's call finds is reported by any of them, once
        c.read(U.device_ints([0, 1]), U.device_ints([10 ** 6]), n_new=1)
        assert [x.poll() for x in layers[::-1]] == [sla.SLA_ERR_DEVICE_INDEX] + [sla.SLA_OK] * (len(layers) - 1)


def test_a_layer_that_needs_no_more_shares_the_handle(sla):
    from paper_2601_18401_b200.paged import PagedCache
    shape = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=32, max_new=300)
    a = PagedCache(40, 6, 500, four_bits=True, **shape)
    for four in (True, False):
        b = PagedCache(40, 6, 500, share=a, four_bits=four, n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=32)
        assert b.handle is a.handle


def test_a_step_can_be_captured(sla):
    """Room, tokens, attention and reading back in a graph, replayed as the sequences grow; a second graph of the same handle beside it."""
    from paper_2601_18401_b200.paged import PagedCache
    c = PagedCache(60, 3, 640, n_q_heads=8, n_kv_heads=2, page_tokens=32, max_new=512, four_bits=True)
    cu = U.device_ints([0, 90, 120, 311])
    kp, vp = normal((311, 2, 128), BF16, 1), normal((311, 2, 128), BF16, 2)
    c.append(cu, c.extend(cu), kp, vp)
    kn, vn, q, q2 = normal((3, 2, 128), BF16, 3), normal((3, 2, 128), BF16, 4), normal((3, 8, 128), BF16, 5), normal((30, 8, 128), BF16, 6)
    cu2 = U.device_ints([0, 7, 11, 30])

    def step():
        first = c.extend()
        c.append(None, first, kn, vn)
        return c.attend(q), c.read(None, first)

    def many():
        return c.attend(q2, cu2, max_new=19)
    step(), many()
    torch.cuda.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        got = step()
    with torch.cuda.graph(two):
        got2 = many()
    for _ in range(40):
        one.replay()
        two.replay()
    torch.cuda.synchronize()
    n = [131, 71, 232]
    assert c.n_tokens.tolist() == n and c.poll() == sla.SLA_OK
    table = c.table.cpu().numpy()
    U.check_attention(*got[0], reference(q, c.k, c.v, table, n, [1, 1, 1], 4, 0, 128 ** -0.5, 32), BF16)
    U.check_attention(*got2, reference(q2, c.k, c.v, table, n, [7, 4, 19], 4, 0, 128 ** -0.5, 32), BF16)
    assert torch.equal(got[1][0].double(), Q.held(kn)) and torch.equal(got[1][1].double(), Q.held(vn))


def test_the_example_runs(sla):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.run(prompts=4, chunk=300, steps=6, four_bits=True)
    assert r["status"] == sla.SLA_OK and r["worst"] < 2e-2
    assert r["tokens"] == sum(200 + 777 * i for i in range(4)) + 3 * 7 + 3 * 6
