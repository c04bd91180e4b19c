"""Attention of new tokens over a paged cache against 64 bits: types, groups, pages, strides, windows, lengths from none to many."""
import math

import numpy as np
import pytest
import torch

import paged_util as U

pytestmark = pytest.mark.gpu


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


def build(sla, n, new, *, hkv=2, G=4, d=128, dtype=torch.bfloat16, page=16, token_major=False, gap=0, seed=3, spare=3):
    """A cache of sequences of n tokens, their pages scattered; what no sequence owns is NaN."""
    rs = np.random.RandomState(seed)
    held = [-(-int(x) // page) for x in n]
    n_pages = sum(held) + spare
    k, v = U.make_pools(n_pages, hkv, page, d, dtype, token_major, gap, seed)
    order = rs.permutation(n_pages)
    width = max(held + [1]) + 1
    table = np.full((len(n), width), -1, dtype=np.int32)
    at = 0
    for x, c in enumerate(held):
        table[x, :c] = order[at:at + c]
        at += c
        if c and n[x] % page:
            k[int(table[x, c - 1]), :, n[x] % page:] = math.nan
            v[int(table[x, c - 1]), :, n[x] % page:] = math.nan
    for p in order[at:]:
        k[int(p)] = math.nan
        v[int(p)] = math.nan
    ref = np.bincount(table[table >= 0], minlength=n_pages)
    tensors = [U.device_ints(table), U.device_ints(n), U.device_ints(ref)]
    cache = sla.make_cache(k, v, *tensors)
    cu = U.device_ints(np.concatenate([[0], np.cumsum(new)]))
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed + 1)
    q = torch.empty(int(sum(new)), hkv * G, d, dtype=dtype, device="cuda:0").normal_(generator=g)
    return cache, k, v, table, q, cu


def run(sla, handle, n, new, window=0, scale=None, max_new=None, prep=None, **kw):
    cache, k, v, table, q, cu = build(sla, n, new, **kw)
    if prep:
        prep(k, v, table, q)
    out, lse = sla.sla_paged_attention(handle, q, cache, cu, window=window, softmax_scale=scale, max_new=max(new) if max_new is None else max_new)
    torch.cuda.synchronize()
    s = 1 / math.sqrt(q.shape[-1]) if scale is None else scale
    ref = U.attention_reference(q, k, v, table, n, new, kw.get("G", 4), window, s, kw.get("page", 16))
    U.check_attention(out, lse, ref, q.dtype)
    return out, lse, ref


BF16, F32 = torch.bfloat16, torch.float32
SINGLE = ([1, 2, 15, 16, 17, 0, 63, 64, 65, 700], [1] * 10)       # one token each, an empty sequence among them
CHUNKS = ([40, 5, 0, 129, 300, 64, 513], [40, 0, 0, 1, 77, 64, 200])   # whole prompts, ends of prompts, nothing new


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("lens", [SINGLE, CHUNKS], ids=["single", "chunks"])
def test_types(sla, handle, dtype, d, lens):
    run(sla, handle, *lens, dtype=dtype, d=d)


@pytest.mark.parametrize("hkv,G", [(1, 1), (3, 2), (2, 3), (1, 5), (2, 7), (1, 8), (1, 12), (2, 16)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_groups(sla, handle, hkv, G, dtype):
    run(sla, handle, *SINGLE, hkv=hkv, G=G, dtype=dtype)
    run(sla, handle, *CHUNKS, hkv=hkv, G=G, dtype=dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("token_major,gap", [(False, 0), (True, 0), (False, 64), (True, 8)])
def test_pages_and_strides(sla, handle, page, token_major, gap):
    run(sla, handle, *SINGLE, page=page, token_major=token_major, gap=gap)
    run(sla, handle, *CHUNKS, page=page, token_major=token_major, gap=gap, hkv=3)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 129, 400, 5000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_window(sla, handle, window, dtype):
    run(sla, handle, *SINGLE, window=window, dtype=dtype)
    run(sla, handle, *CHUNKS, window=window, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_keys(sla, handle, dtype):
    """Sequences shorter than their new tokens: the first rows see nothing."""
    out, lse, _ = run(sla, handle, [3, 0, 20, 1], [5, 4, 20, 3], dtype=dtype)
    assert (out[:2] == 0).all() and (out[5:9] == 0).all()
    run(sla, handle, [0, 0], [1, 1], dtype=dtype)
    run(sla, handle, [0, 7], [1, 0], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G", [4, 16])
def test_long_sequences_are_cut_and_joined(sla, handle, dtype, G):
    """Few rows over long contexts: every CTA takes a part, a second kernel joins them."""
    run(sla, handle, [20000, 33, 9001], [1, 1, 1], G=G, dtype=dtype, page=64)
    run(sla, handle, [20000, 33, 9001], [3, 2, 1], G=G, dtype=dtype, page=64)
    run(sla, handle, [6000], [70], G=G, dtype=dtype, page=64)
    run(sla, handle, [6000, 4000], [70, 130], G=G, dtype=dtype, page=32, window=900)


@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 2), (BF16, 150), (F32, 1), (F32, 150)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(sla, handle, dtype, new, bad):
    """A NaN or an infinity in a key or value is seen by the rows at and after it (inside the window), and by no other."""
    n = [400, 300]
    new = [new, new]
    at = 399 if new[0] == 1 else 398 if new[0] == 2 else 330

    def one(which):
        def prep(k, v, table, q):
            t = (k, v)[which]
            t[int(table[0, at // 16]), 1, at % 16, 5] = bad
        return prep
    run(sla, handle, n, new, dtype=dtype, prep=one(1))
    run(sla, handle, n, new, dtype=dtype, prep=one(1), window=20)

    # keys: a row that sees it is NaN, or has an infinite weight; the others are what they were
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype)
    clean, clean_lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=new[0])
    one(0)(k, v, table, q)
    out, lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=new[0])
    sees = n[0] - new[0] + torch.arange(new[0], device=out.device) >= at
    assert torch.equal(out[:new[0]][~sees], clean[:new[0]][~sees]) and torch.equal(out[new[0]:], clean[new[0]:])
    assert torch.equal(lse[:new[0]][~sees], clean_lse[:new[0]][~sees])
    assert torch.equal(out[:, :4], clean[:, :4])   # the other KV head
    if math.isnan(bad):
        assert torch.isnan(out[:new[0]][sees][:, 4:]).all() and torch.isnan(lse[:new[0]][sees][:, 4:]).all()


@pytest.mark.parametrize("dtype,new", [(BF16, [1, 1]), (BF16, [60, 1]), (F32, [60, 1])])
def test_large_logits_and_scales(sla, handle, dtype, new):
    run(sla, handle, [500, 31], new, dtype=dtype, scale=3.0)
    run(sla, handle, [500, 31], new, dtype=dtype, scale=0.0)
    run(sla, handle, [500, 31], new, dtype=dtype, scale=-0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_queries_slots_and_shared_pages(sla, handle, dtype):
    """Queries inside a larger tensor, sequences named by slot in any order, two sequences on the same pages."""
    n, new = [100, 64, 250], [3, 1, 40]
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype)
    table[1] = table[2]                     # slot 1 shares slot 2's first pages
    cache.tensors[2].copy_(U.device_ints(table))
    big = torch.zeros(44, 3, 8, 128, dtype=dtype, device="cuda:0")
    big[:, 1] = q
    order = [2, 0, 1]
    cu2 = U.device_ints(np.concatenate([[0], np.cumsum([new[s] for s in order])]))
    out = torch.full_like(big, 7.0)
    o, lse = sla.sla_paged_attention(handle, big[:, 1], cache, cu2, seq=U.device_ints(order), max_new=40, out=out[:, 1])
    ref = U.attention_reference(q, k, v, table[order], [n[s] for s in order], [new[s] for s in order], 4, 0, 128 ** -0.5, 16)
    U.check_attention(o, lse, ref, dtype)
    assert (out[:, 0] == 7).all() and (out[:, 2] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 12])
def test_queries_with_tokens_inside_heads(sla, handle, dtype, G):
    """Queries stored head by head: [Hq, n_new, D] seen as [n_new, Hq, D]."""
    for n, new in (SINGLE, CHUNKS, ([300, 41], [300, 41])):
        cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, G=G)
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
        out, lse = sla.sla_paged_attention(handle, q, cache, cu, max_new=max(new))
        assert out.stride() == q.stride()
        U.check_attention(out, lse, U.attention_reference(q, k, v, table, n, new, G, 0, 128 ** -0.5, 16), dtype)


FEW = [(1, 16), (1, 9), (2, 8), (2, 3), (3, 5), (4, 4), (4, 2), (5, 3), (7, 2), (8, 2)]   # heads of a group x new tokens <= 16


@pytest.mark.parametrize("G,new", FEW)
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_few_new_tokens(sla, handle, G, new, dtype, d):
    """As many rows as the kernel of single tokens takes: ragged counts, none, fewer keys than tokens, a long sequence."""
    n = [1, 2, 15, 16, 17, 0, 63, 64, 65, 700, 3, 40, 9001]
    c = [(i * 5 + 2) % (new + 1) for i in range(len(n))]
    c[2] = c[5] = c[10] = c[-1] = new
    for window in (0, 1, 7, 100):
        out, lse, _ = run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=window, max_new=new)
    one, one_lse, _ = run(sla, handle, n, c, dtype=dtype, d=d, G=G, window=100, max_new=400)   # the kernel of chunks
    assert torch.allclose(out.float(), one.float(), atol=0.02) and torch.equal(lse.isinf(), one_lse.isinf())


@pytest.mark.parametrize("G,new", [(1, 16), (2, 3), (4, 4), (8, 2)])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_few_new_tokens_and_values_that_are_not_finite(sla, handle, G, new, dtype, d, bad):
    """At every position that only some of the new tokens see, at either end of the window."""
    n = [400, 300]
    for window in (0, 40):
        for back in range(new):
            for at in (n[0] - 1 - back, n[0] - window - back):
                if at >= n[0]:
                    continue

                def prep(k, v, table, q):
                    v[int(table[0, at // 16]), 1, at % 16, 5] = bad
                    v[int(table[0, at // 16]), 0, at % 16, d - 1] = bad
                run(sla, handle, n, [new, new], dtype=dtype, d=d, G=G, window=window, prep=prep)


@pytest.mark.parametrize("dtype,n_seqs,new,G,d", [(F32, 1030, 1, 16, 128), (F32, 600, 2, 8, 128), (BF16, 1010, 1, 16, 128), (BF16, 1030, 4, 4, 64)])
def test_many_sequences_of_many_rows(sla, handle, dtype, n_seqs, new, G, d):
    """More sequences than fit beside the sums of 16 rows in the shared memory of one launch."""
    rs = np.random.RandomState(n_seqs)
    n = rs.randint(0, 40, n_seqs)
    c = np.minimum(n, rs.randint(0, new + 1, n_seqs)) if new > 1 else np.ones(n_seqs, dtype=int)
    run(sla, handle, n.tolist(), c.tolist(), dtype=dtype, hkv=1, G=G, d=d, max_new=new)


@pytest.mark.parametrize("dtype,n_seqs,new", [(BF16, 1100, 1), (F32, 1030, 1), (BF16, 1500, 3), (F32, 300, 2)])
def test_many_sequences(sla, handle, dtype, n_seqs, new):
    """More sequences than one launch, one warp or one CTA takes at a time."""
    rs = np.random.RandomState(n_seqs)
    n = rs.randint(0, 70, n_seqs)
    c = np.minimum(n, rs.randint(0, new + 1, n_seqs)) if new > 1 else np.minimum(n, 1)
    run(sla, handle, n.tolist(), c.tolist(), dtype=dtype, hkv=1, G=2, d=64, max_new=new)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_above_2_to_31(sla, handle, dtype):
    """A pool of more than 2^31 elements: the pages of the sequences lie behind them."""
    free = torch.cuda.mem_get_info()[0]
    n_pages, hkv, page, d = 33000, 8, 64, 128
    if free < 2.5 * n_pages * hkv * page * d * (2 if dtype == BF16 else 4):
        pytest.skip("not enough device memory")
    k, v = (torch.empty(n_pages, hkv, page, d, dtype=dtype, device="cuda:0") for _ in range(2))
    table = np.full((2, 4), -1, dtype=np.int32)
    table[0, :3], table[1, :1] = [32999, 32800, 40], [32900]
    for p in (32999, 32800, 40, 32900):
        k[p].normal_(), v[p].normal_()
    n = [150, 40]
    ref = np.zeros(n_pages, dtype=np.int32)
    cache = sla.make_cache(k, v, U.device_ints(table), U.device_ints(n), U.device_ints(ref))
    for new in ([1, 1], [100, 40]):
        q = torch.empty(sum(new), 16, d, dtype=dtype, device="cuda:0").normal_()
        out, lse = sla.sla_paged_attention(handle, q, cache, U.device_ints(np.concatenate([[0], np.cumsum(new)])), max_new=max(new))
        U.check_attention(out, lse, U.attention_reference(q, k, v, table, n, new, 2, 0, d ** -0.5, page), dtype)
    kn, vn = (torch.empty(2, hkv, d, dtype=dtype, device="cuda:0").normal_() for _ in range(2))
    sla.sla_cache_append(handle, cache, None, U.device_ints([127, 39]), kn, vn)
    assert torch.equal(k[32800, :, 63], kn[0]) and torch.equal(v[32900, :, 39], vn[1])
    sla.sla_cache_copy(handle, cache, U.device_ints([[32999], [32998]]))
    assert torch.equal(k[32998], k[32999]) and torch.equal(v[32998], v[32999])
    del k, v, cache
    torch.cuda.empty_cache()


def test_calls_can_be_captured(sla):
    """A step -- room, tokens, attention, the span step -- in a graph, replayed as the sequences grow."""
    from paper_2601_18401_b200.paged import PagedCache
    c = PagedCache(40, 3, 640, n_q_heads=8, n_kv_heads=2, page_tokens=32, max_new=512, params=sla.make_params(4, 0))
    g = torch.Generator(device="cuda:0")
    rand = lambda *s: torch.empty(*s, dtype=BF16, device="cuda:0").normal_(generator=g)  # noqa: E731
    cu = U.device_ints([0, 90, 120, 311])
    c.append(cu, c.extend(cu), rand(311, 2, 128), rand(311, 2, 128))
    kn, vn, q, q_s = rand(3, 2, 128), rand(3, 2, 128), rand(3, 8, 128), rand(3, 8, 128)

    def step():
        first = c.extend()
        c.append(None, first, kn, vn)
        return c.attend(q), c.step(q_s, q, max_tokens=640)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(40):
        graph.replay()
    torch.cuda.synchronize()
    n = [131, 71, 232]
    assert c.n_tokens.tolist() == n and c.poll() == sla.SLA_OK
    table = c.table.cpu().numpy()
    U.check_attention(*got[0], U.attention_reference(q, c.k, c.v, table, n, [1, 1, 1], 4, 0, 128 ** -0.5, 32), BF16)
    again = c.step(q_s, q, max_tokens=640)
    assert all(torch.equal(a, b) for a, b in zip(got[1], again))


def test_the_example_runs(sla):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.run(prompts=4, chunk=300, steps=6, span_from=1500)
    assert r["status"] == sla.SLA_OK and r["worst"] < 2e-2
    assert r["tokens"] == sum(200 + 777 * i for i in range(4)) + 3 * 7 + 3 * 6


def test_chunk_bound_may_be_loose(sla, handle):
    """max_new is a bound: single tokens with a bound of many give the same results."""
    a, la, _ = run(sla, handle, *SINGLE)
    b, lb, _ = run(sla, handle, *SINGLE, max_new=500)
    assert (a.float() - b.float()).abs().max() < 0.05


def test_no_new_token_and_one_token_without_offsets(sla, handle):
    cache, k, v, table, q, cu = build(sla, [30, 50], [1, 1])
    a = sla.sla_paged_attention(handle, q, cache)            # one token per slot
    b = sla.sla_paged_attention(handle, q, cache, cu, max_new=1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    zero = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    o, l = sla.sla_paged_attention(handle, q[:0], cache, zero)
    assert o.shape == (0, 8, 128) and l.shape == (0, 8)


def test_same_result_every_time(sla, handle):
    """The order of sums does not depend on timing."""
    cache, k, v, table, q, cu = build(sla, [9000, 100, 4000], [1, 50, 300], page=64)
    a = sla.sla_paged_attention(handle, q, cache, cu, max_new=300)
    for _ in range(3):
        b = sla.sla_paged_attention(handle, q, cache, cu, max_new=300)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_other_stream(sla, handle):
    cache, k, v, table, q, cu = build(sla, *CHUNKS)
    a = sla.sla_paged_attention(handle, q, cache, cu, max_new=200)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        b = sla.sla_paged_attention(handle, q, cache, cu, max_new=200)
    st.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_what_is_out_of_range_is_flagged_and_not_followed(sla):
    """Slots and pages outside the cache, lengths beyond the table, offsets that do not ascend: the status word, no fault."""
    h = sla.Handle(0, 1 << 28)
    for new in ([1, 1], [40, 33]):
        cache, k, v, table, q, cu = build(sla, [100, 60], new)
        sla.sla_paged_attention(h, q, cache, cu, max_new=max(new), seq=U.device_ints([0, 9]))
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
        bad = table.copy()
        bad[0, 1] = 10 ** 6
        cache.tensors[2].copy_(U.device_ints(bad))
        sla.sla_paged_attention(h, q, cache, cu, max_new=max(new))
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
        bad[0, 1] = -1
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


def test_refusals(sla, handle):
    cache, k, v, table, q, cu = build(sla, [30, 50], [1, 1])
    with pytest.raises(sla.SlaError):
        sla.sla_paged_attention(handle, q, cache, cu, window=-1)
    with pytest.raises(sla.SlaError):
        sla.sla_paged_attention(handle, q, cache, cu, softmax_scale=math.nan)
    with pytest.raises(sla.SlaError):
        sla.sla_paged_attention(handle, q[:, :7], cache, cu)         # not a multiple of the KV heads
    with pytest.raises(sla.SlaError):
        sla.sla_paged_attention(handle, torch.zeros(2, 40, 128, dtype=q.dtype, device=q.device), cache, cu)   # groups of 20
    with pytest.raises(sla.SlaError):
        sla.sla_paged_attention(handle, q, cache, cu, max_new=0)
    with pytest.raises(ValueError):
        sla.sla_paged_attention(handle, q[..., :64], cache, cu)
    with pytest.raises(TypeError):
        sla.sla_paged_attention(handle, q.half(), cache, cu)
    with pytest.raises(ValueError):
        sla.sla_paged_attention(handle, q, cache, cu, out=torch.empty(2, 8, 256, dtype=q.dtype, device=q.device)[..., ::2])
    small = sla.Handle(0, 4096)
    with pytest.raises(sla.SlaError) as e:
        sla.sla_paged_attention(small, q, cache, cu)
    assert e.value.status == -3
    small.close()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("max_new", [1, 2, 3])
def test_more_new_tokens_than_max_new_are_flagged(sla, dtype, max_new):
    """Where the rows of a sequence were to fit into one pass: the status word, nothing written outside the call's rows."""
    h = sla.Handle(0, 1 << 28)
    new = [2 * max_new, 0]
    cache, k, v, table, q, cu = build(sla, [100, 60], new, dtype=dtype)
    out = torch.full((q.shape[0] + 8, *q.shape[1:]), 7.0, dtype=dtype, device="cuda:0")
    sla.sla_paged_attention(h, q, cache, cu, max_new=max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    assert (out[q.shape[0]:] == 7).all()
    sla.sla_paged_attention(h, q, cache, U.device_ints([0, 10 ** 6, -5]), max_new=max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    assert (out[q.shape[0]:] == 7).all()
    sla.sla_paged_attention(h, q, cache, cu, max_new=2 * max_new, out=out[:q.shape[0]])
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


@pytest.mark.parametrize("n", [300, 400, 520, 650])
@pytest.mark.parametrize("G,new", [(4, 5), (4, 20), (4, 32), (1, 40), (1, 128), (8, 16), (16, 8)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_small_units_and_values_that_are_not_finite(sla, handle, n, G, new, bad):
    """Units of few tokens, whose tiles two groups of warps take in turn: whichever of them meets the value, all rows that see it
    have it and the others do not, at either end of a window."""
    for window in (0, 200):
        for back in {0, new // 2, new - 1}:
            for at in (n - 1 - back, n - window - back):
                if at >= n:
                    continue

                def prep(k, v, table, q):
                    v[int(table[0, at // 16]), 1, at % 16, 5] = bad
                run(sla, handle, [n], [new], G=G, window=window, prep=prep)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("new", [3, 20, 70, 200])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_cut_units_and_values_that_are_not_finite(sla, handle, dtype, d, new, bad):
    """The same where a sequence is cut into parts that several CTAs attend to: near its end, at a window's beginning, in every tile."""
    n = 4000 + 37 * new
    for window in (0, 2500):
        for at in (n - 1, n - new, n - 1 - new // 2, n - window - new // 2, n - 130):
            if at >= n:
                continue

            def prep(k, v, table, q):
                v[int(table[0, at // 16]), 1, at % 16, d - 3] = bad
                v[int(table[1, 10]), 0, 3, 2] = bad
            run(sla, handle, [n, 350], [new, new], dtype=dtype, d=d, window=window, prep=prep)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("tokens_inside", [False, True])
@pytest.mark.parametrize("G,n,new", [(4, [6000, 90], [3, 4]), (4, [6000, 90], [70, 90]), (3, [300, 41], [300, 41]), (1, [5000], [130]), (16, [2000, 7], [1, 1])])
def test_queries_of_any_16_bytes(sla, handle, dtype, d, tokens_inside, G, n, new):
    """Rows of q and out that begin at any multiple of 16 bytes, tokens inside or outside heads, whole and cut units."""
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, d=d, G=G)
    T, H = q.shape[:2]
    a, b = (H, T) if tokens_inside else (T, H)

    def wide(x):
        big = torch.full((a, b, d + 8), 7.0, dtype=dtype, device="cuda:0")
        view = big[:, :, 8:]
        view.copy_(x.transpose(0, 1) if tokens_inside else x)
        return big, view.transpose(0, 1) if tokens_inside else view
    _, q2 = wide(q)
    big, out = wide(torch.zeros_like(q))
    o, lse = sla.sla_paged_attention(handle, q2, cache, cu, max_new=max(new), out=out)
    U.check_attention(o, lse, U.attention_reference(q, k, v, table, n, new, G, 0, d ** -0.5, 16), dtype)
    assert (big[:, :, :8] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,new,G,window", [([20011], [300], 4, 0), ([20011, 17000], [150, 40], 4, 16900), ([33000], [20], 4, 0), ([18000, 19000], [260, 129], 1, 0)])
@pytest.mark.parametrize("bad", [None, math.nan])
def test_long_units_in_turns(sla, handle, d, n, new, G, window, bad):
    """Units of so many keys that CTAs begin them at different ones."""
    def prep(k, v, table, q):
        if bad is not None:
            at = n[0] - 1 - new[0] // 2
            v[int(table[0, at // 64]), 1, at % 64, 7] = bad
    run(sla, handle, n, new, d=d, G=G, window=window, page=64, prep=prep)


@pytest.mark.parametrize("d", [64, 128])
def test_after_a_wait_that_ran_out_no_row_is_written(sla, d):
    """CTAs that leave early leave their ranges without a cut: the join writes nothing from what an earlier call of the same
    layout, or of another, has left in the scratch memory."""
    h = sla.Handle(0, 1 << 28)
    n, new = [9000, 4000, 2500], [70, 300, 129]
    cache, k, v, table, q, cu = build(sla, n, new, d=d, page=64)
    big = build(sla, [6000] * 9, [700] * 9, d=d, page=64, seed=8)
    want = sla.sla_paged_attention(h, q, cache, cu, max_new=300)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    rows, guard = q.shape[0], 512
    for before in (lambda: None, lambda: sla.sla_paged_attention(h, big[4], big[0], big[5], max_new=700)):
        before()
        out = torch.full((rows + 2 * guard, *q.shape[1:]), 7.0, dtype=q.dtype, device=q.device)
        lse = torch.full((rows + 2 * guard, q.shape[1]), 7.0, device=q.device)
        sla.sla_selftest_paged_expiry(h, True)
        sla.sla_paged_attention(h, q, cache, cu, max_new=300, out=out[guard:guard + rows], lse=lse[guard:guard + rows])
        sla.sla_selftest_paged_expiry(h, False)
        assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_TIMEOUT
        assert (out == 7).all() and (lse == 7).all()
    again = sla.sla_paged_attention(h, q, cache, cu, max_new=300)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    h.close()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window", [2 ** 30, 2 ** 31 - 5, 2 ** 31 - 1])
@pytest.mark.parametrize("n,new", [([1], [4]), ([10], [20]), ([3, 0, 20, 1], [5, 4, 20, 3]), ([130, 40], [200, 300])])
def test_a_window_beyond_any_length_is_none(sla, handle, dtype, window, n, new):
    """Sequences shorter than their new tokens, whose first positions are negative, under windows up to the largest int."""
    for bound in (max(new), 400):
        a, la, _ = run(sla, handle, n, new, window=window, dtype=dtype, max_new=bound)
        b, lb, _ = run(sla, handle, n, new, dtype=dtype, max_new=bound)
        assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("d,window", [(128, 0), (64, 0), (128, 700000)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite_in_long_ranges(sla, d, window, bad):
    """8192 new tokens that end at 2^20: a CTA's ranges are some 900 thousand keys long, and a value in one of the last rows' own keys
    (or at the window's beginning) reaches the rows that see it, in its column, without a wait that runs out."""
    N, T, hkv, G, page = 1 << 20, 8192, 2, 16, 64
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough device memory")
    k, v = U.make_pools(N // page, hkv, page, d, BF16)
    table = np.random.RandomState(1).permutation(N // page).astype(np.int32)[None]
    cache = sla.make_cache(k, v, U.device_ints(table), U.device_ints([N]), U.device_ints(np.ones(N // page)))
    q = torch.empty(T, hkv * G, d, dtype=BF16, device="cuda:0").normal_()
    cu = U.device_ints([0, T])
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, hkv * G, 1, T))
    clean, clean_lse = sla.sla_paged_attention(h, q, cache, cu, window=window)
    pos = torch.arange(N - T, N, device="cuda:0")
    for at in (N - 70, N - window - 70 if window else N - T + 3):
        for g, col in ((0, 5), (1, d - 1)):
            v[int(table[0, at // page]), g, at % page, col] = bad
        out, lse = sla.sla_paged_attention(h, q, cache, cu, window=window)
        assert sla.sla_poll_status(h) == sla.SLA_OK
        sees = (pos >= at) & ((pos - at < window) if window else True)
        assert 0 < sees.sum() < T
        want = clean.clone()
        want[sees, :G, 5] = bad
        want[sees, G:, d - 1] = bad
        assert torch.equal(out.nan_to_num(123.0), want.nan_to_num(123.0)) and torch.equal(out.isnan(), want.isnan())
        assert torch.equal(lse, clean_lse)
        for g, col in ((0, 5), (1, d - 1)):
            v[int(table[0, at // page]), g, at % page, col] = 0.5
        clean, clean_lse = sla.sla_paged_attention(h, q, cache, cu, window=window)
    # a few rows against 64 bits
    scale = d ** -0.5
    pages = torch.from_numpy(table[0].astype(np.int64)).cuda()
    rows = [0, 17, 5000, T - 1]
    ref = [torch.zeros(len(rows), hkv * G, d, dtype=torch.float64, device="cuda:0"), torch.zeros(len(rows), hkv * G, dtype=torch.float64, device="cuda:0")]
    ref += [torch.zeros_like(ref[0]), torch.zeros_like(ref[1]), torch.zeros(len(rows), dtype=torch.float64, device="cuda:0")]
    for g in range(hkv):
        kk, vv = (t[pages, g].reshape(N, d).double() for t in (k, v))
        hs = slice(g * G, (g + 1) * G)
        for x, r in enumerate(rows):
            p = N - T + r
            lo = max(0, p - window + 1) if window else 0
            z = q[r, hs].double() @ kk[lo:p + 1].T * scale
            ref[1][x, hs] = torch.logsumexp(z, -1)
            w = torch.exp(z - ref[1][x, hs, None])
            ref[0][x, hs], ref[2][x, hs] = w @ vv[lo:p + 1], w @ vv[lo:p + 1].abs()
            ref[3][x, hs] = (q[r, hs].double().abs() @ kk[lo:p + 1].abs().T).amax(-1) * scale
            ref[4][x] = p + 1 - lo
    U.check_attention(clean[rows], clean_lse[rows], ref, BF16)
    h.close()
    del k, v, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d,hkv,G", [(BF16, 128, 8, 4), (BF16, 64, 2, 16), (BF16, 128, 2, 1), (F32, 128, 2, 4), (F32, 64, 1, 16)])
@pytest.mark.parametrize("n_seqs,n_new", [(4, 4), (3, 40), (40, 300)])
def test_a_workspace_of_the_size_asked_for_is_enough(sla, dtype, d, hkv, G, n_seqs, n_new):
    """Every bound of the new tokens, loose ones included, batches below the size asked for, either sign of the scale."""
    new = [n_new // n_seqs] * n_seqs
    new[0] += n_new - sum(new)
    n = [30 + x for x in new]
    cache, k, v, table, q, cu = build(sla, n, new, dtype=dtype, d=d, hkv=hkv, G=G)
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, hkv * G, n_seqs, n_new))
    for scale in (None, -0.1):
        ref = U.attention_reference(q, k, v, table, n, new, G, 0, d ** -0.5 if scale is None else scale, 16)
        for bound in sorted({max(new), max(new) + 1, 16, 17, 64, 65, n_new, n_new + 1, 2 ** 31 - 1}):
            if bound >= max(new):
                U.check_attention(*sla.sla_paged_attention(h, q, cache, cu, max_new=bound, softmax_scale=scale), ref, dtype)
        for less in range(1, n_seqs, 7):   # the first sequences alone
            rows = sum(new[:less])
            out, lse = sla.sla_paged_attention(h, q[:rows], cache, cu[:less + 1].contiguous(), max_new=2 ** 31 - 1, softmax_scale=scale)
            U.check_attention(out, lse, [t[:rows] for t in ref], dtype)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


def test_ranges_of_more_than_a_second(sla):
    """2^28 tokens, in pages that are the same one again and again but for forty: a CTA's range takes some three seconds, and the warps
    that wait for its end wait so long.  The keys of the one page have logits of -200 and weights that are 0 in fp32, so that the result is
    that over the forty."""
    N, T, G, page, d = 1 << 28, 1600, 16, 256, 64
    k, v = U.make_pools(8, 1, page, d, BF16)
    k[..., 0] = 0
    k[0] = 0
    k[0, ..., 0] = -200
    table = np.zeros((1, N // page), dtype=np.int32)
    at = np.random.RandomState(4).choice(N // page - T // page - 1, 40, replace=False)
    table[0, at] = 1 + np.arange(40) % 7
    cache = sla.make_cache(k, v, U.device_ints(table), U.device_ints([N]), U.device_ints(np.bincount(table[0], minlength=8)))
    q = torch.empty(T, G, d, dtype=BF16, device="cuda:0").normal_()
    q[..., 0] = 8
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, G, 1, T))
    out, lse = sla.sla_paged_attention(h, q, cache, U.device_ints([0, T]))
    assert sla.sla_poll_status(h) == sla.SLA_OK
    rows = list(range(0, T, 37)) + [T - 1]
    pages = torch.from_numpy(table[0, np.sort(at)].astype(np.int64)).cuda()
    kk, vv = (t[pages, 0].reshape(-1, d).double() for t in (k, v))
    z = torch.einsum("thd,jd->thj", q[rows].double(), kk) * d ** -0.5
    w = z.softmax(-1)
    ref = (torch.einsum("thj,jd->thd", w, vv), z.logsumexp(-1), torch.einsum("thj,jd->thd", w, vv.abs()),
           torch.einsum("thd,jd->thj", q[rows].double().abs(), kk.abs()).amax(-1) * d ** -0.5, torch.full((len(rows),), float(len(kk)), dtype=torch.float64, device="cuda:0"))
    U.check_attention(out[rows], lse[rows], ref, BF16)
    h.close()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("n,T,G", [(1 << 20, 2400, 16), ((1 << 22) + 777, 2400, 16), (1 << 22, 1, 16), (600000, 700, 1)])
def test_long_sums_of_values_of_one_sign(sla, dtype, d, n, T, G):
    """Hundreds of thousands of keys of like weight in a range: the sums lose nothing at their lower end, where the tensor cores cut
    what does not fit.  Pages that are the same 64 again and again, so that a key's weight counts as often as a row sees its page.

    Bounds, relative, values positive: bf16 rounds each weight and the result to 2^-9; a sum of 65536 keys in TMEM is cut 4096 times by at
    most 2^-23; the 8192 or so tiles' sums in fp32 (of O, of the weights) are off by 2^-24 each.  fp32 instead: 2^-24 for every 64 keys'
    sums and within them, and the logits' 2^-19."""
    if dtype == F32 and n > 1 << 20 and T > 1:
        n = (1 << 18) + 777   # (0.2 s)
    page, n_pages = 256, 64
    k, v = U.make_pools(n_pages, 1, page, d, dtype)
    v.abs_()
    width = -(-n // page)
    table = (np.arange(width) % n_pages).astype(np.int32)[None]
    cache = sla.make_cache(k, v, U.device_ints(table), U.device_ints([n]), U.device_ints(np.bincount(table[0], minlength=n_pages)))
    q = torch.empty(T, G, d, dtype=dtype, device="cuda:0").normal_()
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, G, 1, T))
    sla.sla_set_debug_canaries(h, True)
    out, lse = sla.sla_paged_attention(h, q, cache, None if T == 1 else U.device_ints([0, T]))
    assert sla.sla_poll_status(h) == sla.SLA_OK
    kk, vv = (t[:, 0].reshape(-1, d).double() for t in (k, v))
    at = torch.arange(len(kk), device="cuda:0")
    tiles = n / 128
    tol = 2.0 ** -8 + 4096 * 2.0 ** -23 + 2 * tiles * 2.0 ** -24 if dtype == BF16 else 4 * tiles * 2.0 ** -24 + 2.0 ** -18
    for r in {0, T // 2, T - 1}:
        seen = n - T + r + 1
        times = (seen // len(kk) + (at < seen % len(kk))).double()
        z = q[r].double() @ kk.T * d ** -0.5
        w = torch.exp(z) * times
        want = (w @ vv) / w.sum(-1, keepdim=True)
        assert ((out[r].double() / want - 1).abs() <= tol).all()
        assert ((lse[r].double() - w.sum(-1).log()).abs() <= tol).all()
    h.close()
