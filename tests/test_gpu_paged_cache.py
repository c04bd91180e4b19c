"""Bookkeeping of the paged cache -- extend, append, fork, release, compact, copy -- against a model in plain Python: every table
entry, length, count and every page's contents equal."""
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
    h = sla.Handle(0, 1 << 28)
    yield h
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


class Pair:
    """A cache on the device and its model; the model's tokens are a list of rows per slot."""

    def __init__(self, sla, h, n_pages=40, page=16, n_slots=8, width=12, hkv=2, d=64, dtype=torch.bfloat16, token_major=False, gap=0):
        self.sla, self.h, self.page = sla, h, page
        self.m = U.Model(n_pages, page, n_slots, width)
        self.k, self.v = U.make_pools(n_pages, hkv, page, d, dtype, token_major, gap)
        self.dev = [U.device_ints(a) for a in (self.m.table, self.m.n, self.m.ref)]
        self.cache = sla.make_cache(self.k, self.v, *self.dev)
        self.rows = {s: [] for s in range(n_slots)}   # (k, v) rows [hkv, d] by position
        self.gen = torch.Generator(device="cuda:0")

    def same(self):
        torch.cuda.synchronize()
        for a, b in zip(self.dev, (self.m.table, self.m.n, self.m.ref)):
            assert np.array_equal(a.cpu().numpy(), b)
        for s, rows in self.rows.items():
            assert len(rows) == self.m.n[s]
            for p, (k, v) in enumerate(rows):
                page = int(self.m.table[s, p // self.page])
                assert torch.equal(self.k[page, :, p % self.page], k), (s, p)
                assert torch.equal(self.v[page, :, p % self.page], v), (s, p)

    def add(self, seq, new, strided=False):
        hkv, d = self.k.shape[1], self.k.shape[3]
        T = int(sum(new))
        x = torch.empty(2, max(T, 1), hkv + (1 if strided else 0), d, dtype=self.k.dtype, device="cuda:0").normal_(generator=self.gen)
        k_new, v_new = x[0, :T, :hkv], x[1, :T, :hkv]
        cu = U.device_ints(np.concatenate([[0], np.cumsum(new)]))
        first = self.sla.sla_cache_extend(self.h, self.cache, cu, seq=U.device_ints(seq))
        want = self.m.extend(seq, new)
        assert np.array_equal(first.cpu().numpy(), want)
        self.sla.sla_cache_append(self.h, self.cache, cu, first, k_new, v_new, seq=U.device_ints(seq))
        at = 0
        for s, c, f in zip(seq, new, want):
            if f >= 0:
                self.rows[s] += [(k_new[at + r], v_new[at + r]) for r in range(c)]
            at += c
        self.same()
        return want

    def fork(self, src, dst):
        pairs = self.sla.sla_cache_fork(self.h, self.cache, U.device_ints(src), U.device_ints(dst))
        want = self.m.fork(src, dst)
        assert np.array_equal(pairs.cpu().numpy(), want)
        for s, d in zip(src, dst):
            if self.m.n[d]:
                self.rows[d] = list(self.rows[s])
        self.same()
        return pairs

    def release(self, seq):
        self.sla.sla_cache_release(self.h, self.cache, U.device_ints(seq))
        self.m.release(seq)
        for s in seq:
            self.rows[s] = []
        self.same()

    def compact(self):
        pairs = self.sla.sla_cache_compact(self.h, self.cache)
        assert np.array_equal(pairs.cpu().numpy(), self.m.compact())
        self.same()
        live = int((self.m.ref > 0).sum())
        assert (self.m.ref[:live] > 0).all()
        return pairs


@pytest.mark.parametrize("dtype,d,hkv", [(torch.bfloat16, 64, 2), (torch.bfloat16, 128, 8), (torch.float32, 128, 3), (torch.float32, 64, 1)])
@pytest.mark.parametrize("token_major,gap", [(False, 0), (True, 0), (True, 24)])
def test_a_life_of_a_cache(sla, handle, dtype, d, hkv, token_major, gap):
    """Prompts, steps of one token, forks, ends, compaction, and on."""
    c = Pair(sla, handle, dtype=dtype, d=d, hkv=hkv, token_major=token_major, gap=gap)
    c.add([0, 2, 5], [40, 0, 33])
    c.add([5, 0], [1, 15])
    c.fork([0, 5, 0, 2], [1, 3, 4, 6])       # a partly filled page, another of the same parent, an empty parent
    for _ in range(3):
        c.add([4, 3, 1, 0], [1, 1, 1, 1])
    c.release([0, 5])
    c.add([7], [50], strided=True)
    c.compact()
    c.compact()                                # nothing left to move
    c.add([1, 3, 4, 7], [17, 16, 1, 2])
    c.release([1, 3, 4, 7, 2, 6])
    assert (c.m.ref == 0).all()
    c.compact()
    c.add([0], [100])


@pytest.mark.parametrize("page", [16, 64, 256])
def test_page_edges(sla, handle, page):
    c = Pair(sla, handle, page=page, n_pages=20, width=5)
    c.add([0, 1, 2], [page, page - 1, 1])
    c.add([0, 1, 2], [0, 1, page - 1])
    c.fork([0, 1], [3, 4])                     # only full pages: nothing is copied
    c.add([0, 1, 2, 3], [1, page, page + 1, 1])
    c.fork([0], [5])
    c.release([0])
    c.compact()


def test_refused_sequences_stay_as_they_were(sla):
    h = sla.Handle(0, 1 << 26)
    c = Pair(sla, h, n_pages=6, width=4)
    assert list(c.add([0, 1], [40, 20])) == [0, 0]
    assert sla.sla_poll_status(h) == sla.SLA_OK
    # one page is left: 1 wants one and gets it, 2 wants two and 0 one more than there are, 3 wants none
    assert list(c.add([1, 2, 0, 3], [13, 17, 9, 0])) == [20, -1, -1, 0]
    assert sla.sla_poll_status(h) == sla.SLA_ERR_CACHE_FULL
    assert list(c.add([0, 1], [8, 100])) == [40, -1]        # fits the last page; a table row of four pages is too short
    assert sla.sla_poll_status(h) == sla.SLA_ERR_CACHE_FULL
    # no page for the copy of a partly filled one
    pairs = sla.sla_cache_fork(h, c.cache, U.device_ints([1, 0]), U.device_ints([4, 5]))
    assert np.array_equal(pairs.cpu().numpy(), c.m.fork([1, 0], [4, 5]))
    assert c.m.n[4] == 0 and c.m.n[5] == 48
    c.rows[5] = list(c.rows[0])
    c.same()
    assert sla.sla_poll_status(h) == sla.SLA_ERR_CACHE_FULL
    # a slot that is not empty
    sla.sla_cache_fork(h, c.cache, U.device_ints([0]), U.device_ints([1]))
    c.same()
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    # slots outside the cache
    first = sla.sla_cache_extend(h, c.cache, U.device_ints([0, 1, 2]), seq=U.device_ints([-1, 8]))
    assert list(first.cpu()) == [-1, -1] and sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    sla.sla_cache_release(h, c.cache, U.device_ints([99]))
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    sla.sla_cache_copy(h, c.cache, U.device_ints([[0], [6]]))
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    c.same()
    # released twice in one call: every reference goes once
    sla.sla_cache_release(h, c.cache, U.device_ints([0, 0]))
    c.m.release([0])
    c.rows[0] = []
    c.same()
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()


def test_copy_follows_the_pairs_of_another_layer(sla, handle):
    """fork and compact run on one layer; a second layer's pools follow by the pairs they return."""
    c = Pair(sla, handle)
    k2, v2 = U.make_pools(40, 2, 16, 64, torch.bfloat16, seed=9)
    other = sla.make_cache(k2, v2, *c.dev)
    c.add([0, 1], [40, 20])
    before = [k2[int(c.m.table[0, p // 16]), :, p % 16].clone() for p in range(40)]
    pairs = c.fork([0, 0], [2, 3])
    sla.sla_cache_copy(handle, other, pairs)
    c.release([0, 1])
    sla.sla_cache_copy(handle, other, c.compact())
    for s in (2, 3):
        for p in range(40):
            assert torch.equal(k2[int(c.m.table[s, p // 16]), :, p % 16], before[p])


@pytest.mark.parametrize("n_pages", [5000, 70000])
def test_many_pages_and_sequences(sla, n_pages):
    """Pools of several chunks, more sequences than a warp or a CTA has threads."""
    h = sla.Handle(0, 1 << 26)
    rs = np.random.RandomState(n_pages)
    slots = 1500
    m = U.Model(n_pages, 16, slots, 40)
    k, v = U.make_pools(n_pages, 1, 16, 64, torch.bfloat16)
    dev = [U.device_ints(a) for a in (m.table, m.n, m.ref)]
    cache = sla.make_cache(k, v, *dev)
    for _ in range(3):
        seq = rs.permutation(slots)
        new = rs.randint(0, 40, slots)
        first = sla.sla_cache_extend(h, cache, U.device_ints(np.concatenate([[0], np.cumsum(new)])), seq=U.device_ints(seq))
        assert np.array_equal(first.cpu().numpy(), m.extend(seq, new))
    gone = rs.permutation(slots)[:700]
    sla.sla_cache_release(h, cache, U.device_ints(gone))
    m.release(gone)
    kids, parents = gone[:300], rs.permutation(np.setdiff1d(np.arange(slots), gone))[:300]
    pairs = sla.sla_cache_fork(h, cache, U.device_ints(parents), U.device_ints(kids))
    assert np.array_equal(pairs.cpu().numpy(), m.fork(parents, kids))
    old_k, old_table = k.clone(), m.table.copy()
    pairs = sla.sla_cache_compact(h, cache)
    assert np.array_equal(pairs.cpu().numpy(), m.compact())
    for a, b in zip(dev, (m.table, m.n, m.ref)):
        assert np.array_equal(a.cpu().numpy(), b)
    on = old_table >= 0
    assert torch.equal(k[torch.from_numpy(m.table[on].astype(np.int64)).cuda()], old_k[torch.from_numpy(old_table[on].astype(np.int64)).cuda()])
    sla.sla_poll_status(h)
    h.close()


def test_refusals(sla, handle):
    c = Pair(sla, handle)
    k = torch.zeros(4, 2, 24, 64, dtype=torch.bfloat16, device="cuda:0")
    t, n, r = U.device_ints([[0, 1]]), U.device_ints([0]), U.device_ints([0] * 4)
    odd = sla.make_cache(k, k.clone(), t, n, r)                      # 24 tokens a page
    with pytest.raises(sla.SlaError):
        sla.sla_cache_extend(handle, odd, U.device_ints([0, 1]))
    assert sla.sla_paged_workspace_bytes(odd, 2, 1, 1) == 0
    assert sla.sla_paged_workspace_bytes(c.cache, 3, 1, 1) == 0 and sla.sla_paged_workspace_bytes(c.cache, 2, 1, 1) > 0
    for bad in (lambda: sla.make_cache(k, k[:3], t, n, r), lambda: sla.make_cache(k, k.clone(), t.long(), n, r),
                lambda: sla.make_cache(k, k.clone(), t, n, r[:2]), lambda: sla.make_cache(k, k.transpose(2, 3), t, n, r)):
        with pytest.raises(ValueError):
            bad()
    cu, first = U.device_ints([0, 2]), U.device_ints([0])
    new = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    with pytest.raises(ValueError):
        sla.sla_cache_append(handle, c.cache, cu, first, new[:, :1], new[:, :1])
    with pytest.raises(ValueError):
        sla.sla_cache_append(handle, c.cache, cu, first, new.float(), new.float())
    with pytest.raises(ValueError):
        sla.sla_cache_append(handle, c.cache, cu, U.device_ints([0, 0]), new, new)
    with pytest.raises(ValueError):
        sla.sla_cache_fork(handle, c.cache, U.device_ints([0, 1]), U.device_ints([2]))
    small = sla.Handle(0, 256)
    with pytest.raises(sla.SlaError) as e:
        sla.sla_cache_compact(small, c.cache)
    assert e.value.status == -3
    small.close()


# ---- the span decode step over the cache -----------------------------------------------------------------


def contiguous(k, table, n, page):
    pages = torch.from_numpy(table[: -(-n // page)].astype(np.int64)).cuda()
    return k[pages].transpose(0, 1).reshape(1, k.shape[1], -1, k.shape[3])[:, :, :n].contiguous()


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("mode", ["union", "window", "gated", "exponents"])
def test_span_step_equals_the_step_over_each_sequence_alone(sla, dtype, d, mode):
    """Every sequence's step is the one of sla_decode_step on a contiguous copy of it: the same anchors and scores, outputs within
    rounding."""
    import test_gpu_paged_attention as A
    h = sla.Handle(0, 1 << 28)
    n = [1, 2, 100, 1031, 0, 5000, 777]
    cache, k, v, table, _, _ = A.build(sla, n, [0] * len(n), dtype=dtype, d=d, page=32, G=4)
    kw = {"union": {}, "window": dict(window=33), "gated": dict(window=35, mode=sla.SLA_PER_SPAN),
          "exponents": dict(search_exponent=0.4, span_exponent=0.6)}[mode]
    params = sla.make_params(4, 0, fwd_factor=1, head_dim=d, **kw)
    g = torch.Generator(device="cuda:0")
    q_s, q = (torch.empty(len(n), 8, d, dtype=dtype, device="cuda:0").normal_(generator=g) for _ in range(2))
    need = sla.sla_paged_workspace_bytes(cache, 8, len(n), len(n), params=params)
    assert need <= 1 << 28
    order = [6, 0, 5, 4, 3, 2, 1]
    out, lse, anchor, score = sla.sla_paged_decode_step(h, q_s, q, cache, params, seq=U.device_ints(order), max_tokens=6000)
    assert sla.sla_poll_status(h) == sla.SLA_OK
    for x, s in enumerate(order):
        if n[s] == 0:
            assert (out[x] == 0).all() and (lse[x] == -math.inf).all() and (anchor[x] == -1).all() and (score[x] == -math.inf).all()
            continue
        one = sla.sla_decode_step(h, q_s[x:x + 1], q[x:x + 1], contiguous(k, table[s], n[s], 32), contiguous(v, table[s], n[s], 32), n[s], params)
        assert torch.equal(one[2][0], anchor[x]) and torch.equal(one[3][0], score[x])
        # the two differ in how a head's tokens are shared out: fp32 sums of at most n terms in another order, one rounding of the result
        big = v.float().nan_to_num().abs().max()
        tol = 2.0 ** -8 * one[0][0].float().abs() + 1e-6 * big if dtype == torch.bfloat16 else 2e-6 * big
        assert ((one[0][0].float() - out[x].float()).abs() <= tol).all()
        a, b = one[1][0], lse[x]
        assert torch.equal(torch.isfinite(a), torch.isfinite(b)) and ((a - b).abs().nan_to_num() <= 4e-6 * (1 + a.abs().nan_to_num(posinf=0, neginf=0))).all()
    h.close()


def test_span_step_refusals(sla):
    import test_gpu_paged_attention as A
    h = sla.Handle(0, 1 << 26)
    cache, k, v, table, _, _ = A.build(sla, [100, 60], [0, 0])
    params = sla.make_params(4, 0)
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda:0")
    # longer than the bound, or a slot outside the cache: flagged, no result
    out, lse, anchor, _ = sla.sla_paged_decode_step(h, q, q, cache, params, max_tokens=80)
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    assert (out[0] == 0).all() and (anchor[0] == -1).all() and (anchor[1] >= 0).all()
    sla.sla_paged_decode_step(h, q, q, cache, params, seq=U.device_ints([5, -1]))
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    for bad in (lambda: sla.sla_paged_decode_step(h, q, q, cache, sla.make_params(65, 0)),
                lambda: sla.sla_paged_decode_step(h, q, q, cache, params, max_tokens=0),
                lambda: sla.sla_paged_decode_step(h, q[:, :7], q[:, :7], cache, params)):
        with pytest.raises(sla.SlaError):
            bad()
    with pytest.raises(ValueError):
        sla.sla_paged_decode_step(h, q.float(), q, cache, params)
    h.close()


@pytest.mark.parametrize("mode,n_seqs,hkv,G", [("union", 500, 8, 4), ("gated", 130, 8, 4), ("union", 300, 3, 16)])
def test_span_step_of_more_sequences_than_one_launch_takes(sla, mode, n_seqs, hkv, G):
    """The same anchors and scores as by parts of 20 sequences, outputs within rounding; slots in order and by name."""
    import test_gpu_paged_attention as A
    rs = np.random.RandomState(n_seqs)
    n = rs.randint(0, 300, n_seqs).tolist()
    cache, k, v, table, _, _ = A.build(sla, n, [0] * n_seqs, d=64, hkv=hkv, G=G, page=32)
    params = sla.make_params(8, 0, head_dim=64, **(dict(window=9, mode=sla.SLA_PER_SPAN) if mode == "gated" else {}))
    g = torch.Generator(device="cuda:0")
    q_s, q = (torch.empty(n_seqs, hkv * G, 64, dtype=torch.bfloat16, device="cuda:0").normal_(generator=g) for _ in range(2))
    h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, hkv * G, n_seqs, n_seqs, params=params))
    for order in (None, rs.permutation(n_seqs)):
        slots = np.arange(n_seqs) if order is None else order
        out, lse, anchor, score = sla.sla_paged_decode_step(h, q_s, q, cache, params, max_tokens=400,
                                                            seq=None if order is None else U.device_ints(order))
        assert sla.sla_poll_status(h) == sla.SLA_OK
        for x in range(0, n_seqs, 20):
            part = sla.sla_paged_decode_step(h, q_s[x:x + 20], q[x:x + 20], cache, params, max_tokens=400, seq=U.device_ints(slots[x:x + 20]))
            assert torch.equal(part[2], anchor[x:x + 20]) and torch.equal(part[3], score[x:x + 20])
            # sums of at most 300 terms in another order, one rounding of the result each
            big = v.float().nan_to_num().abs().max()
            assert ((part[0].float() - out[x:x + 20].float()).abs() <= 2.0 ** -7 * part[0].float().abs() + 1e-5 * big).all()
            a, b = part[1], lse[x:x + 20]
            assert torch.equal(torch.isfinite(a), torch.isfinite(b)) and ((a - b).abs().nan_to_num() <= 4e-6 * (1 + a.abs().nan_to_num(posinf=0, neginf=0))).all()
    h.close()


def test_a_refusal_beside_another_error_is_reported_too(sla):
    h = sla.Handle(0, 1 << 26)
    c = Pair(sla, h, n_pages=2, width=4)
    for _ in range(2):
        first = sla.sla_cache_extend(h, c.cache, U.device_ints([0, 40, 41]), seq=U.device_ints([0, 9]))   # three pages; no such slot
        assert list(first.cpu()) == [-1, -1]
        assert [sla.sla_poll_status(h) for _ in range(3)] == [sla.SLA_ERR_DEVICE_INDEX, sla.SLA_ERR_CACHE_FULL, sla.SLA_OK]
    # one refused while the other waits to be reported: once more, not twice
    sla.sla_cache_extend(h, c.cache, U.device_ints([0, 40, 41]), seq=U.device_ints([0, 9]))
    assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_INDEX
    sla.sla_cache_extend(h, c.cache, U.device_ints([0, 40]), seq=U.device_ints([0]))
    assert [sla.sla_poll_status(h) for _ in range(2)] == [sla.SLA_ERR_CACHE_FULL, sla.SLA_OK]
    h.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [3, 2, 1, 4], [90, 40, 17, 33]])
def test_a_refused_sequence_is_not_attended(sla, dtype, new):
    """With what extend returned: the rows of a refused sequence are 0 and -inf, the others as in a call without it."""
    from paper_2601_18401_b200.paged import PagedCache
    c = PagedCache(12, 6, 16 * 8, n_q_heads=8, n_kv_heads=2, page_tokens=16, dtype=dtype, max_new=400, params=sla.make_params(4, 0))
    g = torch.Generator(device="cuda:0")
    rand = lambda n, h: torch.empty(n, h, 128, dtype=dtype, device="cuda:0").normal_(generator=g)  # noqa: E731
    start, slots = [16, 32, 15, 16], [4, 0, 2, 5]
    cu = U.device_ints(np.concatenate([[0], np.cumsum(start)]))
    c.append(cu, c.extend(cu, seq=U.device_ints(slots)), rand(sum(start), 2), rand(sum(start), 2), seq=U.device_ints(slots))
    c.ref[5:] = 1                                            # two free pages are left
    c.ref[6:8] = 0
    if new[0] == 1:
        c.ref[7] = 1                                         # or one
    cu = U.device_ints(np.concatenate([[0], np.cumsum(new)]))
    first = c.extend(cu, seq=U.device_ints(slots))
    ok = [f >= 0 for f in first.tolist()]
    assert c.poll() == sla.SLA_ERR_CACHE_FULL and 0 < sum(ok) + (new[0] == 90) and not all(ok)
    kn, vn, q, q_s = rand(sum(new), 2), rand(sum(new), 2), rand(sum(new), 8), rand(sum(new), 8)
    c.append(cu, first, kn, vn, seq=U.device_ints(slots))
    n = [int(x) for x in c.n_tokens[torch.tensor(slots).cuda()]]
    seen = [x if o else 0 for x, o in zip(n, ok)]
    table = c.table.cpu().numpy()[slots]
    for bound in (max(new), sum(new)):
        out, lse = c.attend(q, cu, seq=U.device_ints(slots), max_new=bound, first=first)
        U.check_attention(out, lse, U.attention_reference(q, c.k, c.v, table, seen, new, 4, 0, 128 ** -0.5, 16), dtype)
    out, lse, anchor, score = c.step(q_s[:4], q[:4], seq=U.device_ints(slots), max_tokens=128, first=first)
    whole = c.step(q_s[:4], q[:4], seq=U.device_ints(slots), max_tokens=128)
    for x in range(4):
        if ok[x]:
            assert all(torch.equal(a[x], b[x]) for a, b in zip((out, lse, anchor, score), whole))
        else:
            assert (out[x] == 0).all() and (lse[x] == -math.inf).all() and (anchor[x] == -1).all() and (score[x] == -math.inf).all()
    assert c.poll() == sla.SLA_OK
    with pytest.raises(ValueError):
        c.attend(q, cu, seq=U.device_ints(slots), first=first[:3])


def test_canaries_of_the_paged_calls(sla):
    """Gaps between the scratch regions of every call that has some: intact after it, the same results as without, and a damaged one
    is reported.  Handles of exactly the size asked for."""
    import test_gpu_paged_attention as A
    params = sla.make_params(4, 0)
    results = []
    for on in (False, True):
        got = []
        for dtype, lens in ((torch.bfloat16, A.SINGLE), (torch.bfloat16, A.CHUNKS), (torch.bfloat16, ([9000, 40], [70, 33])), (torch.float32, A.CHUNKS), (torch.float32, ([6000], [70]))):
            cache, k, v, table, q, cu = A.build(sla, *lens, dtype=dtype)
            h = sla.Handle(0, sla.sla_paged_workspace_bytes(cache, 8, len(lens[0]), q.shape[0], params=params))
            sla.sla_set_debug_canaries(h, on)
            got += sla.sla_paged_attention(h, q, cache, cu, max_new=max(lens[1]))
            if on:
                assert sla.sla_poll_status(h) == sla.SLA_OK
                sla.sla_selftest_canary_trip(h)
                assert sla.sla_poll_status(h) == sla.SLA_ERR_DEVICE_OVERRUN
            got += sla.sla_paged_decode_step(h, q[:len(lens[0])], q[:len(lens[0])], cache, params)
            assert sla.sla_poll_status(h) == sla.SLA_OK
            h.close()
        c = Pair(sla, sla.Handle(0, sla.sla_paged_workspace_bytes(Pair(sla, None).cache, 2, 8, 100)))
        sla.sla_set_debug_canaries(c.h, on)

        def checked():
            if on:
                assert sla.sla_poll_status(c.h) == sla.SLA_OK
                sla.sla_selftest_canary_trip(c.h)
                assert sla.sla_poll_status(c.h) == sla.SLA_ERR_DEVICE_OVERRUN
        c.add([0, 2, 5], [40, 0, 33])
        checked()
        c.fork([0, 5, 0], [1, 3, 4])
        checked()
        c.release([0])
        c.compact()
        checked()
        assert sla.sla_poll_status(c.h) == sla.SLA_OK
        c.h.close()
        results.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*results, strict=True))


def test_layers_that_share_a_table(sla):
    """Three layers of one model: table, lengths and counts in common, room, forks, ends and compaction once, copies, appends,
    attention and span steps for every layer."""
    from paper_2601_18401_b200.paged import PagedCache
    kw = dict(n_q_heads=8, n_kv_heads=2, page_tokens=16, max_new=400)
    first_layer = PagedCache(60, 6, 300, params=sla.make_params(4, 0), **kw)
    layers = [first_layer] + [PagedCache(60, 6, 300, share=first_layer, **kw) for _ in range(2)]
    assert all(c.table is first_layer.table and c.handle is first_layer.handle and c.params is first_layer.params for c in layers)
    g = torch.Generator(device="cuda:0")
    rand = lambda n, h: torch.empty(n, h, 128, dtype=torch.bfloat16, device="cuda:0").normal_(generator=g)  # noqa: E731
    rows = [{s: [] for s in range(6)} for _ in layers]       # (k, v) of every position, by layer and slot

    def add(slots, new):
        cu = U.device_ints(np.concatenate([[0], np.cumsum(new)]))
        first = layers[0].extend(cu, seq=U.device_ints(slots))
        assert (first >= 0).all()
        for c, mine in zip(layers, rows):
            kn, vn, q = rand(sum(new), 2), rand(sum(new), 2), rand(sum(new), 8)
            c.append(cu, first, kn, vn, seq=U.device_ints(slots))
            at = 0
            for s, x in zip(slots, new):
                mine[s] += [(kn[at + r], vn[at + r]) for r in range(x)]
                at += x
            out, lse = c.attend(q, cu, seq=U.device_ints(slots), max_new=max(new), first=first)
            n = [len(mine[s]) for s in slots]
            k, v = (torch.zeros(len(slots), 2, 320, 128, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))   # a page each
            for x, s in enumerate(slots):
                k[x, :, :n[x]] = torch.stack([a for a, _ in mine[s]], 1)
                v[x, :, :n[x]] = torch.stack([b for _, b in mine[s]], 1)
            U.check_attention(out, lse, U.attention_reference(q, k, v, np.arange(len(slots))[:, None], n, new, 4, 0, 128 ** -0.5, 320), torch.bfloat16)
            if max(new) == 1:
                got = c.step(q, q, seq=U.device_ints(slots), max_tokens=300, first=first)
                for x in range(len(slots)):
                    one = sla.sla_decode_step(c.handle, q[x:x + 1], q[x:x + 1], k[x:x + 1, :, :n[x]].contiguous(), v[x:x + 1, :, :n[x]].contiguous(), n[x], c.params)
                    assert torch.equal(one[2][0], got[2][x]) and torch.equal(one[3][0], got[3][x])
                    assert ((one[0][0].float() - got[0][x].float()).abs() <= 2.0 ** -8 * one[0][0].float().abs() + 1e-5).all()

    add([0, 3], [100, 37])
    pairs = layers[0].fork(U.device_ints([0, 3, 0]), U.device_ints([1, 2, 5]))
    for c, mine in zip(layers, rows):
        if c is not layers[0]:
            c.copy(pairs)
        mine[1], mine[2], mine[5] = list(mine[0]), list(mine[3]), list(mine[0])
    add([1, 2, 5, 0], [1, 1, 1, 1])
    layers[0].release(U.device_ints([0, 3]))
    for mine in rows:
        mine[0], mine[3] = [], []
    pairs = layers[0].compact()
    for c in layers[1:]:
        c.copy(pairs)
    add([5, 2, 1], [1, 1, 1])
    add([3, 1], [60, 20])
    assert layers[0].poll() == sla.SLA_OK
    for bad in (dict(page_tokens=32), dict(n_slots=5), dict(max_tokens=400), dict(n_pages=61)):
        a = dict(n_pages=60, n_slots=6, max_tokens=300, share=first_layer) | kw | bad
        with pytest.raises(ValueError):
            PagedCache(**a)


def test_queries_that_lie_over_one_another_are_refused(sla):
    """Broadcast queries: the output has their strides, and its rows would be written by several sequences or heads."""
    import test_gpu_paged_attention as A
    h = sla.Handle(0, 1 << 26)
    cache, k, v, table, _, _ = A.build(sla, [100, 60], [0, 0])
    params = sla.make_params(4, 0)
    one = torch.ones(1, 8, 128, dtype=torch.bfloat16, device="cuda:0")
    for q in (one.expand(2, 8, 128), one[:, :1].repeat(2, 1, 1).expand(2, 8, 128), one[:, :1].expand(2, 8, 128)):
        with pytest.raises(sla.SlaError) as e:
            sla.sla_paged_decode_step(h, q, q, cache, params)
        assert e.value.status == -1
        with pytest.raises(sla.SlaError) as e:
            sla.sla_paged_attention(h, q, cache)
        assert e.value.status == -1
    sla.sla_paged_decode_step(h, one.expand(1, 8, 128), one, cache, params, seq=U.device_ints([1]))   # a single sequence has no such stride
    assert sla.sla_poll_status(h) == sla.SLA_OK
    h.close()
