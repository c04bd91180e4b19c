"""Host-only checks of the paged calls: workspace sizes, refusals before anything is launched, and the model the GPU tests use."""
import ctypes as C

import numpy as np
import pytest
import torch

import paged_util as U


@pytest.fixture(scope="module")
def sla():
    from paper_2601_18401_b200 import build
    build.build_library()
    import paper_2601_18401_b200 as sla_pkg
    return sla_pkg


def cache_of(sla, n_pages=64, hkv=8, page=64, d=128, slots=4, width=32, dtype=torch.bfloat16):
    k = torch.empty(n_pages, hkv, page, d, dtype=dtype)
    ints = [torch.zeros(slots, width, dtype=torch.int32), torch.zeros(slots, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)]
    return sla.make_cache(k, k.clone(), *ints)


def test_workspace_sizes(sla):
    c = cache_of(sla)
    step, chunk = sla.sla_paged_workspace_bytes(c, 32, 4, 4), sla.sla_paged_workspace_bytes(c, 32, 4, 4096)
    assert 0 < step <= chunk < 1 << 30
    assert sla.sla_paged_workspace_bytes(c, 32, 4, 4, params=sla.make_params(8, 0)) >= step
    assert sla.sla_paged_workspace_bytes(cache_of(sla, dtype=torch.float32, d=64), 8, 4, 100) > 0


@pytest.mark.parametrize("change", [dict(page=8), dict(page=48), dict(page=512), dict(d=96)])
def test_unsupported_shapes_have_no_workspace(sla, change):
    assert sla.sla_paged_workspace_bytes(cache_of(sla, **change), 8, 1, 1) == 0


def test_invalid_arguments_have_no_workspace(sla):
    c = cache_of(sla)
    assert sla.sla_paged_workspace_bytes(c, 12, 1, 1) == 0           # not a multiple of the KV heads
    assert sla.sla_paged_workspace_bytes(c, 8 * 17, 1, 1) == 0       # groups of 17
    assert sla.sla_paged_workspace_bytes(c, 32, -1, 1) == 0
    assert sla.sla_paged_workspace_bytes(c, 32, 1, 1, params=sla.make_params(65, 0)) == 0
    c.reserved = 1
    assert sla.sla_paged_workspace_bytes(c, 32, 1, 1) == 0
    c.reserved, c.stride_t = 0, 60
    assert sla.sla_paged_workspace_bytes(c, 32, 1, 1) == 0
    c.stride_t, c.table_width = 128, 1 << 30
    assert sla.sla_paged_workspace_bytes(c, 32, 1, 1) == 0
    c.table_width, c.n_pages = 32, 1 << 30
    assert sla.sla_paged_workspace_bytes(c, 32, 1, 1) == 0


def test_a_missing_handle_is_refused(sla):
    lib, c = sla.load_library(), cache_of(sla)
    b = sla.sla_batch_t(1, 1, 1, 0, None, None)
    ca, ba = C.addressof(c), C.addressof(b)
    assert lib.sla_cache_extend(None, ca, ba, 16, None) == -1
    assert lib.sla_cache_append(None, ca, ba, 16, 16, 16, 128, 128, None) == -1
    assert lib.sla_cache_release(None, ca, 16, 1, None) == -1
    assert lib.sla_cache_fork(None, ca, 16, 16, 1, 16, None) == -1
    assert lib.sla_cache_compact(None, ca, 16, None) == -1
    assert lib.sla_cache_copy(None, ca, 16, 1, None) == -1
    assert lib.sla_paged_attention(None, 16, ca, ba, 8, 128, 128, 0, 1.0, 16, 16, None) == -1
    p = sla.make_params(4, 0)
    assert lib.sla_paged_decode_step(None, 16, 16, ca, ba, 64, 8, 128, 128, C.byref(p), 16, 16, 16, 16, None) == -1
    assert lib.sla_status_string(-8) == b"SLA_ERR_CACHE_FULL"


def test_make_cache_checks_its_tensors(sla):
    k = torch.empty(4, 2, 16, 64, dtype=torch.bfloat16)
    t, n, r = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    sla.make_cache(k, k.clone(), t, n, r)
    for bad in ((k, k.float(), t, n, r), (k, k[:, :, :8], t, n, r), (k, k.transpose(1, 2).contiguous().transpose(1, 2), t, n, r),
                (k, k.clone(), t[:, ::2], n, r), (k, k.clone(), t, n[:2], r), (k, k.clone(), t, n, r.float()),
                (k.half(), k.half(), t, n, r)):
        with pytest.raises((ValueError, TypeError)):
            sla.make_cache(*bad)


def test_host_tensors_are_refused(sla):
    """A cache or an argument in host memory is refused by the binding: no kernel ever gets its address."""
    c = cache_of(sla)
    i = torch.zeros(4, dtype=torch.int32)
    new, q = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(4, 32, 128, dtype=torch.bfloat16)
    for call in (lambda: sla.sla_cache_extend(None, c), lambda: sla.sla_cache_append(None, c, None, i, new, new),
                 lambda: sla.sla_cache_release(None, c, i), lambda: sla.sla_cache_fork(None, c, i, i),
                 lambda: sla.sla_cache_compact(None, c), lambda: sla.sla_cache_copy(None, c, torch.zeros(2, 3, dtype=torch.int32)),
                 lambda: sla.sla_paged_attention(None, q, c), lambda: sla.sla_paged_decode_step(None, q, q, c, sla.make_params(4, 0))):
        with pytest.raises(ValueError):
            call()


def test_model_of_the_bookkeeping():
    """The model by hand: pages of two tokens."""
    m = U.Model(6, 2, 4, 4)
    assert list(m.extend([0, 1], [3, 2])) == [0, 0]
    assert m.table[0].tolist() == [0, 1, -1, -1] and m.table[1].tolist() == [2, -1, -1, -1]
    assert m.fork([0, 1], [2, 3]).tolist() == [[1, -1], [3, -1]]
    assert m.table[2].tolist() == [0, 3, -1, -1] and m.table[3].tolist() == [2, -1, -1, -1]
    assert m.ref.tolist() == [2, 1, 2, 1, 0, 0] and m.n.tolist() == [3, 2, 3, 2]
    m.release([0])
    assert m.ref.tolist() == [1, 0, 2, 1, 0, 0]
    assert m.compact()[:, :2].tolist() == [[3, -1], [1, -1]]
    assert m.table[2].tolist() == [0, 1, -1, -1] and m.ref.tolist() == [1, 1, 2, 0, 0, 0]
    assert list(m.extend([2, 3, 0], [4, 9, 3])) == [3, -1, -1]       # 2 takes two of the three pages; 3's row is too short; 0 wants two
    assert m.n.tolist() == [0, 2, 7, 2]


def test_reference_against_dense_attention():
    """The row-by-row reference equals softmax over the whole sequence with a mask."""
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(5, 2, 16, 8, generator=g) for _ in range(2))
    q = torch.randn(20, 4, 8, generator=g)
    table = np.array([[3, 0, -1], [4, 1, -1]], dtype=np.int32)
    n, new = [30, 17], [12, 8]
    out, lse, *_ = U.attention_reference(q, k, v, table, n, new, 2, 5, 0.3, 16)
    r = 0
    for x in range(2):
        kk, vv = (p[torch.from_numpy(table[x, :2].astype(np.int64))].transpose(1, 2).reshape(-1, 2, 8)[:n[x]].double().repeat_interleave(2, 1) for p in (k, v))
        z = torch.einsum("thd,jhd->htj", q[r:r + new[x]].double(), kk) * 0.3
        p, j = torch.arange(n[x] - new[x], n[x])[:, None], torch.arange(n[x])
        z = z.masked_fill(~((j <= p) & (j > p - 5)), -np.inf)
        assert torch.allclose(out[r:r + new[x]], torch.einsum("htj,jhd->thd", z.softmax(-1), vv))
        assert torch.allclose(lse[r:r + new[x]], z.logsumexp(-1).T)
        r += new[x]


def test_tiles_of_a_unit_do_not_overflow(tmp_path):
    """unit_tiles, compiled for the host with signed overflow as an error, against plain Python: positions from below zero to the
    longest sequence, windows up to the largest int."""
    import os
    import subprocess
    from paper_2601_18401_b200 import build
    src, exe = tmp_path / "t.cu", tmp_path / "t"
    src.write_text("""
#include <stdio.h>
#include "sla_paged.cuh"
int main() {
    int n, q, t0, t1, window, shift, lo, hi;
    while (scanf("%d %d %d %d %d %d", &n, &q, &t0, &t1, &window, &shift) == 6) {
        sla::unit_tiles(n, q, t0, t1, window, shift, lo, hi);
        printf("%d %d\\n", lo, hi);
    }
}
""")
    subprocess.run([build._nvcc(), "-std=c++17", "-Xcompiler", "-fsanitize=signed-integer-overflow,-fno-sanitize-recover=all", "-I", build.CSRC,
                    "-I", os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True, capture_output=True)
    top = 2 ** 31 - 1025
    cases = [(n, q, t0, min(t0 + 32, q), w, s) for n in (0, 1, 10, 129, 5000, top) for q in (1, 4, 20, 5000) for t0 in (0, 3, 64, 4990) if t0 < q
             for w in (0, 1, 7, 128, 5000, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1) for s in (6, 7)]
    r = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    for (n, q, t0, t1, w, s), line in zip(cases, r.stdout.splitlines(), strict=True):
        p0, end = n - q + t0, n - q + t1
        lo = (max(p0 - w + 1, 0) if w else 0) >> s
        assert line == f"{lo} {max(-(-end >> s) if end > 0 else lo, lo)}", (n, q, t0, t1, w, s)


def test_every_call_wants_a_slot_per_sequence(sla):
    """seq shorter or longer than the sequences of cu_new: refused before its address goes anywhere."""
    c = cache_of(sla)
    cu = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    new, q = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    from paper_2601_18401_b200 import binding as B
    for n in (2, 4):
        seq = torch.arange(n, dtype=torch.int32)
        with pytest.raises(ValueError, match="one slot per sequence"):
            sla.sla_cache_extend(None, c, cu, seq=seq)
        with pytest.raises(ValueError, match="one slot per sequence"):
            B._batch(cu, 3, None, seq)
        with pytest.raises(ValueError, match="one slot per sequence"):
            B._batch(None, 3, 1, seq)
    with pytest.raises(ValueError, match="contiguous int32"):
        sla.sla_cache_extend(None, c, cu, seq=torch.arange(3))
    for call in (lambda s: sla.sla_cache_append(None, c, cu, torch.zeros(3, dtype=torch.int32), new, new, seq=s),
                 lambda s: sla.sla_paged_attention(None, q, c, cu, seq=s), lambda s: sla.sla_paged_decode_step(None, q, q, c, sla.make_params(4, 0), seq=s)):
        with pytest.raises(ValueError):
            call(torch.arange(2, dtype=torch.int32))


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_the_current_stream_without_torchs_private_names(monkeypatch, missing):
    from types import SimpleNamespace

    from paper_2601_18401_b200 import binding as B
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=4711))
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.setattr(torch._C, name, lambda *a: 0, raising=False)
    monkeypatch.delattr(torch._C, missing)
    assert B._stream_ptr(None) == 4711
    assert B._stream_ptr(SimpleNamespace(cuda_stream=12)) == 12
