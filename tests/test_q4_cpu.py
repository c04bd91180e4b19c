"""Host-only checks of the paged cache in four bits: the model of its format that the GPU tests use, workspaces and refusals."""
import ctypes as C

import pytest
import torch

import q4_util as Q


@pytest.fixture(scope="module")
def sla():
    from paper_2601_18401_b200 import build
    build.build_library()
    import paper_2601_18401_b200 as sla_pkg
    return sla_pkg


def cache_of(sla, n_pages=16, hkv=4, page=64, d=128, slots=4, width=8, dtype=torch.bfloat16, **kw):
    k = torch.zeros(n_pages, hkv, sla.q4_plane_bytes(page, d), dtype=torch.uint8)
    ints = [torch.zeros(slots, width, dtype=torch.int32), torch.zeros(slots, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)]
    return sla.make_cache_q4(k, k.clone(), *ints, page_tokens=page, head_dim=d, dtype=dtype)


def test_model_scales_by_hand():
    s = Q.scales(torch.tensor([0.0, 7.5, 7.6, 1.0, 2.0 ** -60, 7.5 * 31 * 2.0 ** 35, 7.6 * 31 * 2.0 ** 35, float("inf"), float("nan")], dtype=torch.float64))
    assert s[:6].tolist() == [2.0 ** -40, 1.0, 1 + 1 / 16, 18 / 128, 2.0 ** -40, 31 * 2.0 ** 35]   # 1 / 7.5 = 17.07 / 128
    assert torch.isnan(s[6:]).all()


def test_model_rounds_halves_away_and_stays_within_half_a_scale():
    x = torch.zeros(1, 64, dtype=torch.float64)
    x[0, :8] = torch.tensor([7.5, 0.5, -0.5, 1.5, -2.5, 6.5, 0.49, -7.5])
    x[0, 32:34] = torch.tensor([3.0, -1.0])
    codes, s = Q.quantise(x)
    assert s.tolist() == [[1.0, 26 / 64]]                               # 3 / 7.5 = 25.6 / 64
    assert codes[0, :8].tolist() == [7, 1, -1, 2, -3, 7, 0, -7] and codes[0, 32:34].tolist() == [7, -2]
    g = torch.Generator().manual_seed(1)
    y = torch.randn(500, 128, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(500, 1, generator=g, dtype=torch.float64))
    c, s = Q.quantise(y)
    assert ((Q.dequantise(c, s) - y).abs() <= (s / 2).repeat_interleave(32, -1) * (1 + 1e-12)).all()
    assert (Q.dequantise(c, s).bfloat16().double() == Q.dequantise(c, s)).all()     # a bf16 number


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("values", [False, True])
def test_model_planes_go_there_and_back(d, values):
    g = torch.Generator().manual_seed(2)
    c, s = Q.quantise(torch.randn(3, 2, 16, d, generator=g))
    planes = Q.pack(c, s, values)
    assert planes.shape == (3, 2, 16 * (d // 2 + d // 16))
    assert torch.equal(Q.unpack(planes, 16, d, values), Q.dequantise(c, s))
    # by hand: dimension 32 + 8 + 2 * 3 + 1 = 47 is code 3 of the word (g 1, c 1, h 1)
    c, s = torch.zeros(16, d), torch.ones(16, d // 32)
    c[5, 47] = -5
    words = Q.pack(c, s, values)[: 16 * d // 2].view(torch.int16).view(16, d // 4)
    at = (2 * 1 + 1) * (d // 32) + 1 if values else 2 * (1 * (d // 32) + 1) + 1
    assert words[5, at] == (5 << 11) + (1 << 6) and (words != 0).sum() == 1


def test_plane_bytes(sla):
    assert sla.q4_plane_bytes(64, 128) == 64 * 72 and sla.q4_plane_bytes(16, 64) == 16 * 36


def test_workspace_sizes(sla):
    c = cache_of(sla)
    assert 0 < sla.sla_paged_workspace_bytes(c, 16, 4, 4) <= sla.sla_paged_workspace_bytes(c, 16, 4, 4096) < 1 << 30
    assert sla.sla_paged_workspace_bytes(cache_of(sla, dtype=torch.float32, d=64), 16, 4, 100) > 0
    assert sla.sla_paged_workspace_bytes(c, 16, 4, 4, params=sla.make_params(8, 0)) == 0     # no span decode step
    for name, bad in (("stride_t", 128), ("stride_h", 64 * 72 - 16), ("stride_page", 64 * 72 * 4 + 8), ("head_dim", 96), ("dtype", 4), ("reserved", 1)):
        c = cache_of(sla)
        setattr(c, name, bad)
        assert sla.sla_paged_workspace_bytes(c, 16, 4, 4) == 0, name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_workspace_for_span_steps_that_there_are_none_of(sla, dtype):
    """Whatever the batch, no sequences among them."""
    c, params = cache_of(sla, dtype=dtype), sla.make_params(8, 0)
    for n_seqs, n_new in ((0, 0), (0, 5), (4, 4), (4, 4096)):
        assert sla.sla_paged_workspace_bytes(c, 16, n_seqs, n_new) > 0
        assert sla.sla_paged_workspace_bytes(c, 16, n_seqs, n_new, params=params) == 0


def test_make_cache_checks_its_tensors(sla):
    k = torch.zeros(4, 2, sla.q4_plane_bytes(16, 64), dtype=torch.uint8)
    t, n, r = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    kw = dict(page_tokens=16, head_dim=64)
    c = sla.make_cache_q4(k, k.clone(), t, n, r, **kw)
    assert c.dtype == sla.SLA_Q4 and sla.make_cache_q4(k, k, t, n, r, dtype=torch.float32, **kw).dtype == sla.SLA_Q4_F32
    for args, more in (((k, k.float(), t, n, r), kw), ((k, k[:, :1], t, n, r), kw), ((k, k, t, n, r), dict(page_tokens=32, head_dim=64)),
                       ((k, k, t, n[:2], r), kw), ((k, k, t, n, r.float()), kw), ((k, k, t, n, r), dict(kw, dtype=torch.float16)),
                       ((k.int(), k.int(), t, n, r), kw), ((k[..., ::2], k[..., ::2], t, n, r), dict(page_tokens=8, head_dim=64))):
        with pytest.raises((ValueError, TypeError)):
            sla.make_cache_q4(*args, **more)


def test_host_tensors_and_wrong_types_are_refused(sla):
    c = cache_of(sla)
    i = torch.zeros(4, dtype=torch.int32)
    new, q = torch.zeros(4, 4, 128, dtype=torch.bfloat16), torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    for call in (lambda: sla.sla_cache_append(None, c, None, i, new, new), lambda: sla.sla_cache_append(None, c, None, i, new.float(), new.float()),
                 lambda: sla.sla_cache_read(None, c, None, i), lambda: sla.sla_cache_read(None, c, i, i), lambda: sla.sla_cache_read(None, c, i, i, k_out=new),
                 lambda: sla.sla_cache_read(None, c, None, None, k_out=new.float(), v_out=new.float()),
                 lambda: sla.sla_cache_read(None, c, None, None, k_out=new, v_out=new, n_new=3),
                 lambda: sla.sla_cache_read(None, c, None, None, k_out=new[:, :2], v_out=new[:, :2]),
                 lambda: sla.sla_paged_attention(None, q, c), lambda: sla.sla_paged_attention(None, q.float(), c),
                 lambda: sla.sla_paged_decode_step(None, q, q, c, sla.make_params(4, 0))):
        with pytest.raises(ValueError):
            call()


def test_a_missing_handle_is_refused(sla):
    lib, c = sla.load_library(), cache_of(sla)
    b = sla.sla_batch_t(1, 1, 1, 0, None, None)
    assert lib.sla_cache_read(None, C.addressof(c), C.addressof(b), None, 16, 16, 128, 128, None) == -1
