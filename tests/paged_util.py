"""A paged cache in plain Python and its attention in 64 bits, for the tests of the paged calls."""
import math

import numpy as np
import torch


class Model:
    """Bookkeeping of a paged cache as include/sla.h states it: table, lengths, reference counts."""

    def __init__(self, n_pages, page, n_slots, width):
        self.P = page
        self.table = np.full((n_slots, width), -1, dtype=np.int32)
        self.n = np.zeros(n_slots, dtype=np.int32)
        self.ref = np.zeros(n_pages, dtype=np.int32)

    def pages(self, n):
        return -(-int(n) // self.P)

    def free(self):
        return [int(p) for p in np.flatnonzero(self.ref == 0)]

    def extend(self, seq, new):
        """-> first; a sequence is refused when the pages wanted up to and with it exceed the free ones."""
        free, at, first = self.free(), 0, []
        wants = []
        for s, c in zip(seq, new):
            ok = self.pages(self.n[s] + c) <= self.table.shape[1]
            need = self.pages(self.n[s] + c) - self.pages(self.n[s]) if ok else 0
            wants.append((s, c, need, ok))
        for s, c, need, ok in wants:
            begin, at = at, at + need
            if not ok or (need and at > len(free)):
                first.append(-1)
                continue
            first.append(int(self.n[s]))
            have = self.pages(self.n[s])
            for j in range(need):
                self.table[s, have + j] = free[begin + j]
                self.ref[free[begin + j]] = 1
            self.n[s] += c
        return np.array(first, dtype=np.int32)

    def release(self, seq):
        for s in seq:
            for p in self.table[s]:
                if p >= 0:
                    self.ref[p] -= 1
            self.table[s] = -1
            self.n[s] = 0

    def fork(self, src, dst):
        free, at, pairs = self.free(), 0, []
        plan = []
        for s, d in zip(src, dst):
            part = self.n[s] % self.P != 0
            plan.append((s, d, part, at if part else None))
            at += int(part)
        for s, d, part, j in plan:
            if part and j >= len(free):
                pairs.append((-1, -1))
                continue
            full = int(self.n[s]) // self.P
            self.table[d, :full] = self.table[s, :full]
            for p in self.table[s, :full]:
                self.ref[p] += 1
            if part:
                self.table[d, full] = free[j]
                self.ref[free[j]] = 1
                pairs.append((int(self.table[s, full]), free[j]))
            else:
                pairs.append((-1, -1))
            self.n[d] = self.n[s]
        return np.array(pairs, dtype=np.int32).reshape(-1, 2).T

    def compact(self):
        live = int((self.ref > 0).sum())
        movers = [p for p in range(live, len(self.ref)) if self.ref[p] > 0]
        holes = [p for p in range(live) if self.ref[p] == 0]
        to = np.arange(len(self.ref))
        pairs = np.full((2, len(self.ref)), -1, dtype=np.int32)
        for j, (a, b) in enumerate(zip(movers, holes)):
            to[a] = b
            self.ref[b], self.ref[a] = self.ref[a], 0
            pairs[:, j] = a, b
        self.table = np.where(self.table >= 0, to[np.maximum(self.table, 0)], -1).astype(np.int32)
        return pairs


def device_ints(a, dev="cuda:0"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def make_pools(n_pages, hkv, page, d, dtype, token_major=False, gap=0, seed=0, dev="cuda:0"):
    """k, v as views [n_pages, hkv, page, d]; gap: unused elements behind every page."""
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    out = []
    for _ in range(2):
        flat = torch.empty(n_pages, hkv * page * d + gap, dtype=dtype, device=dev).normal_(generator=g)
        body = flat[:, : hkv * page * d]
        out.append(body.view(n_pages, page, hkv, d).transpose(1, 2) if token_major else body.view(n_pages, hkv, page, d))
    return out


def attention_reference(q, k, v, table, n, new, G, window, scale, page):
    """64 bits, on the tensors' device, row by row over the keys each row sees -> out, lse, and two bounds: sum_j p_j |v_j| per
    output, and max_j sum_d |q_d k_jd| per row."""
    T, Hq, D = q.shape
    dev = q.device
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=dev)
    mag = torch.zeros_like(out)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=dev)
    dot = torch.zeros(T, Hq, dtype=torch.float64, device=dev)
    keys = torch.zeros(T, dtype=torch.float64, device=dev)
    r = 0
    for x, c in enumerate(new):
        pages = torch.from_numpy(table[x, : -(-int(n[x]) // page)].astype(np.int64)).to(dev)
        ks = k[pages].transpose(1, 2).reshape(-1, k.shape[1], D)[: int(n[x])].double()
        vs = v[pages].transpose(1, 2).reshape(-1, k.shape[1], D)[: int(n[x])].double()
        for t in range(int(c)):
            p = int(n[x]) - int(c) + t
            if p >= 0:
                lo = max(0, p - window + 1) if window else 0
                kk, vv = ks[lo : p + 1].repeat_interleave(G, 1), vs[lo : p + 1].repeat_interleave(G, 1)   # [J, Hq, D]
                z = torch.einsum("hd,jhd->hj", q[r].double(), kk) * scale
                lse[r] = torch.logsumexp(z, -1)
                w = torch.exp(z - lse[r][:, None])
                out[r] = torch.einsum("hj,jhd->hd", w, vv)
                mag[r] = torch.einsum("hj,jhd->hd", w, vv.abs())
                dot[r] = torch.einsum("hd,jhd->hj", q[r].double().abs(), kk.abs()).amax(-1) * abs(scale)
                keys[r] = p + 1 - lo
            r += 1
    return out, lse, mag, dot, keys


def tolerances(ref, dtype, D):
    """Worst-case rounding of each output and of lse.  A logit is off by at most D 2^-23 of the sum of its products' magnitudes
    (fp32 sums of exact or once-rounded products, in any order, truncated ones included), which moves a weight by that factor; the
    exponential and its argument are good to 2^-21 and 2^-23 of the logit; the sums over J keys to J 2^-24; bf16 rounds each
    weight to 2^-9 and the result once more."""
    out, lse, mag, dot, keys = ref
    logit = D * 2.0 ** -23 * dot + 2.0 ** -20 * (1 + dot)
    sums = keys[:, None] * 2.0 ** -24
    tol_lse = logit + sums + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0, neginf=0.0)
    rel = 2 * logit + 2 * sums
    if dtype == torch.bfloat16:
        rel = rel + 2 * 2.0 ** -9
        tol = rel[..., None] * mag + 2.0 ** -8 * out.abs()
    else:
        tol = rel[..., None] * mag + 2.0 ** -23 * out.abs()
    return tol + 1e-30, tol_lse + 1e-30


def check_attention(out, lse, ref, dtype):
    tol, tol_lse = tolerances(ref, dtype, out.shape[-1])
    empty = ref[4] == 0
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
    o, l = out.double()[~empty], lse.double()[~empty]
    r_o, r_l = ref[0][~empty], ref[1][~empty]
    fin = torch.isfinite(r_o)
    assert torch.equal(torch.isnan(r_o), torch.isnan(o))
    assert torch.equal(r_o[~fin & ~torch.isnan(r_o)], o[~fin & ~torch.isnan(r_o)])
    worst = ((o - r_o).abs() / tol[~empty])[fin]
    assert worst.numel() == 0 or worst.max() <= 1, f"out: {worst.max().item():.2f} of the tolerance"
    fin = torch.isfinite(r_l)
    assert torch.equal(torch.isfinite(l), fin)
    worst = ((l - r_l).abs() / tol_lse[~empty])[fin]
    assert worst.numel() == 0 or worst.max() <= 1, f"lse: {worst.max().item():.2f} of the tolerance"
