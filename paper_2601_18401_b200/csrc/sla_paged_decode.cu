// Attention of one new token a sequence over a paged cache, bf16.  One launch.
//
// All G query heads of a KV head share its keys, so that K and V are read once: bound by HBM.  The products run on the tensor
// cores by mma.sync with the keys as the 16 rows of A and the heads as the 8 columns of B,
//     S^T [16 keys, 8 heads] = K Q^T,      O^T [D, 8 heads] += V^T P^T,
// which wastes nothing for groups of 8 and needs no shared memory on the way: a thread fetches pieces of 16 bytes of its rows
// straight into the registers of the A operand.  The order of the D dimensions inside a product is free (Q is fetched in the same
// order), and a row of V^T is any dimension, so that pieces stay whole; pairs of neighbouring keys are put together by a byte
// permutation, P^T is the 8 x 8 transpose of P (movmatrix).  A warp goes through 16 keys at a time -- they lie in one page -- with
// the keys of the next step fetched as soon as these are used up, and the values after them.
//
// The running maximum of a head moves only when a logit passes it by 2^8 (a factor that neither the fp32 sums nor the bf16 weights
// notice), decided by one vote of the warp.  Sums are fp32; a weight is rounded to bf16 before it meets its value, as the tensor
// cores want it, the denominator adds the unrounded weights.
//
// The units (sequence, KV head) of the call lie end to end, weighted by their keys, and are cut into as many equal ranges as there
// are CTAs.  The CTA that finishes a cut unit last joins the partial results, in the order of the ranges.
#include <math_constants.h>

#include "sla_paged_attn.h"

namespace sla {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
// resident CTAs an SM: two where 16 heads of 128 dimensions fill the registers
__host__ __device__ constexpr int ctas_per_sm(int D, int NT) { return D == 128 && NT == 2 ? 2 : 3; }
constexpr int kMaxSeqs = 1024;        // of a launch
constexpr int kTileShift = 6;         // weights count 64 keys
constexpr int kMinWeight = 2;         // of a range

__device__ __forceinline__ uint4 load_stream(const void *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t y;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(D, NT))
paged_decode(const __nv_bfloat16 *__restrict__ q, PagedCall a, int x_base, int n_seqs, Parts parts, int *__restrict__ done,
             __nv_bfloat16 *__restrict__ out, float *__restrict__ lse) {
    constexpr int kChunks = D / 32;       // 16-byte pieces of a key row per thread
    constexpr int kVChunks = D / 64;      // of a value row
    constexpr int kMt = D / 16;           // m-tiles of O^T
    constexpr int R = 16;                 // rows of a partial result
    __shared__ float s_o[kWarps][8 * NT][D];
    __shared__ float s_m[kWarps][8 * NT], s_l[kWarps][8 * NT];
    __shared__ long long s_scan[kWarps];
    __shared__ int s_last;
    extern __shared__ long long s_seq_at[];   // [n_seqs + 1] weight before a sequence; then its tokens and its slot
    int *s_n = reinterpret_cast<int *>(s_seq_at + n_seqs + 1), *s_slot = s_n + n_seqs;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int G = a.G;
    const float scale2 = a.scale * kLog2e;
    chain_wait();
    chain_release();

    // ---- the units and this CTA's range
    {
        long long sum = 0;
        for (int x0 = 0; x0 < n_seqs; x0 += kThreads) {
            const int x = x0 + tid;
            long long w = 0;
            if (x < n_seqs) {
                int lo, hi, n = 0;
                new_rows(a.b, x_base + x, lo, hi);
                const int slot = slot_of(a.c, a.b, x_base + x);
                if (slot < 0) atomicOr(a.c.status, kStatusBadIndex);
                else n = tokens_of(a.c, slot);
                s_n[x] = n;
                s_slot[x] = slot;
                if (hi > lo) {
                    unit_tiles(n, 1, 0, 1, a.window, kTileShift, lo, hi);
                    w = (long long)(hi - lo + kUnitWeight) * a.c.Hkv;
                }
            }
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, w, off);
                if (lane >= off) w += y;
            }
            if (lane == 31) s_scan[warp] = w;
            __syncthreads();
            long long before = sum;
            for (int v = 0; v < kWarps; ++v) {
                if (v < warp) before += s_scan[v];
                sum += s_scan[v];
            }
            if (x < n_seqs) s_seq_at[x + 1] = before + w;
            __syncthreads();
        }
        if (tid == 0) s_seq_at[0] = 0;
        __syncthreads();
    }
    const long long total = s_seq_at[n_seqs];
    int n_ranges = gridDim.x;
    if (n_ranges > total / kMinWeight) n_ranges = (int)(total / kMinWeight);
    if (n_ranges < 1) n_ranges = 1;
    const int r = blockIdx.x;
    if (r >= n_ranges || total == 0) return;
    long long w = range_at(total, n_ranges, r);
    const long long w_end = range_at(total, n_ranges, r + 1);
    if (w >= w_end) return;
    int x = warp_last_le(s_seq_at, n_seqs, w);
    long long per_head = (s_seq_at[x + 1] - s_seq_at[x]) / a.c.Hkv;
    int head = (int)((w - s_seq_at[x]) / per_head);

    while (true) {
        const long long start = s_seq_at[x] + head * per_head, stop = start + per_head;
        const int n = s_n[x];
        int lo, hi, row_q;
        new_rows(a.b, x_base + x, row_q, hi);
        unit_tiles(n, 1, 0, 1, a.window, kTileShift, lo, hi);
        const int from = (int)(w - start), to = (int)((w_end < stop ? w_end : stop) - start);
        const int first = a.window > 0 && n > a.window ? n - a.window : 0;
        int key = max((lo + max(from - kUnitWeight, 0)) << kTileShift, first & ~15);
        const int key_end = min((lo + max(to - kUnitWeight, 0)) << kTileShift, n);
        key += 16 * warp;

        float m[NT][2], l[NT][2], acc[NT][kMt][4];
        uint32_t qf[NT][kChunks][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const bool on = 8 * t + g < G;
            const __nv_bfloat16 *src = q + (long long)row_q * a.q_st + (long long)(head * G + (on ? 8 * t + g : 0)) * a.q_sh + c * 8;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const uint4 v = on ? __ldg(reinterpret_cast<const uint4 *>(src + 32 * j)) : make_uint4(0, 0, 0, 0);
                qf[t][j][0] = v.x; qf[t][j][1] = v.y; qf[t][j][2] = v.z; qf[t][j][3] = v.w;
            }
            m[t][0] = m[t][1] = -CUDART_INF_F;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int i = 0; i < kMt; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][i][e] = 0.f;
        }

        const int *table = a.c.table + (long long)max(s_slot[x], 0) * a.c.width;
        const __nv_bfloat16 *kb = reinterpret_cast<const __nv_bfloat16 *>(a.c.k) + head * a.c.s_h;
        const __nv_bfloat16 *vb = reinterpret_cast<const __nv_bfloat16 *>(a.c.v) + head * a.c.s_h;
        uint4 kr[2][kChunks], vr[4][kVChunks];
        long long at = 0;   // of the step's first row
        auto find = [&](int k0) { return valid_page(a.c, __ldg(table + (k0 >> a.c.shift))) * a.c.s_page + (long long)(k0 & (a.c.P - 1)) * a.c.s_t; };
        auto load_k = [&](long long to_) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int j = 0; j < kChunks; ++j) kr[e][j] = load_stream(kb + to_ + (long long)(g + 8 * e) * a.c.s_t + c * 8 + 32 * j);
        };
        auto load_v = [&](long long to_, int k0) {   // values of keys outside [first, n) may be anything: they are not read
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int kk = 2 * c + (e & 1) + 8 * (e >> 1);
                const bool on = k0 + kk >= first && k0 + kk < n;
#pragma unroll
                for (int j = 0; j < kVChunks; ++j)
                    vr[e][j] = on ? load_stream(vb + to_ + (long long)kk * a.c.s_t + g * 8 + 64 * j) : make_uint4(0, 0, 0, 0);
            }
        };
        long long at_next = 0;
        if (key < key_end) {
            at = find(key);
            load_k(at);
            load_v(at, key);
            if (key + 16 * kWarps < key_end) at_next = find(key + 16 * kWarps);
        }
        for (; key < key_end; key += 16 * kWarps) {
            const int next = key + 16 * kWarps;
            float s[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
                for (int j = 0; j < kChunks; ++j) {
                    mma16816(s[t], kr[0][j].x, kr[1][j].x, kr[0][j].y, kr[1][j].y, qf[t][j][0], qf[t][j][1]);
                    mma16816(s[t], kr[0][j].z, kr[1][j].z, kr[0][j].w, kr[1][j].w, qf[t][j][2], qf[t][j][3]);
                }
            }
            if (next < key_end) load_k(at_next);
            bool over = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] *= scale2;
            if (key < first || key + 16 > n) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int kk = key + g + 8 * (e >> 1);
                        if (kk < first || kk >= n) s[t][e] = -CUDART_INF_F;
                    }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) over |= fmaxf(s[t][e], s[t][e + 2]) > m[t][e] + 8.f;
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(m[t][e], fmaxf(s[t][e], s[t][e + 2]));
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                        const float keep = m[t][e] == mx ? 1.f : exp2_fast(m[t][e] - mx);
                        m[t][e] = mx;
                        l[t][e] *= keep;
#pragma unroll
                        for (int i = 0; i < kMt; ++i) {
                            acc[t][i][e] *= keep;
                            acc[t][i][e + 2] *= keep;
                        }
                    }
            }
            uint32_t pf[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float base = m[t][e & 1] == -CUDART_INF_F ? 0.f : m[t][e & 1];
                    s[t][e] = exp2_fast(s[t][e] - base);
                    l[t][e & 1] += s[t][e];
                }
                pf[t][0] = transpose8x8(pack_bf16(s[t][0], s[t][1]));
                pf[t][1] = transpose8x8(pack_bf16(s[t][2], s[t][3]));
            }
            // row g of m-tile i: dimension 8 g + i; row g + 8: 64 + 8 g + i (D = 64: 8 g + 4 + i)
#pragma unroll
            for (int i = 0; i < kMt; ++i) {
                const int i1 = D == 128 ? i : i + 4, j1 = D == 128 ? kVChunks - 1 : 0;
                const uint32_t sel = i & 1 ? 0x7632u : 0x5410u, sel1 = i1 & 1 ? 0x7632u : 0x5410u;
                const uint32_t a0 = __byte_perm(word(vr[0][0], i / 2), word(vr[1][0], i / 2), sel);
                const uint32_t a2 = __byte_perm(word(vr[2][0], i / 2), word(vr[3][0], i / 2), sel);
                const uint32_t a1 = __byte_perm(word(vr[0][j1], i1 / 2), word(vr[1][j1], i1 / 2), sel1);
                const uint32_t a3 = __byte_perm(word(vr[2][j1], i1 / 2), word(vr[3][j1], i1 / 2), sel1);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16816(acc[t][i], a0, a1, a2, a3, pf[t][0], pf[t][1]);
            }
            if (next < key_end) {
                load_v(at_next, next);
                if (next + 16 * kWarps < key_end) at_next = find(next + 16 * kWarps);
            }
        }

        // ---- join the warps
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v = l[t][e];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
                const int qi = 8 * t + 2 * c + e;
                if (g == 0) { s_m[warp][qi] = m[t][e]; s_l[warp][qi] = v; }
#pragma unroll
                for (int i = 0; i < kMt; ++i) {
                    s_o[warp][qi][8 * g + i] = acc[t][i][e];
                    s_o[warp][qi][D == 128 ? 64 + 8 * g + i : 8 * g + 4 + i] = acc[t][i][e + 2];
                }
            }
        __syncthreads();
        const bool begins = from == 0, ends = w_end >= stop;
        const int part = begins && ends ? -1 : begins ? 2 * r + 1 : 2 * r;
        for (int it = tid; it < G * (D / 4); it += kThreads) {
            const int qi = it / (D / 4), d = (it % (D / 4)) * 4;
            float mx = s_m[0][qi];
#pragma unroll
            for (int v = 1; v < kWarps; ++v) mx = fmaxf(mx, s_m[v][qi]);
            float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < kWarps; ++v) {
                const float wt = s_m[v][qi] == -CUDART_INF_F && s_l[v][qi] == 0.f ? 0.f : exp2_fast(s_m[v][qi] - (mx == -CUDART_INF_F ? 0.f : mx));
                // a warp without a key has no weight; one whose only logits are NaN carries them in its sum
                const float wv = s_m[v][qi] == -CUDART_INF_F && !(s_l[v][qi] == 0.f) ? 1.f : wt;
                const float4 ov = *reinterpret_cast<const float4 *>(&s_o[v][qi][d]);
                sum = fmaf(wv, s_l[v][qi], sum);
                o[0] = fmaf(wv, ov.x, o[0]); o[1] = fmaf(wv, ov.y, o[1]); o[2] = fmaf(wv, ov.z, o[2]); o[3] = fmaf(wv, ov.w, o[3]);
            }
            const bool none = sum == 0.f && mx == -CUDART_INF_F;
            const float inv = none ? 0.f : 1.f / sum, z = none ? -CUDART_INF_F : mx + log2f(sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] *= inv;
            if (part < 0) {
                const int h = head * G + qi;
                *reinterpret_cast<uint2 *>(out + (long long)row_q * a.q_st + (long long)h * a.q_sh + d) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
                if (d == 0) lse[(long long)row_q * a.Hq + h] = z * kLn2;
            } else {
                if (!none) __stcg(reinterpret_cast<float4 *>(parts.o + ((long long)part * R + qi) * D + d), make_float4(o[0], o[1], o[2], o[3]));
                if (d == 0) __stcg(parts.lse2 + (long long)part * R + qi, z);
            }
        }
        if (part >= 0) {
            // ranges [r0, r1] hold this unit
            auto range_of = [&](long long p) {   // the range of position p
                int z = (int)((double)p * n_ranges / (double)total);
                z = min(max(z, 0), n_ranges - 1);
                while (z > 0 && range_at(total, n_ranges, z) > p) --z;
                while (range_at(total, n_ranges, z + 1) <= p) ++z;
                return z;
            };
            const int r0 = begins ? r : range_of(start), r1 = ends ? r : range_of(stop - 1), n_parts = r1 - r0 + 1;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                s_last = atomicAdd(done + r0, 1) == n_parts - 1;
                if (s_last) done[r0] = 0;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                auto part_at = [&](int e) { return (long long)(e == 0 ? 2 * r0 + 1 : 2 * (r0 + e)) * R; };
                for (int it = tid; it < G * (D / 4); it += kThreads) {
                    const int qi = it / (D / 4), d = (it % (D / 4)) * 4;
                    float mx = -CUDART_INF_F, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int e0 = 0; e0 < n_parts; e0 += 8) {
                        float z[8], top = mx;
                        float4 v[8];
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            z[u] = -CUDART_INF_F;
                            if (e0 + u < n_parts) {
                                z[u] = __ldcg(parts.lse2 + part_at(e0 + u) + qi);
                                v[u] = __ldcg(reinterpret_cast<const float4 *>(parts.o + (part_at(e0 + u) + qi) * D + d));
                            }
                            top = fmaxf(top, z[u]);
                        }
                        const float keep = mx == top ? 1.f : exp2_fast(mx - top);
                        mx = top;
                        sum *= keep;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] *= keep;
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            if (z[u] == -CUDART_INF_F) continue;   // nothing was written
                            const float wt = exp2_fast(z[u] - mx);
                            sum += wt;
                            o[0] = fmaf(wt, v[u].x, o[0]); o[1] = fmaf(wt, v[u].y, o[1]); o[2] = fmaf(wt, v[u].z, o[2]); o[3] = fmaf(wt, v[u].w, o[3]);
                        }
                    }
                    const bool none = mx == -CUDART_INF_F && sum == 0.f;
                    const float inv = none ? 0.f : 1.f / sum;
                    const int h = head * G + qi;
                    *reinterpret_cast<uint2 *>(out + (long long)row_q * a.q_st + (long long)h * a.q_sh + d) =
                        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
                    if (d == 0) lse[(long long)row_q * a.Hq + h] = none ? -CUDART_INF_F : (mx + log2f(sum)) * kLn2;
                }
            }
        }
        w = stop;
        if (w >= w_end) break;
        __syncthreads();   // shared memory has been read
        if (++head == a.c.Hkv) {
            head = 0;
            do ++x; while (s_seq_at[x + 1] == s_seq_at[x]);
            per_head = (s_seq_at[x + 1] - s_seq_at[x]) / a.c.Hkv;
        }
    }
}

}  // namespace

bool paged_decode_supported(const PagedCall &a, int dtype) { return dtype == SLA_BF16 && a.b.max_new == 1; }

void plan_paged_decode(const PagedCall &a, PagedPlan &p, int sm_count) {
    p.R = p.RS = 16;
    p.TS = p.TQ = 1;
    p.n_ctas = ctas_per_sm(a.c.D, a.G <= 8 ? 1 : 2) * sm_count;
}

template <int D, int NT>
static cudaError_t decode_of(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, int *counters, void *out, float *lse,
                             cudaStream_t st, long long *launches) {
    cudaError_t e = cudaSuccess;
    for (int x0 = 0; x0 < a.b.n_seqs && e == cudaSuccess; x0 += kMaxSeqs) {
        const int n = a.b.n_seqs - x0 < kMaxSeqs ? a.b.n_seqs - x0 : kMaxSeqs;
        e = launch_chained(paged_decode<D, NT>, dim3(p.n_ctas), dim3(kThreads), (size_t)(n + 1) * 8 + (size_t)n * 8, st,
                           (const __nv_bfloat16 *)q, a, x0, n, parts_at(p, scratch), counters, (__nv_bfloat16 *)out, lse);
        ++*launches;
    }
    return e;
}

cudaError_t launch_paged_decode_attention(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, int *counters, void *out,
                                          float *lse, cudaStream_t st, long long *launches) {
    if (a.c.D == 64) return a.G <= 8 ? decode_of<64, 1>(q, a, p, scratch, counters, out, lse, st, launches) : decode_of<64, 2>(q, a, p, scratch, counters, out, lse, st, launches);
    return a.G <= 8 ? decode_of<128, 1>(q, a, p, scratch, counters, out, lse, st, launches) : decode_of<128, 2>(q, a, p, scratch, counters, out, lse, st, launches);
}

}  // namespace sla
