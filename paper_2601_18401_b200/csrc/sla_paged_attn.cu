// Attention of new tokens over a paged cache: the plan of a call, the kernel for fp32 (and for bf16 pools whose strides no tensor
// map can follow), and the join of partial results.
//
//   paged_plan     one CTA: units, their weights, the cut into equal ranges (sla_paged.cuh)
//   paged_rows     a range per CTA: tiles of KT keys against R rows (tokens x heads of a group) in fp32; running maximum and sum
//   paged_merge    per row of a cut unit: the partial results weighted by their log-sum-exp
//
// paged_rows: a tile's 2 R KT D multiply-adds run on the FMA pipe out of shared memory, each of 16 x 16 threads holding a
// (R/16) x (KT/16) piece of S and a (R/16) x (D/16) piece of O; bound by the FMA pipe and the shared-memory reads that feed it at
// R = 64, by the reads of K and V at R = 16 (one token of few heads).
#include <math_constants.h>

#include "sla_paged_attn.h"

namespace sla {

namespace {

constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) paged_plan(PagedCall a, Shape f, int n_ctas, int max_groups, int min_weight, Plan plan) {
    __shared__ long long s_sum[kPlanThreads / 32];
    chain_wait();
    chain_release();
    build_plan<kPlanThreads>(a, f, n_ctas, max_groups, min_weight, plan, s_sum);
}

// ------------------------------------------------------------------------------------------------
constexpr int kRowThreads = 256;
template <int D> constexpr int row_keys = D == 64 ? 64 : 32;
template <int D, int R> constexpr size_t row_smem() {
    constexpr int KT = row_keys<D>;
    return (size_t)(R * (D + 4) + KT * (D + 4) + KT * D + R * (KT + 4)) * sizeof(float);
}

template <typename T, int D, int R>
__global__ void __launch_bounds__(kRowThreads, 2)
paged_rows(const T *__restrict__ q, PagedCall a, int TQ, Plan plan, Parts parts, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int KT = row_keys<D>, kShift = KT == 64 ? 6 : 5;
    constexpr int RT = R / 16, CT = KT / 16, DT = D / 16;   // rows, keys, dimensions of a thread
    constexpr int QS = D + 4, PS = KT + 4;
    extern __shared__ float4 row_sm[];
    float *sq = reinterpret_cast<float *>(row_sm), *sk = sq + R * QS, *sv = sk + KT * QS, *sp = sv + KT * D;
    __shared__ int s_odd;   // a value of the tile is not finite
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int G = a.G;
    const float scale2 = a.scale * kLog2e;
    chain_wait();
    chain_release();
    for (int range = blockIdx.x;; range += gridDim.x) {
        Cursor cur;
        Segment s;
        int last_range;
        Cut cut = {0, 0, 0, -1};
        if (!cur.start(a, plan, range)) break;
        while (cur.next(a, plan, Shape{TQ, kShift, 0}, s, last_range)) {
            if (last_range >= 0) cut = {s.row0 + s.t0, s.t1 - s.t0, s.head, last_range};
            const int rows = (s.t1 - s.t0) * G;
            __syncthreads();   // the tiles of the segment before have been read
            constexpr int E = Vec16<T>::kElems;
            for (int c = tid; c < R * (D / E); c += kRowThreads) {
                const int i = c / (D / E), d = (c % (D / E)) * E, t = i / G, g = i - t * G;
                float f[E];
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = 0.f;
                if (i < rows) Vec16<T>::load(q + (long long)(s.row0 + s.t0 + t) * a.q_st + (long long)(s.head * G + g) * a.q_sh + d, f);
#pragma unroll
                for (int e = 0; e < E; ++e) sq[i * QS + d + e] = f[e] * scale2;
            }
            int last[RT], first[RT];   // keys [first, last] of this thread's rows
            float m[RT], l[RT], acc[RT][DT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int i = ty * RT + r;
                last[r] = i < rows ? s.n - s.q + s.t0 + i / G : -1;
                first[r] = a.window > 0 ? last[r] - a.window + 1 : 0;
                m[r] = -CUDART_INF_F;
                l[r] = 0.f;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[r][d] = 0.f;
            }
            const int keys_end = min(s.n, s.n - s.q + s.t1);
            const int *table = a.c.table + (long long)max(s.slot, 0) * a.c.width;
            const long long head_at = s.head * a.c.s_h;
            for (int tile = s.lo; tile < s.hi; ++tile) {
                const int j0 = tile * KT;
                if (tid == 0) s_odd = 0;
                __syncthreads();
                for (int c = tid; c < KT * (D / E); c += kRowThreads) {
                    const int jj = c / (D / E), d = (c % (D / E)) * E, j = j0 + jj;
                    float fk[E], fv[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) fk[e] = fv[e] = 0.f;
                    if (j < keys_end) {
                        const long long at = valid_page(a.c, table[j >> a.c.shift]) * a.c.s_page + head_at + (j & (a.c.P - 1)) * a.c.s_t + d;
                        Vec16<T>::load(reinterpret_cast<const T *>(a.c.k) + at, fk);
                        Vec16<T>::load(reinterpret_cast<const T *>(a.c.v) + at, fv);
                    }
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        sk[jj * QS + d + e] = fk[e];
                        const bool fin = fabsf(fv[e]) <= 3.4028235e38f;
                        odd |= !fin;
                        sv[jj * D + d + e] = fin ? fv[e] : 0.f;   // reaches only the rows that see its key, below
                    }
                    if (odd) s_odd = 1;
                }
                __syncthreads();
                float x[RT][CT];
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int k = 0; k < CT; ++k) x[r][k] = 0.f;
#pragma unroll 4
                for (int d = 0; d < D; d += 4) {
                    float4 qv[RT], kv[CT];
#pragma unroll
                    for (int r = 0; r < RT; ++r) qv[r] = *reinterpret_cast<const float4 *>(sq + (ty * RT + r) * QS + d);
#pragma unroll
                    for (int k = 0; k < CT; ++k) kv[k] = *reinterpret_cast<const float4 *>(sk + (tx + 16 * k) * QS + d);
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int k = 0; k < CT; ++k) {
                            x[r][k] = fmaf(qv[r].x, kv[k].x, x[r][k]);
                            x[r][k] = fmaf(qv[r].y, kv[k].y, x[r][k]);
                            x[r][k] = fmaf(qv[r].z, kv[k].z, x[r][k]);
                            x[r][k] = fmaf(qv[r].w, kv[k].w, x[r][k]);
                        }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    float mx = -CUDART_INF_F;
#pragma unroll
                    for (int k = 0; k < CT; ++k) {
                        const int j = j0 + tx + 16 * k;
                        if (j > last[r] || j < first[r]) x[r][k] = -CUDART_INF_F;
                        mx = fmaxf(mx, x[r][k]);
                    }
#pragma unroll
                    for (int off = 8; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                    const float mn = fmaxf(m[r], mx), base = mn == -CUDART_INF_F ? 0.f : mn;
                    const float keep = exp2f(m[r] - base);   // 0 for the first tile: m is -inf
                    m[r] = mn;
                    l[r] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) acc[r][d] *= keep;
#pragma unroll
                    for (int k = 0; k < CT; ++k) {
                        const float p = exp2f(x[r][k] - base);
                        l[r] += p;
                        sp[(ty * RT + r) * PS + tx + 16 * k] = p;
                    }
                }
                __syncwarp();   // a row's 16 threads are of one warp
#pragma unroll 4
                for (int jj = 0; jj < KT; jj += 4) {
                    float4 pv[RT];
#pragma unroll
                    for (int r = 0; r < RT; ++r) pv[r] = *reinterpret_cast<const float4 *>(sp + (ty * RT + r) * PS + jj);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float vv[DT];
#pragma unroll
                        for (int d = 0; d < DT; d += 4) *reinterpret_cast<float4 *>(vv + d) = *reinterpret_cast<const float4 *>(sv + (jj + e) * D + (d / 4) * 64 + tx * 4);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const float p = e == 0 ? pv[r].x : e == 1 ? pv[r].y : e == 2 ? pv[r].z : pv[r].w;
#pragma unroll
                            for (int d = 0; d < DT; ++d) acc[r][d] = fmaf(p, vv[d], acc[r][d]);
                        }
                    }
                }
                if (s_odd) {   // values that are not finite, for the rows that see their keys
                    for (int jj = 0; jj < KT && j0 + jj < keys_end; ++jj) {
                        const int j = j0 + jj;
                        const long long at = valid_page(a.c, table[j >> a.c.shift]) * a.c.s_page + head_at + (j & (a.c.P - 1)) * a.c.s_t;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const float v = (float)(reinterpret_cast<const T *>(a.c.v) + at)[(d / 4) * 64 + tx * 4 + d % 4];
                            if (fabsf(v) <= 3.4028235e38f) continue;
#pragma unroll
                            for (int r = 0; r < RT; ++r)
                                if (j <= last[r] && j >= first[r]) acc[r][d] = fmaf(sp[(ty * RT + r) * PS + jj], v, acc[r][d]);
                        }
                    }
                }
                __syncthreads();   // the tile has been read
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float total = l[r];
#pragma unroll
                for (int off = 8; off >= 1; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
                const int i = ty * RT + r;
                if (i >= rows) continue;
                const bool none = total == 0.f && m[r] == -CUDART_INF_F;
                const float inv = none ? 0.f : 1.f / total, lse2 = none ? -CUDART_INF_F : m[r] + log2f(total);
                if (s.part < 0) {
                    const int t = i / G, g = i - t * G;
                    const long long row = s.row0 + s.t0 + t;
                    T *o = out + row * a.q_st + (long long)(s.head * G + g) * a.q_sh;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[(d / 4) * 64 + tx * 4 + d % 4] = from_float<T>(none ? 0.f : acc[r][d] * inv);
                    if (tx == 0) lse[row * a.Hq + s.head * G + g] = lse2 * kLn2;
                } else {
                    float *o = parts.o + ((long long)s.part * R + i) * D;
#pragma unroll
                    for (int d = 0; d < DT; d += 4)
                        if (!none) *reinterpret_cast<float4 *>(o + (d / 4) * 64 + tx * 4) = make_float4(acc[r][d] * inv, acc[r][d + 1] * inv, acc[r][d + 2] * inv, acc[r][d + 3] * inv);
                    if (tx == 0) parts.lse2[(long long)s.part * R + i] = lse2;
                }
            }
        }
        if (tid == 0) parts.cut[range] = cut;
    }
}

// ------------------------------------------------------------------------------------------------
// blockIdx.x: the range a cut unit starts in.  A warp takes kMergeRows rows at a time, blockIdx.y and the warp saying which, and requests
// two parts of each together: bound by the latency of two dependent loads where units have few parts.  Row i of a unit is token
// i / G of sub-tile i / RS (TS tokens each).
constexpr int kMergeRows = 4;
template <typename T, int D>
__global__ void __launch_bounds__(256, 2) paged_merge(PagedCall a, int R, int RS, int TS, Plan plan, Parts parts, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int N = D / 32, kParts = 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    chain_wait();
    const int n_ranges = *plan.n_ranges;
    Cut cut = parts.cut[blockIdx.x];   // (beyond n_ranges: not looked at)
    for (int r = blockIdx.x; r < n_ranges;) {
        const int n_parts = cut.last - r + 1;
        const int rows = cut.last < 0 ? 0 : R;
        for (int i0 = (blockIdx.y * 8 + warp) * kMergeRows; i0 < rows; i0 += gridDim.y * 8 * kMergeRows) {
            int t[kMergeRows], h[kMergeRows];
            bool on[kMergeRows], any = false;
            float mx[kMergeRows], sum[kMergeRows], acc[kMergeRows][N];
#pragma unroll
            for (int u = 0; u < kMergeRows; ++u) {
                const int i = i0 + u, in = i % RS;
                t[u] = i / RS * TS + in / a.G;
                h[u] = cut.head * a.G + in % a.G;
                on[u] = in < TS * a.G && t[u] < cut.tokens;
                any |= on[u];
                mx[u] = -CUDART_INF_F;
                sum[u] = 0.f;
#pragma unroll
                for (int d = 0; d < N; ++d) acc[u][d] = 0.f;
            }
            if (!any) continue;
            for (int e0 = 0; e0 < n_parts; e0 += kParts) {
                float z[kMergeRows][kParts], v[kMergeRows][kParts][N];
#pragma unroll
                for (int u = 0; u < kMergeRows; ++u)
#pragma unroll
                    for (int e = 0; e < kParts; ++e) {
                        // (a part that is not there: the first one's place, without a weight; of a part without keys the sums
                        // were not written, and are not used)
                        const int part = e0 + e == 0 || e0 + e >= n_parts ? 2 * r + 1 : 2 * (r + e0 + e);
                        const long long at = (long long)part * R + i0 + u;
                        z[u][e] = __ldcg(parts.lse2 + at);
                        const float *src = parts.o + at * D + lane * N;
                        if constexpr (N == 4) *reinterpret_cast<float4 *>(v[u][e]) = __ldcg(reinterpret_cast<const float4 *>(src));
                        else *reinterpret_cast<float2 *>(v[u][e]) = __ldcg(reinterpret_cast<const float2 *>(src));
                        if (e0 + e >= n_parts) z[u][e] = -CUDART_INF_F;
                    }
#pragma unroll
                for (int u = 0; u < kMergeRows; ++u) {
                    float top = mx[u];   // a NaN reaches the result through its weight
#pragma unroll
                    for (int e = 0; e < kParts; ++e) top = fmaxf(top, z[u][e]);
                    const float keep = mx[u] == top ? 1.f : exp2f(mx[u] - top);
                    mx[u] = top;
                    sum[u] *= keep;
#pragma unroll
                    for (int d = 0; d < N; ++d) acc[u][d] *= keep;
#pragma unroll
                    for (int e = 0; e < kParts; ++e) {
                        if (z[u][e] == -CUDART_INF_F) continue;
                        const float w = exp2f(z[u][e] - top);
                        sum[u] += w;
#pragma unroll
                        for (int d = 0; d < N; ++d) acc[u][d] = fmaf(w, v[u][e][d], acc[u][d]);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kMergeRows; ++u) {
                if (!on[u]) continue;
                const bool none = mx[u] == -CUDART_INF_F && sum[u] == 0.f;
                const float inv = none ? 0.f : 1.f / sum[u];
                const long long row = cut.row0 + t[u];
                T *o = out + row * a.q_st + (long long)h[u] * a.q_sh + lane * N;
                alignas(16) T w[N];
#pragma unroll
                for (int d = 0; d < N; ++d) w[d] = from_float<T>(acc[u][d] * inv);
                if constexpr (N * sizeof(T) == 16) *reinterpret_cast<uint4 *>(o) = *reinterpret_cast<const uint4 *>(w);
                else if constexpr (N * sizeof(T) == 8) *reinterpret_cast<uint2 *>(o) = *reinterpret_cast<const uint2 *>(w);
                else *reinterpret_cast<uint32_t *>(o) = *reinterpret_cast<const uint32_t *>(w);
                if (lane == 0) lse[row * a.Hq + h[u]] = none ? -CUDART_INF_F : (mx[u] + log2f(sum[u])) * kLn2;
            }
        }
        r += gridDim.x;
        if (r < n_ranges) cut = parts.cut[r];
    }
}

template <typename T, int D, int R>
cudaError_t run_rows(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    static bool allowed[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev]) {
        e = cudaFuncSetAttribute(paged_rows<T, D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)row_smem<D, R>());
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev] = true;
    }
    return launch_chained(paged_rows<T, D, R>, dim3(p.n_ctas), dim3(kRowThreads), (row_smem<D, R>()), st, (const T *)q, a, p.TQ,
                          plan_at(p, scratch), parts_at(p, scratch), (T *)out, lse);
}

}  // namespace

cudaError_t launch_paged_plan(const PagedCall &a, const PagedPlan &p, char *scratch, cudaStream_t st) {
    return launch_chained(paged_plan, dim3(1), dim3(kPlanThreads), 0, st, a, Shape{p.TQ, p.kt_shift, p.small}, p.n_ctas, p.max_groups, p.min_weight,
                          plan_at(p, scratch));
}

template <typename T, int D>
static cudaError_t merge_of(const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    const int per = 8 * kMergeRows;
    return launch_chained(paged_merge<T, D>, dim3(p.n_ctas, (p.R + per - 1) / per), dim3(256), 0, st, a, p.R, p.RS, p.TS, plan_at(p, scratch),
                          parts_at(p, scratch), (T *)out, lse);
}

cudaError_t launch_paged_merge(const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    if (dtype == SLA_F32) return a.c.D == 64 ? merge_of<float, 64>(a, p, scratch, out, lse, st) : merge_of<float, 128>(a, p, scratch, out, lse, st);
    return a.c.D == 64 ? merge_of<__nv_bfloat16, 64>(a, p, scratch, out, lse, st) : merge_of<__nv_bfloat16, 128>(a, p, scratch, out, lse, st);
}

// Which kernel and with what tiles.
PagedPlan plan_paged(const PagedCall &a, int dtype, int sm_count) {
    PagedPlan p;
    p.kind = PagedPlan::kRows;
    p.R = a.b.max_new * (long long)a.G <= 16 ? 16 : 64;
    p.RS = p.R;
    p.TS = p.TQ = p.R / a.G;
    p.kt_shift = a.c.D == 64 ? 6 : 5;
    p.n_ctas = 2 * sm_count;
    p.max_groups = 1;
    p.min_weight = 4;
    p.small = 0;
    if (paged_decode_supported(a, dtype)) {
        p.kind = PagedPlan::kDecode;
        plan_paged_decode(a, p, sm_count);
    } else if (paged_tiles_supported(a, dtype)) {
        p.kind = PagedPlan::kTiles;
        plan_paged_tiles(a, p, sm_count);
    }
    const size_t ranges = (size_t)p.n_ctas * p.max_groups, units = (size_t)(a.b.n_new / p.TQ) + a.b.n_seqs + 1;
    p.max_units = (int)units;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = (off + bytes + 255) & ~(size_t)255;
        return at;
    };
    p.off_seq_at = take((size_t)(a.b.n_seqs + 1) * 8);
    p.off_unit_at = take((size_t)(a.b.n_seqs + 1) * 4);
    p.off_unit_end = take(units * 8);
    p.off_n_ranges = take(4);
    p.off_cut = take(ranges * sizeof(Cut));
    p.off_lse2 = take(2 * ranges * p.R * 4);
    p.off_o = take(2 * ranges * p.R * a.c.D * 4);
    p.bytes = off;
    return p;
}

cudaError_t launch_paged_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                   float *lse, cudaStream_t st, long long *launches) {
    if (p.kind == PagedPlan::kDecode) return launch_paged_decode_attention(q, a, p, scratch, counters, out, lse, st, launches);
    cudaError_t e = launch_paged_plan(a, p, scratch, st);
    if (e == cudaSuccess && p.kind == PagedPlan::kTiles) {
        e = launch_paged_tiles(q, a, p, scratch, out, lse, st);
    } else if (e == cudaSuccess) {
        if (dtype == SLA_F32) {
            if (a.c.D == 64) e = p.R == 16 ? run_rows<float, 64, 16>(q, a, p, scratch, out, lse, st) : run_rows<float, 64, 64>(q, a, p, scratch, out, lse, st);
            else e = p.R == 16 ? run_rows<float, 128, 16>(q, a, p, scratch, out, lse, st) : run_rows<float, 128, 64>(q, a, p, scratch, out, lse, st);
        } else {
            if (a.c.D == 64) e = p.R == 16 ? run_rows<__nv_bfloat16, 64, 16>(q, a, p, scratch, out, lse, st) : run_rows<__nv_bfloat16, 64, 64>(q, a, p, scratch, out, lse, st);
            else e = p.R == 16 ? run_rows<__nv_bfloat16, 128, 16>(q, a, p, scratch, out, lse, st) : run_rows<__nv_bfloat16, 128, 64>(q, a, p, scratch, out, lse, st);
        }
    }
    if (e == cudaSuccess) e = launch_paged_merge(a, dtype, p, scratch, out, lse, st);
    if (e == cudaSuccess) *launches += 3;
    return e;
}

}  // namespace sla
