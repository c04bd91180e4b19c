// Attention of new tokens over a paged cache: the plan of a call, the kernel for fp32 (and for bf16 pools whose strides no tensor
// map can follow), and the join of partial results.
//
//   paged_plan     one CTA: units, their weights, the cut into equal ranges, where each begins (sla_paged.cuh)
//   paged_rows     a range per CTA: tiles of 64 keys against R rows (tokens x heads of a group) in fp32; running maximum and sum
//   paged_merge    per row of a cut unit: the partial results weighted by their log-sum-exp
//
// paged_rows: a tile's 2 R 64 D multiply-adds run on the FMA pipe out of shared memory; bound by that pipe and by the reads that feed
// it (ncu, 8/2 heads, D 64, 4096 tokens: FMA pipe 62 %, shared memory 61 %).  Measured there: 443 us, 39 TFLOP/s; the same with D 128:
// 883 us.  Single rows of fp32 FMA reach 75 TFLOP/s; tf32 tensor products were not taken: they round the inputs to 11 bits.
#include <math_constants.h>

#include <type_traits>

#include "sla_paged_attn.h"
#include "sla_q4.cuh"

namespace sla {

namespace {

constexpr int kPlanThreads = 1024;

// The plan is built in shared memory where it fits (4 to 6 us), else where it goes.
constexpr int kPlanSeqs = 512, kPlanUnits = 2048;
__global__ void __launch_bounds__(kPlanThreads) paged_plan(PagedCall a, Shape f, int n_ctas, int max_groups, int min_weight, Plan plan, Cut *__restrict__ cut) {
    __shared__ long long s_sum[kPlanThreads / 32], s_seq_at[kPlanSeqs + 1], s_unit_end[kPlanUnits];
    __shared__ int s_unit_at[kPlanSeqs + 1];
    __shared__ int4 s_seqs[kPlanSeqs];
    __shared__ Ranges s_ranges;
    const bool fits = a.b.n_seqs <= kPlanSeqs && plan.max_units <= kPlanUnits;
    Plan own = plan;
    own.ranges = &s_ranges;
    if (fits) {
        own.seq_at = s_seq_at;
        own.unit_at = s_unit_at;
        own.unit_end = s_unit_end;
        own.seqs = s_seqs;
    }
    chain_wait();
    chain_release();
    build_plan<kPlanThreads>(a, f, n_ctas, max_groups, min_weight, own, s_sum);
    const Ranges ranges = s_ranges;
    if (fits) {   // (by the threads that have no range, if there are such)
        const int last = kPlanThreads - 1 - threadIdx.x;
        for (int x = last; x <= a.b.n_seqs; x += kPlanThreads) {
            plan.seq_at[x] = s_seq_at[x];
            plan.unit_at[x] = s_unit_at[x];
            if (x < a.b.n_seqs) plan.seqs[x] = s_seqs[x];
        }
        for (int u = last; u < s_unit_at[a.b.n_seqs]; u += kPlanThreads) plan.unit_end[u] = s_unit_end[u];
    }
    if (threadIdx.x == kPlanThreads - 1) *plan.ranges = ranges;
    for (int r = threadIdx.x; r < ranges.count; r += kPlanThreads) {
        Cursor c;
        Start b;
        c.seek(a, own, ranges, r);
        c.next(a, own, f, b.s, b.last_range);
        b.w = c.w; b.x = c.x; b.unit = c.unit; b.units = c.units;
        plan.starts[r] = b;
        cut[r] = {0, 0, 0, -1};   // a CTA that leaves early (a wait that ran out) leaves its ranges so, and paged_merge writes nothing for them
    }
}

// ------------------------------------------------------------------------------------------------
// Tiles of KT = 64 keys against R = 16 RT rows, 16 x 16 threads: thread (ty, tx) has rows RT ty .. of S and O, keys tx + 16 k of S and
// dimensions 64 (d / 4) + 4 tx + d % 4 of O.  Two neighbouring rows share an fma.f32x2: Q and P lie in shared memory by dimension and by
// key, rows next to each other, so that pairs of rows come out of a 16-byte load; the key's (the value's) number is doubled in registers.
constexpr int kRowThreads = 256, kRowKeys = 64;
template <int D, int R> constexpr size_t kRowSmem = (size_t)(D * R + kRowKeys * (D + 4) + kRowKeys * D + kRowKeys * (R + 4)) * sizeof(float);
// two CTAs an SM where their shared memory fits
template <int D, int R> constexpr int kRowCtas = kRowSmem<D, R> <= 112 * 1024 ? 2 : 1;

__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void of_pair(unsigned long long r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

template <typename T, int D, int R, bool kQ4>
__global__ void __launch_bounds__(kRowThreads, (kRowCtas<D, R>))
paged_rows(const T *__restrict__ q, PagedCall a, int TQ, Plan plan, Parts parts, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int KT = kRowKeys, kShift = 6;
    constexpr int RT = R / 16, RP = RT / 2, CT = KT / 16, DT = D / 16;   // rows, pairs of rows, keys, dimensions of a thread
    constexpr int KS = D + 4, PS = R + 4;   // (padded against bank conflicts)
    constexpr int E = kQ4 ? 8 : Vec16<T>::kElems, kLoads = KT * D / E / kRowThreads;   // pieces of a tile per thread: 16 bytes, or 8 codes and their scale
    constexpr int QE = Vec16<T>::kElems;
    static_assert(RT % 4 == 0, "rows of a thread come in 16-byte loads");
    extern __shared__ float4 row_sm[];
    float *sq = reinterpret_cast<float *>(row_sm), *sk = sq + D * R, *sv = sk + KT * KS, *sp = sv + KT * D;   // [D][R], [KT][KS], [KT][D], [KT][PS]
    __shared__ int s_odd;      // a value of the tile is not finite
    __shared__ int s_pos[R];   // positions of the rows, -1 for rows that do not exist
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
        if (!cur.open(plan, range, s, last_range)) break;
        do {
            if (last_range >= 0) cut = {s.row0 + s.t0, s.t1 - s.t0, s.head, last_range};
            const int rows = (s.t1 - s.t0) * G;
            const int keys_end = min(s.n, s.n - s.q + s.t1);
            const int *table = a.c.table + (long long)max(s.slot, 0) * a.c.width;
            const long long head_at = s.head * a.c.s_h;
            // pieces of a tile: piece c is E values of key c / (D / E)
            using Raw = typename std::conditional<kQ4, uint2, uint4>::type;
            Raw raw[kLoads];
            auto fetch = [&](const char *pool, int tile) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int c = tid + i * kRowThreads, j = tile * KT + c / (D / E), d = (c % (D / E)) * E;
                    raw[i] = Raw{};
                    if (j >= keys_end) continue;
                    if constexpr (kQ4) {
                        const char *plane = pool + valid_page(a.c, __ldg(table + (j >> a.c.shift))) * a.c.s_page + head_at;
                        if (pool == a.c.k) q4::load_piece<false>(plane, a.c.P, D, j & (a.c.P - 1), d / 8, raw[i].x, raw[i].y);
                        else q4::load_piece<true>(plane, a.c.P, D, j & (a.c.P - 1), d / 8, raw[i].x, raw[i].y);
                    } else {
                        const long long at = valid_page(a.c, __ldg(table + (j >> a.c.shift))) * a.c.s_page + head_at + (j & (a.c.P - 1)) * a.c.s_t + d;
                        raw[i] = __ldg(reinterpret_cast<const uint4 *>(pool + at * sizeof(T)));
                    }
                }
            };
            auto widen = [&](const Raw &v, float (&f)[E]) {
                if constexpr (kQ4) {
                    uint32_t w[4];
                    q4::values(v.x, q4::factor(v.y), w);
                    Vec16<__nv_bfloat16>::unpack(make_uint4(w[0], w[1], w[2], w[3]), f);
                } else if constexpr (sizeof(T) == 2) {
                    Vec16<__nv_bfloat16>::unpack(v, f);
                } else {
                    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
                }
            };
            if (s.lo < s.hi) fetch(a.c.k, s.lo);
            __syncthreads();   // shared memory of the segment before has been read
            for (int c = tid; c < R * (D / QE); c += kRowThreads) {
                const int i = c % R, d = (c / R) * QE, t = i / G, g = i - t * G;   // neighbouring threads, neighbouring rows: no conflicts
                float f[QE];
#pragma unroll
                for (int e = 0; e < QE; ++e) f[e] = 0.f;
                if (i < rows) Vec16<T>::load(q + (long long)(s.row0 + s.t0 + t) * a.q_st + (long long)(s.head * G + g) * a.q_sh + d, f);
#pragma unroll
                for (int e = 0; e < QE; ++e) sq[(d + e) * R + i] = f[e] * scale2;
            }
            if (tid < R) s_pos[tid] = tid < rows ? s.n - s.q + s.t0 + tid / G : -1;
            // keys that every row of the unit sees; a row sees [position - window + 1, position]
            const int all_hi = rows == R ? s.n - s.q + s.t0 : -1, all_lo = a.window > 0 ? minus(s.n - s.q + s.t1, a.window) : 0;
            const int reach = a.window > 0 ? a.window : 0x7fffffff;
            float m[RT], l[RT];
            unsigned long long acc[RP][DT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                m[r] = -CUDART_INF_F;
                l[r] = 0.f;
            }
#pragma unroll
            for (int r = 0; r < RP; ++r)
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[r][d] = 0ull;
            for (int tile = s.lo; tile < s.hi; ++tile) {
                const int j0 = tile * KT;
                // K of this tile is on its way; its V is requested before S, the next tile's K before O
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int c = tid + i * kRowThreads;
                    float f[E];
                    widen(raw[i], f);
#pragma unroll
                    for (int e = 0; e < E; e += 4)
                        *reinterpret_cast<float4 *>(sk + (c / (D / E)) * KS + (c % (D / E)) * E + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                }
                if (tid == 0) s_odd = 0;
                __syncthreads();
                fetch(a.c.v, tile);
                unsigned long long x[RP][CT];
#pragma unroll
                for (int r = 0; r < RP; ++r)
#pragma unroll
                    for (int k = 0; k < CT; ++k) x[r][k] = 0ull;
#pragma unroll 8
                for (int d0 = 0; d0 < D; d0 += 4) {
                    float4 kv[CT];
#pragma unroll
                    for (int k = 0; k < CT; ++k) kv[k] = *reinterpret_cast<const float4 *>(sk + (tx + 16 * k) * KS + d0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        unsigned long long qv[RP];
#pragma unroll
                        for (int r = 0; r < RP; r += 2) {
                            const ulonglong2 w = *reinterpret_cast<const ulonglong2 *>(sq + (d0 + e) * R + ty * RT + 2 * r);
                            qv[r] = w.x;
                            qv[r + 1] = w.y;
                        }
#pragma unroll
                        for (int k = 0; k < CT; ++k) {
                            const float kk = e == 0 ? kv[k].x : e == 1 ? kv[k].y : e == 2 ? kv[k].z : kv[k].w;
                            const unsigned long long k2 = pair_of(kk, kk);
#pragma unroll
                            for (int r = 0; r < RP; ++r) x[r][k] = fma_pair(qv[r], k2, x[r][k]);
                        }
                    }
                }
                const bool edge = j0 + KT - 1 > all_hi || j0 < all_lo;
#pragma unroll
                for (int r = 0; r < RT; r += 2) {
                    float keep[2];
                    float y[2][CT];
#pragma unroll
                    for (int k = 0; k < CT; ++k) of_pair(x[r / 2][k], y[0][k], y[1][k]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (edge) {
                            const int back = s_pos[ty * RT + r + h] - j0 - tx;   // how far a key lies before the row's position
#pragma unroll
                            for (int k = 0; k < CT; ++k)
                                if (back - 16 * k < 0 || back - 16 * k >= reach) y[h][k] = -CUDART_INF_F;
                        }
                        float mx = y[h][0];
#pragma unroll
                        for (int k = 1; k < CT; ++k) mx = fmaxf(mx, y[h][k]);
#pragma unroll
                        for (int off = 8; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                        const float mn = fmaxf(m[r + h], mx), base = mn == -CUDART_INF_F ? 0.f : mn;
                        keep[h] = ex2(m[r + h] - base);   // 0 for the first tile: m is -inf
                        m[r + h] = mn;
                        l[r + h] *= keep[h];
#pragma unroll
                        for (int k = 0; k < CT; ++k) {
                            y[h][k] = ex2(y[h][k] - base);
                            l[r + h] += y[h][k];
                        }
                    }
#pragma unroll
                    for (int k = 0; k < CT; ++k) x[r / 2][k] = pair_of(y[0][k], y[1][k]);
                    const unsigned long long kp = pair_of(keep[0], keep[1]);
#pragma unroll
                    for (int d = 0; d < DT; ++d) acc[r / 2][d] = fma_pair(acc[r / 2][d], kp, 0ull);
                }
#pragma unroll
                for (int k = 0; k < CT; ++k)
#pragma unroll
                    for (int r = 0; r < RP; r += 2)
                        *reinterpret_cast<ulonglong2 *>(sp + (tx + 16 * k) * PS + ty * RT + 2 * r) = make_ulonglong2(x[r][k], x[r + 1][k]);
                bool odd = false;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int c = tid + i * kRowThreads;
                    float f[E];
                    widen(raw[i], f);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const bool fin = fabsf(f[e]) <= 3.4028235e38f;
                        odd |= !fin;
                        f[e] = fin ? f[e] : 0.f;   // reaches only the rows that see its key, below
                    }
#pragma unroll
                    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4 *>(sv + c * E + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                }
                if (odd) s_odd = 1;
                __syncthreads();
                if (tile + 1 < s.hi) fetch(a.c.k, tile + 1);
#pragma unroll 8
                for (int jj = 0; jj < KT; ++jj) {
                    unsigned long long pv[RP];
#pragma unroll
                    for (int r = 0; r < RP; r += 2) {
                        const ulonglong2 w = *reinterpret_cast<const ulonglong2 *>(sp + jj * PS + ty * RT + 2 * r);
                        pv[r] = w.x;
                        pv[r + 1] = w.y;
                    }
#pragma unroll
                    for (int d = 0; d < DT; d += 4) {
                        const float4 v = *reinterpret_cast<const float4 *>(sv + jj * D + (d / 4) * 64 + tx * 4);
                        const unsigned long long v0 = pair_of(v.x, v.x), v1 = pair_of(v.y, v.y), v2 = pair_of(v.z, v.z), v3 = pair_of(v.w, v.w);
#pragma unroll
                        for (int r = 0; r < RP; ++r) {
                            acc[r][d] = fma_pair(pv[r], v0, acc[r][d]);
                            acc[r][d + 1] = fma_pair(pv[r], v1, acc[r][d + 1]);
                            acc[r][d + 2] = fma_pair(pv[r], v2, acc[r][d + 2]);
                            acc[r][d + 3] = fma_pair(pv[r], v3, acc[r][d + 3]);
                        }
                    }
                }
                if (s_odd) {   // values that are not finite, for the rows that see their keys
#pragma unroll 1
                    for (int jj = 0; jj < KT && j0 + jj < keys_end; ++jj) {
                        const int j = j0 + jj;
                        const long long plane = valid_page(a.c, table[j >> a.c.shift]) * a.c.s_page + head_at, at = plane + (j & (a.c.P - 1)) * a.c.s_t;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const int dim = (d / 4) * 64 + tx * 4 + d % 4;
                            float v;   // (of a four-bit cache: whether it is finite, which its scale says)
                            if constexpr (kQ4) v = __uint_as_float(q4::scale_of(a.c.v + plane, a.c.P, D, j & (a.c.P - 1), dim) << 16);
                            else v = (float)(reinterpret_cast<const T *>(a.c.v) + at)[dim];
                            if (fabsf(v) <= 3.4028235e38f) continue;
#pragma unroll
                            for (int r = 0; r < RP; ++r) {
                                float o0, o1;
                                of_pair(acc[r][d], o0, o1);
                                const int b0 = s_pos[ty * RT + 2 * r] - j, b1 = s_pos[ty * RT + 2 * r + 1] - j;
                                if (b0 >= 0 && b0 < reach) o0 = fmaf(sp[jj * PS + ty * RT + 2 * r], v, o0);
                                if (b1 >= 0 && b1 < reach) o1 = fmaf(sp[jj * PS + ty * RT + 2 * r + 1], v, o1);
                                acc[r][d] = pair_of(o0, o1);
                            }
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
                float o[DT];
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    float o0, o1;
                    of_pair(acc[r / 2][d], o0, o1);
                    o[d] = none ? 0.f : (r & 1 ? o1 : o0) * inv;
                }
                if (s.part < 0) {
                    const int t = i / G, g = i - t * G;
                    const long long row = s.row0 + s.t0 + t;
                    T *dst = out + row * a.q_st + (long long)(s.head * G + g) * a.q_sh;
#pragma unroll
                    for (int d = 0; d < DT; ++d) dst[(d / 4) * 64 + tx * 4 + d % 4] = from_float<T>(o[d]);
                    if (tx == 0) lse[row * a.Hq + s.head * G + g] = lse2 * kLn2;
                } else {
#pragma unroll
                    for (int d = 0; d < DT; d += 4)
                        if (!none) *reinterpret_cast<float4 *>(parts.at(s.part, R, D, i, (d / 4) * 64 + tx * 4)) = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
                    if (tx == 0) parts.lse2[(long long)s.part * R + i] = lse2;
                }
            }
        } while (cur.next(a, plan, Shape{TQ, kShift, 0}, s, last_range));
        if (tid == 0) parts.cut[range] = cut;
    }
}

// ------------------------------------------------------------------------------------------------
// blockIdx.x: the range a cut unit starts in.  A thread takes kMergeCols columns of a row, neighbouring threads neighbouring rows, and requests
// kParts parts together: bound by the latency of dependent loads (8 us).  22 tokens at 23199, 32/4 heads, D 64, 37 parts a unit, whole call:
// 30.7 us, 34.7 with 16 columns and two parts at a time; four threads a row that take every fourth part, 28.0, but then calls of few parts
// a unit take longer for the number of CTAs (1 to 600 tokens of 16 sequences: 66 us instead of 59.6).  Row i of a unit is token i / G of
// sub-tile i / RS (TS tokens each).
constexpr int kMergeThreads = 256, kMergeCols = 8;
__device__ __forceinline__ void load8(const float *p, float *v) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "l"(p));
}
template <typename T, int D>
__global__ void __launch_bounds__(kMergeThreads, 4) paged_merge(PagedCall a, int R, int RS, int TS, Plan plan, Parts parts, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int kParts = 4;
    chain_wait();
    chain_release();
    const int r = blockIdx.x, n_ranges = plan.ranges->count;
    const Cut cut = parts.cut[r];   // (beyond n_ranges: not looked at)
    if (r >= n_ranges || cut.last < 0) return;
    const int n_parts = cut.last - r + 1;
    const int i = threadIdx.x & (R - 1), d0 = kMergeCols * (blockIdx.y * (kMergeThreads / R) + threadIdx.x / R);
    const int in = i % RS, t = i / RS * TS + in / a.G, h = cut.head * a.G + in % a.G;
    if (in >= TS * a.G || t >= cut.tokens) return;
    float mx = -CUDART_INF_F, sum = 0.f, acc[kMergeCols];
#pragma unroll
    for (int d = 0; d < kMergeCols; ++d) acc[d] = 0.f;
    for (int e0 = 0; e0 < n_parts; e0 += kParts) {
        float z[kParts], v[kParts][kMergeCols];
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
            z[e] = -CUDART_INF_F;
            if (e0 + e >= n_parts) continue;
            // (of a part without keys the sums were not written, and are not used)
            const int part = e0 + e == 0 ? 2 * r + 1 : 2 * (r + e0 + e);
            z[e] = parts.lse2[(long long)part * R + i];
#pragma unroll
            for (int d = 0; d < kMergeCols; d += 8) load8(parts.at(part, R, D, i, d0 + d), v[e] + d);
        }
        float top = mx;   // a NaN reaches the result through its weight
#pragma unroll
        for (int e = 0; e < kParts; ++e) top = fmaxf(top, z[e]);
        const float keep = mx == top ? 1.f : exp2f(mx - top);
        mx = top;
        sum *= keep;
#pragma unroll
        for (int d = 0; d < kMergeCols; ++d) acc[d] *= keep;
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
            if (z[e] == -CUDART_INF_F) continue;
            const float w = exp2f(z[e] - top);
            sum += w;
#pragma unroll
            for (int d = 0; d < kMergeCols; ++d) acc[d] = fmaf(w, v[e][d], acc[d]);
        }
    }
    const bool none = mx == -CUDART_INF_F && sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    const long long row = cut.row0 + t;
    T *o = out + row * a.q_st + (long long)h * a.q_sh + d0;
    constexpr int E = Vec16<T>::kElems;
#pragma unroll
    for (int d = 0; d < kMergeCols; d += E) {
        alignas(16) T w[E];
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = from_float<T>(acc[d + e] * inv);
        *reinterpret_cast<uint4 *>(o + d) = *reinterpret_cast<const uint4 *>(w);
    }
    if (d0 == 0) lse[row * a.Hq + h] = none ? -CUDART_INF_F : (mx + log2f(sum)) * kLn2;
}

template <typename T, int D, int R, bool kQ4>
cudaError_t run_rows(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    static bool allowed[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev]) {
        e = cudaFuncSetAttribute(paged_rows<T, D, R, kQ4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowSmem<D, R>);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev] = true;
    }
    return launch_chained(paged_rows<T, D, R, kQ4>, dim3(p.n_ctas), dim3(kRowThreads), (kRowSmem<D, R>), st, (const T *)q, a, p.TQ,
                          plan_at(p, scratch), parts_at(p, scratch), (T *)out, lse);
}

}  // namespace

cudaError_t launch_paged_plan(const PagedCall &a, const PagedPlan &p, char *scratch, cudaStream_t st) {
    return launch_chained(paged_plan, dim3(1), dim3(kPlanThreads), 0, st, a, Shape{p.TQ, p.kt_shift, p.small}, p.n_ctas, p.max_groups, p.min_weight,
                          plan_at(p, scratch), parts_at(p, scratch).cut);
}

template <typename T, int D>
static cudaError_t merge_of(const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    return launch_chained(paged_merge<T, D>, dim3(p.n_ctas * p.max_groups, D / kMergeCols * p.R / kMergeThreads), dim3(kMergeThreads), 0, st, a, p.R,
                          p.RS, p.TS, plan_at(p, scratch), parts_at(p, scratch), (T *)out, lse);
}

cudaError_t launch_paged_merge(const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    if (dtype == SLA_F32) return a.c.D == 64 ? merge_of<float, 64>(a, p, scratch, out, lse, st) : merge_of<float, 128>(a, p, scratch, out, lse, st);
    return a.c.D == 64 ? merge_of<__nv_bfloat16, 64>(a, p, scratch, out, lse, st) : merge_of<__nv_bfloat16, 128>(a, p, scratch, out, lse, st);
}

// Which kernel and with what tiles.
PagedPlan plan_paged(const PagedCall &a, int dtype, int sm_count, size_t gap) {
    PagedPlan p;
    p.kind = PagedPlan::kRows;
    // 64 rows where no sequence has more, else 128: fp32, 2 sequences of 4000 to 9000 tokens, 12 to 16 new, 8/2 heads, D 64, 40 us against 53
    // with 128; 1000 new at 4000, D 128, 374 us with 128 against 468.
    p.R = a.b.max_new * (long long)a.G <= 64 ? 64 : 128;
    p.RS = p.R;
    p.TS = p.TQ = p.R / a.G;
    p.kt_shift = 6;
    p.n_ctas = (a.c.D == 128 ? 1 : 2) * sm_count;
    p.max_groups = 1;
    p.min_weight = 2;
    p.small = 0;
    p.fold_bytes = 0;
    if (paged_decode_supported(a)) {
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
        if (gap) { p.canaries.add(off); off += gap; }
        const size_t at = off;
        off = (off + bytes + 255) & ~(size_t)255;
        return at;
    };
    p.off_seq_at = take((size_t)(a.b.n_seqs + 1) * 8);
    p.off_unit_at = take((size_t)(a.b.n_seqs + 1) * 4);
    p.off_unit_end = take(units * 8);
    p.off_ranges = take(sizeof(Ranges));
    p.max_ranges = (int)ranges;
    p.off_seqs = take((size_t)a.b.n_seqs * sizeof(int4));
    p.off_starts = take(ranges * sizeof(Start));
    p.off_cut = take(ranges * sizeof(Cut));
    p.off_lse2 = take(2 * ranges * p.R * 4);
    p.off_o = take(2 * ranges * p.R * a.c.D * 4);
    p.off_fold = take(p.fold_bytes);
    if (gap) { p.canaries.add(off); off += gap; }
    p.bytes = off;
    return p;
}

template <typename T, int D, bool kQ4>
static cudaError_t rows_of(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    return p.R == 64 ? run_rows<T, D, 64, kQ4>(q, a, p, scratch, out, lse, st) : run_rows<T, D, 128, kQ4>(q, a, p, scratch, out, lse, st);
}
template <bool kQ4>
static cudaError_t rows_for(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    if (dtype == SLA_F32) return a.c.D == 64 ? rows_of<float, 64, kQ4>(q, a, p, scratch, out, lse, st) : rows_of<float, 128, kQ4>(q, a, p, scratch, out, lse, st);
    return a.c.D == 64 ? rows_of<__nv_bfloat16, 64, kQ4>(q, a, p, scratch, out, lse, st) : rows_of<__nv_bfloat16, 128, kQ4>(q, a, p, scratch, out, lse, st);
}

cudaError_t launch_paged_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                   float *lse, cudaStream_t st, long long *launches) {
    if (p.kind == PagedPlan::kDecode) return launch_paged_decode_attention(q, a, dtype, p, scratch, counters, out, lse, st, launches);
    cudaError_t e = launch_paged_plan(a, p, scratch, st);
    if (e == cudaSuccess && p.kind == PagedPlan::kTiles) {
        e = launch_paged_tiles(q, a, p, scratch, out, lse, st);
    } else if (e == cudaSuccess) {
        e = q4::is(a.c) ? rows_for<true>(q, a, dtype, p, scratch, out, lse, st) : rows_for<false>(q, a, dtype, p, scratch, out, lse, st);
    }
    if (e == cudaSuccess) e = launch_paged_merge(a, dtype, p, scratch, out, lse, st);
    if (e == cudaSuccess) *launches += 3;
    return e;
}

}  // namespace sla
