// Attention of one new token a sequence over a paged cache, or of so few that tokens x heads of a group are at most 16 rows (a step that
// checks guessed tokens).  One launch.
//
// All rows of a KV head share its keys, so that K and V are read once: bound by HBM.  (The heads below are rows.)  The bound of 16 is
// what the registers hold.  Against the kernels of chunks, D 128: 32 sequences of 198 tokens with 1 to 3 new ones, 8/2 heads, 11.5 us
// here and 22 there; 28 of 14 to 583, 32/8 heads, 17 and 27; 32 of 1000 to 65536 with 4, 272 and 268; fp32, 16 of 1000 to 20000 with 4,
// 259 and 581.
//
// bf16 (attend_bf16): the products run on the tensor
// cores by mma.sync with the keys as the 16 rows of A and the heads as the 8 columns of B,
//     S^T [16 keys, 8 heads] = K Q^T,      O^T [D, 8 heads] += V^T P^T,
// which wastes nothing for groups of 8 and needs no shared memory on the way: a thread fetches pieces of 16 bytes of its rows
// straight into the registers of the A operand.  The order of the D dimensions inside a product is free (Q is fetched in the same
// order), and a row of V^T is any dimension, so that pieces stay whole; pairs of neighbouring keys are put together by a byte
// permutation, P^T is the 8 x 8 transpose of P (movmatrix).  A warp goes through 16 keys at a time -- they lie in one page -- with
// the keys of the next step fetched as soon as these are used up, and the values after them.
//
// fp32 (attend_f32): on the FMA pipe, 32 keys a step and warp.  For S a lane has a key of its own and goes along its row, the heads' queries
// broadcast from shared memory; for O a lane has dimensions of its own and the warp goes along the keys, the weights
// broadcast: no sum crosses lanes.
//
// The running maximum of a head moves only when a logit passes it by 2^8 (a factor that neither the fp32 sums nor the bf16 weights
// notice), decided by one vote of the warp.  Sums are fp32; in bf16 a weight is rounded before it meets its value, as the tensor
// cores want it, and the denominator adds the unrounded weights.
//
// The units (sequence, KV head) of the call lie end to end, weighted by their keys, and are cut into as many equal ranges as there
// are CTAs.  The CTA that finishes a cut unit last joins the partial results, in the order of the ranges.
//
// Measured (32/8 heads, D 128, pages of 64 tokens, bf16): 32 sequences of 200 to 65536 tokens in 246 us, 6.64 TB/s, as fast as a copy
// (ncu: issue slots 26 %, tensor pipe 10 %, 168 registers); 4 of 17 to 700 (8/2 heads, D 64,
// pages of 16) in 8.6 us, which is the launch and a chain of dependent
// loads (lengths, table, keys, values, counters).  fp32, 16 sequences of 1000 to 20000: 149 us.
#include <math_constants.h>

#include "sla_paged_attn.h"

namespace sla {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
// resident CTAs an SM: two where 16 heads of 128 dimensions fill the registers
__host__ __device__ constexpr int ctas_per_sm(int D, int NT) { return D == 128 && NT == 2 ? 2 : 3; }
// sequences of a launch: as many as there is room for (16 bytes each) beside the kernel's arrays in 48 KB
template <typename T> constexpr int max_seqs(int D, int NT) {
    const int arrays = kWarps * 8 * NT * (D + 2) * 4 + (sizeof(T) == 4 ? D * 8 * NT * 4 : 16) + 128, room = (48 * 1024 - arrays) / 16 - 1;
    return room < 1024 ? room : 1024;
}
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
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float a, float b, float c, float d) { *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d)); }
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// What one warp does of a segment: the keys key, key + stride, .. below key_end in steps of the path's own, of which those in [first, n) count,
// for the G heads of KV head `head`.  Its maxima, sums and weighted values go to w_m, w_l [heads] and w_o [heads][D].
// With several new tokens (kTok) the rows are tokens x heads: row r is head r % G of token r / G.
struct Walk {
    int key, key_end, first, n, head, row_q;
    const int *table;
    int q, rows, window;   // tokens; rows; 0: no window
    // all rows see the keys [all_first, all_n)
    int all_first, all_n;
    // the rows that see key k of [first, n)
    __device__ __forceinline__ void rows_of(int k, int G, int &lo, int &hi) const {
        const int t = k - (n - q);   // the token at k
        lo = max(t, 0) * G;
        hi = window > 0 && t + window < q ? (t + window) * G : rows;
    }
};

template <int D, int NT, bool kTok>
__device__ __forceinline__ void attend_bf16(const __nv_bfloat16 *__restrict__ q, const PagedCall &a, const Walk &wk, float *w_m, float *w_l, float *w_o) {
    constexpr int kChunks = D / 32;       // 16-byte pieces of a key row per thread
    constexpr int kVChunks = D / 64;      // of a value row
    constexpr int kMt = D / 16;           // m-tiles of O^T
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int G = a.G, first = wk.first, n = wk.n, head = wk.head, row_q = wk.row_q, key_end = wk.key_end;
    const int *table = wk.table;
    const float scale2 = a.scale * kLog2e;
    int key = wk.key;
    float m[NT][2], l[NT][2], acc[NT][kMt][4];
    uint32_t qf[NT][kChunks][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const bool on = 8 * t + g < (kTok ? wk.rows : G);
        const int r = on ? 8 * t + g : 0, tok = kTok ? r / G : 0;
        const __nv_bfloat16 *src = q + (long long)(row_q + tok) * a.q_st + (long long)(head * G + r - tok * G) * a.q_sh + c * 8;
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
        const bool edge = kTok ? key < wk.all_first || key + 16 > wk.all_n : key < first || key + 16 > n;
        if (edge) {
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                const int kk = key + g + 8 * e2;
                int lo = 0, hi = 8 * NT;
                if constexpr (kTok) wk.rows_of(kk, G, lo, hi);
                if (kk < first || kk >= n) hi = 0;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (8 * t + 2 * c + e < lo || 8 * t + 2 * c + e >= hi) s[t][2 * e2 + e] = -CUDART_INF_F;
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
        if constexpr (kTok) {
            // keys that some rows see and others do not: 0 times a value that is not finite is NaN.  Where there is one, the products of these
            // keys are left out of the MMA and added row by row.
            if (edge) {
                bool part[4];
                uint32_t bad = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = key + 2 * c + (e & 1) + 8 * (e >> 1);
                    part[e] = k < wk.all_first || k >= wk.all_n;
#pragma unroll
                    for (int j = 0; j < kVChunks; ++j)
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (part[e]) bad |= ((word(vr[e][j], u) & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // exponent all ones
                }
                if (__any_sync(0xffffffffu, bad != 0)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < kVChunks; ++j)
                            if (part[e]) vr[e][j] = make_uint4(0, 0, 0, 0);
                    const __nv_bfloat16 *vs = vb + find(key);
#pragma unroll 1
                    for (int kk = 0; kk < 16; ++kk) {
                        const int k = key + kk;
                        if (k < first || k >= n || (k >= wk.all_first && k < wk.all_n)) continue;
                        int lo, hi;
                        wk.rows_of(k, G, lo, hi);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float wt = __shfl_sync(0xffffffffu, kk < 8 ? s[t][e] : s[t][e + 2], (kk & 7) * 4 + c);
                                const int r = 8 * t + 2 * c + e;
                                if (r < lo || r >= hi) continue;
#pragma unroll
                                for (int i = 0; i < kMt; ++i) {
                                    acc[t][i][e] = fmaf(wt, __bfloat162float(vs[(long long)kk * a.c.s_t + 8 * g + i]), acc[t][i][e]);
                                    acc[t][i][e + 2] = fmaf(wt, __bfloat162float(vs[(long long)kk * a.c.s_t + (D == 128 ? 64 + 8 * g + i : 8 * g + 4 + i)]), acc[t][i][e + 2]);
                                }
                            }
                    }
                }
            }
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

    // ---- the warp's sums
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float v = l[t][e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
            const int qi = 8 * t + 2 * c + e;
            if (g == 0) { w_m[qi] = m[t][e]; w_l[qi] = v; }
#pragma unroll
            for (int i = 0; i < kMt; ++i) {
                w_o[qi * D + 8 * g + i] = acc[t][i][e];
                w_o[qi * D + (D == 128 ? 64 + 8 * g + i : 8 * g + 4 + i)] = acc[t][i][e + 2];
            }
        }
}

// fp32: S by lanes of a key each, O by lanes of D / 32 dimensions each.  s_q: the queries [D][8 NT], scaled.
template <int D, int NT, bool kTok>
__device__ __forceinline__ void attend_f32(const PagedCall &a, const Walk &wk, const float *s_q, float *w_m, float *w_l, float *w_o) {
    float *s_p = w_o;   // a step's weights, until the sums are written
    constexpr int H = 8 * NT, N = D / 32, kDeep = 8;   // heads, dimensions of a lane, loads in flight
    const int lane = threadIdx.x & 31, first = wk.first, n = wk.n;
    const float *kb = reinterpret_cast<const float *>(a.c.k) + wk.head * a.c.s_h;
    const float *vb = reinterpret_cast<const float *>(a.c.v) + wk.head * a.c.s_h + lane * N;
    auto row_of = [&](int j) { return valid_page(a.c, __ldg(wk.table + (j >> a.c.shift))) * a.c.s_page + (long long)(j & (a.c.P - 1)) * a.c.s_t; };
    float m[H], l[H], acc[H][N];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        m[h] = -CUDART_INF_F;
        l[h] = 0.f;
#pragma unroll
        for (int d = 0; d < N; ++d) acc[h][d] = 0.f;
    }
    for (int key = wk.key; key < wk.key_end; key += 32 * kWarps) {
        const int j = key + lane;
        const bool on = j >= first && j < n && j < wk.key_end;
        const long long at = row_of(on ? j : min(max(first, 0), n - 1));
        const float *kr = kb + at;
        float s[H];
#pragma unroll
        for (int h = 0; h < H; ++h) s[h] = 0.f;
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 4 * kDeep) {
            float4 k4[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) k4[u] = __ldg(reinterpret_cast<const float4 *>(kr + d0 + 4 * u));
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float kk = e == 0 ? k4[u].x : e == 1 ? k4[u].y : e == 2 ? k4[u].z : k4[u].w;
#pragma unroll
                    for (int h = 0; h < H; h += 4) {
                        const float4 q4 = *reinterpret_cast<const float4 *>(s_q + (d0 + 4 * u + e) * H + h);
                        s[h] = fmaf(q4.x, kk, s[h]); s[h + 1] = fmaf(q4.y, kk, s[h + 1]);
                        s[h + 2] = fmaf(q4.z, kk, s[h + 2]); s[h + 3] = fmaf(q4.w, kk, s[h + 3]);
                    }
                }
        }
        bool over = false;
        int lo = 0, hi = H;   // rows that see the lane's key
        if constexpr (kTok) {
            wk.rows_of(j, a.G, lo, hi);
            if (!on) hi = 0;
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (kTok ? h < lo || h >= hi : !on) s[h] = -CUDART_INF_F;
            over |= s[h] > m[h] + 8.f;
        }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float mx = fmaxf(m[h], s[h]);
#pragma unroll
                for (int off = 16; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                const float keep = m[h] == mx ? 1.f : exp2_fast(m[h] - mx);
                m[h] = mx;
                l[h] *= keep;
#pragma unroll
                for (int d = 0; d < N; ++d) acc[h][d] *= keep;
            }
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
            s[h] = exp2_fast(s[h] - (m[h] == -CUDART_INF_F ? 0.f : m[h]));
            l[h] += s[h];
        }
        __syncwarp();
#pragma unroll
        for (int h = 0; h < H; h += 4) *reinterpret_cast<float4 *>(s_p + lane * H + h) = make_float4(s[h], s[h + 1], s[h + 2], s[h + 3]);
        __syncwarp();
        const unsigned seen = __ballot_sync(0xffffffffu, on);   // values of other keys may be anything: they are not read
        const unsigned part = kTok ? __ballot_sync(0xffffffffu, on && (j < wk.all_first || j >= wk.all_n)) : 0u;   // not every row sees them
#pragma unroll 1
        for (int i0 = 0; i0 < 32; i0 += kDeep) {
            float v[kDeep][N];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const long long to = __shfl_sync(0xffffffffu, at, i0 + u);
#pragma unroll
                for (int d = 0; d < N; ++d) v[u][d] = 0.f;
                if (seen >> (i0 + u) & 1) {
                    if constexpr (N == 4) *reinterpret_cast<float4 *>(v[u]) = __ldg(reinterpret_cast<const float4 *>(vb + to));
                    else *reinterpret_cast<float2 *>(v[u]) = __ldg(reinterpret_cast<const float2 *>(vb + to));
                }
            }
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                int lo_u = 0, hi_u = H;
                if (kTok && (part >> (i0 + u) & 1)) wk.rows_of(j - lane + i0 + u, a.G, lo_u, hi_u);
#pragma unroll
                for (int h = 0; h < H; h += 4) {
                    const float4 p4 = *reinterpret_cast<const float4 *>(s_p + (i0 + u) * H + h);
                    const float pp[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int d = 0; d < N; ++d)
                            if (!kTok || (h + e >= lo_u && h + e < hi_u)) acc[h + e][d] = fmaf(pp[e], v[u][d], acc[h + e][d]);
                }
            }
        }
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
        float sum = l[h];
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (lane == 0) { w_m[h] = m[h]; w_l[h] = sum; }
        if (h == 0) __syncwarp();   // the weights have been read
#pragma unroll
        for (int d = 0; d < N; ++d) w_o[h * D + lane * N + d] = acc[h][d];
    }
}

template <typename T, int D, int NT, bool kTok>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(D, NT))
paged_decode(const T *__restrict__ q, PagedCall a, int x_base, int n_seqs, Parts parts, int *__restrict__ done,
             T *__restrict__ out, float *__restrict__ lse) {
    constexpr int R = 16;                 // rows of a partial result
    __shared__ alignas(16) float s_o[kWarps][8 * NT][D];
    __shared__ float s_m[kWarps][8 * NT], s_l[kWarps][8 * NT];
    __shared__ long long s_scan[kWarps];
    __shared__ int s_last;
    extern __shared__ long long s_seq_at[];   // [n_seqs + 1] weight before a sequence; then its tokens and its slot
    int *s_n = reinterpret_cast<int *>(s_seq_at + n_seqs + 1), *s_slot = s_n + n_seqs;
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kStep = kF32 ? 32 : 16;   // keys of a warp's step
    __shared__ alignas(16) float s_q[kF32 ? D * 8 * NT : 4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = a.G;
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
                else n = tokens_of(a.c, a.first, x_base + x, slot);
                s_n[x] = n;
                s_slot[x] = slot;
                if (hi > lo) {
                    const int q_x = kTok ? hi - lo : 1;
                    if (hi - lo > a.b.max_new) atomicOr(a.c.status, kStatusBadIndex);   // (no more than max_new of its rows are computed)
                    unit_tiles(n, q_x, 0, q_x, a.window, kTileShift, lo, hi);
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
    const long long each = total / n_ranges;
    const Ranges ranges = {each, n_ranges, (int)(total - each * n_ranges)};
    long long w = ranges.at(r);
    const long long w_end = ranges.at(r + 1);
    if (w >= w_end) return;
    int x = warp_last_le(s_seq_at, n_seqs, w);
    long long per_head = (s_seq_at[x + 1] - s_seq_at[x]) / a.c.Hkv;
    int head = (int)quotient(w - s_seq_at[x], per_head);

    while (true) {
        const long long start = s_seq_at[x] + head * per_head, stop = start + per_head;
        const int n = s_n[x];
        int lo, hi, row_q;
        new_rows(a.b, x_base + x, row_q, hi);
        const int q_x = kTok ? hi - row_q : 1, rows = kTok ? min(q_x, a.b.max_new) * G : G;
        unit_tiles(n, q_x, 0, q_x, a.window, kTileShift, lo, hi);
        const int from = (int)(w - start), to = (int)((w_end < stop ? w_end : stop) - start);
        // keys seen by any row [first, n), by all rows [all_first, all_n)
        const int window = a.window > 0 && a.window < n ? a.window : 0;
        const int all_first = window > 0 ? n - window : 0, all_n = n - q_x + 1, first = max(all_first - q_x + 1, 0);
        const int key = max((lo + max(from - kUnitWeight, 0)) << kTileShift, first & ~(kStep - 1));
        const int key_end = min((lo + max(to - kUnitWeight, 0)) << kTileShift, n);
        const Walk walk = {key + kStep * warp, key_end, first, n, head, row_q, a.c.table + (long long)max(s_slot[x], 0) * a.c.width, q_x, rows, window, all_first, all_n};
        if constexpr (kF32) {
            // (s_q: the segment before has been joined)
            for (int c = tid; c < D * 8 * NT; c += kThreads) {
                const int h = c / D, d = c % D;   // neighbouring threads, neighbouring dimensions
                const int tok = kTok ? h / G : 0;
                s_q[d * 8 * NT + h] = h < rows ? q[(long long)(row_q + tok) * a.q_st + (long long)(head * G + h - tok * G) * a.q_sh + d] * (a.scale * kLog2e) : 0.f;
            }
            __syncthreads();
            attend_f32<D, NT, kTok>(a, walk, s_q, s_m[warp], s_l[warp], &s_o[warp][0][0]);
        } else {
            attend_bf16<D, NT, kTok>(q, a, walk, s_m[warp], s_l[warp], &s_o[warp][0][0]);
        }
        __syncthreads();
        const bool begins = from == 0, ends = w_end >= stop;
        const int part = begins && ends ? -1 : begins ? 2 * r + 1 : 2 * r;
        for (int it = tid; it < rows * (D / 4); it += kThreads) {
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
                const int tok = kTok ? qi / G : 0, h = head * G + qi - tok * G;
                store4(out + (long long)(row_q + tok) * a.q_st + (long long)h * a.q_sh + d, o[0], o[1], o[2], o[3]);
                if (d == 0) lse[(long long)(row_q + tok) * a.Hq + h] = z * kLn2;
            } else {
                if (!none) __stcg(reinterpret_cast<float4 *>(parts.o + ((long long)part * R + qi) * D + d), make_float4(o[0], o[1], o[2], o[3]));
                if (d == 0) __stcg(parts.lse2 + (long long)part * R + qi, z);
            }
        }
        if (part >= 0) {
            // ranges [r0, r1] hold this unit
            const int r0 = begins ? r : ranges.holding(start), r1 = ends ? r : ranges.holding(stop - 1), n_parts = r1 - r0 + 1;
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
                for (int it = tid; it < rows * (D / 4); it += kThreads) {
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
                    const int tok = kTok ? qi / G : 0, h = head * G + qi - tok * G;
                    store4(out + (long long)(row_q + tok) * a.q_st + (long long)h * a.q_sh + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
                    if (d == 0) lse[(long long)(row_q + tok) * a.Hq + h] = none ? -CUDART_INF_F : (mx + log2f(sum)) * kLn2;
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

bool paged_decode_supported(const PagedCall &a) { return (long long)a.b.max_new * a.G <= 16; }

void plan_paged_decode(const PagedCall &a, PagedPlan &p, int sm_count) {
    p.R = p.RS = 16;
    p.TS = p.TQ = 1;
    p.n_ctas = ctas_per_sm(a.c.D, a.b.max_new * a.G <= 8 ? 1 : 2) * sm_count;
}

template <typename T, int D, int NT, bool kTok>
static cudaError_t decode_of(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, int *counters, void *out, float *lse,
                             cudaStream_t st, long long *launches) {
    cudaError_t e = cudaSuccess;
    constexpr int kMost = max_seqs<T>(D, NT);
    for (int x0 = 0; x0 < a.b.n_seqs && e == cudaSuccess; x0 += kMost) {
        const int n = a.b.n_seqs - x0 < kMost ? a.b.n_seqs - x0 : kMost;
        e = launch_chained(paged_decode<T, D, NT, kTok>, dim3(p.n_ctas), dim3(kThreads), (size_t)(n + 1) * 8 + (size_t)n * 8, st,
                           (const T *)q, a, x0, n, parts_at(p, scratch), counters, (T *)out, lse);
        ++*launches;
    }
    return e;
}

template <typename T, int D>
static cudaError_t decode_for(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, int *counters, void *out, float *lse,
                              cudaStream_t st, long long *launches) {
    const bool small = a.b.max_new * a.G <= 8;
    if (a.b.max_new == 1)
        return small ? decode_of<T, D, 1, false>(q, a, p, scratch, counters, out, lse, st, launches) : decode_of<T, D, 2, false>(q, a, p, scratch, counters, out, lse, st, launches);
    return small ? decode_of<T, D, 1, true>(q, a, p, scratch, counters, out, lse, st, launches) : decode_of<T, D, 2, true>(q, a, p, scratch, counters, out, lse, st, launches);
}

cudaError_t launch_paged_decode_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                          float *lse, cudaStream_t st, long long *launches) {
    if (dtype == SLA_F32)
        return a.c.D == 64 ? decode_for<float, 64>(q, a, p, scratch, counters, out, lse, st, launches) : decode_for<float, 128>(q, a, p, scratch, counters, out, lse, st, launches);
    return a.c.D == 64 ? decode_for<__nv_bfloat16, 64>(q, a, p, scratch, counters, out, lse, st, launches)
                       : decode_for<__nv_bfloat16, 128>(q, a, p, scratch, counters, out, lse, st, launches);
}

}  // namespace sla
