// Attention of a few rows over a range of keys of a cache in four bits, by a warp: what paged_decode (sla_paged_decode.cuh) calls in the place of
// attend_bf16.
//
// The codes go into mma.sync as the bf16 subnormals that q4::pairs makes of them, without their scales:
//     S^T [16 keys, 8 rows] = sum over groups of (C_g Q_g^T) s,      O^T [16 dimensions of a group, 8 rows] += C^T (P s)^T.
// A logit is the sum of four products of 32 dimensions, each times the scale of its group and key; a weight is multiplied by the scale of the
// value's group and rounded to bf16 once, which is what rounding the weight alone costs.  So no value is ever formed, and eight
// codes cost seven instructions.  P s goes through the 8 x 8 transpose (movmatrix) on its way into the second product.  (With the rows as
// A, so that P stays where it is, half of A is empty for groups of 8 and less: 400 instructions for 16 keys where this form then took 366.)
//
// A cache in four bits brings a quarter of the bytes for the same work: what matters is how many instructions a key takes, and that no warp ever
// waits for memory.  Every warp has a ring of stages of 32 keys in shared memory, which its lanes fill by asynchronous copies of 16
// bytes: nine instructions a stage, since a plane's rows lie on end.  (With the pieces in registers, requested a step of 16 keys ahead, as
// attend_bf16 has them, 32 sequences of 1000 to 65536 took 164 us.  Bulk copies take 40 instructions more a stage: their operands are
// those of a warp, and each lane's copy goes on its own.)
//
// Measured in a graph (32/8 heads, D 128, pages of 64 tokens): 32 sequences of 1000 to 65536 in 96 us, 4.8 TB/s of the cache's bytes (105 us call by call),
// D 64 66 us; 16 sequences of 500 to 30000 with up to four new tokens 38 us; one of 2^20 245 us, 4.9 TB/s.  No pipe is full (ALU 51 %, issue slots
// 54 %, DRAM 49 %): 290 instructions for 16 keys of a head, half of them on the ALU pipe, whose latencies three warps a scheduler do not cover.
//
// Powers of two: Q is multiplied by F, a power of two that brings its row's largest magnitude next to 2^125 (a sixteenth of it where codes
// carry a factor of 16); logits are divided by F 2^-133, in two steps where that and the softmax's scale make no fp32 number.  Weights are
// 2^78 times what they are: 2^78 2^40 2^8 (the largest scale, the slack of the running maximum) stays in the range of bf16, and products with
// subnormals down to 2^-133 2^78 2^-40 in that of fp32.
#pragma once

#include <math_constants.h>

#include "sla_q4.cuh"
#include "sla_tc_ptx.cuh"

namespace sla {
namespace q4 {

// d += A B, and d = A B
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ float half_of(uint32_t w, int i) { return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t y;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transpose(uint32_t x) {   // of an 8 x 8 matrix of 16-bit numbers
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

constexpr float kLift = 78.f;    // log2 of what the weights are multiplied by
constexpr int kKeys = 32;        // of a stage
constexpr int kStages = 2;       // (three: 32 sequences of 1000 to 65536 no faster)
__host__ __device__ constexpr int stage_bytes(int D) { return 2 * kKeys * (D / 2 + D / 16); }   // K codes, K scales, V codes, V scales
// of a warp: its stages, and behind them Q as the products take it
__host__ __device__ constexpr int ring_bytes(int D, int NT) { return kStages * stage_bytes(D) + NT * D * 16; }

// The codes of a stage lie in lines of 128 bytes (two rows, or four of 64 dimensions) of eight pieces of 16 bytes; piece x of line y has the place x ^ mix(y).
// A warp's loads then meet all banks: those of K have a row's pieces in neighbouring lanes, those of V the rows of four keys in four.
template <int D> __device__ __forceinline__ uint32_t mix(uint32_t line) { return D == 128 ? 2 * (line >> 1 & 3) : 4 * (line & 1) + (line & 2); }

// 8 NT rows at most, four where kFour; Walk, w_m, w_l and w_o as for attend_bf16, w_o over the ring, but the warp takes 32 keys at a time.  A thread
// (g, c) = (lane / 4, lane % 4) has of the products' operands (16 keys a step) the keys ka = 4 (g / 2) + g % 2 and kb = ka + 2 of K, S and P, row g of Q (and g + 8) and
// the values of keys 4 c .. 4 c + 3.
//
// kFour: the products' eight columns have the four rows twice.  The weights of the first four are scaled for a group, those of the others for the next
// group, so that one operand P s serves the products of both: of the first group's, columns 0 to 3 are results, of the second's 4 to 7.
// (With the places of the codes mixed, 309 instructions for 16 keys instead of 319, 32 sequences of 1000 to 65536 104 us instead of 107.)
template <int D, int NT, bool kTok, bool kFour, int kWarps, typename Walk>
__device__ __forceinline__ void attend(const __nv_bfloat16 *__restrict__ q, const PagedCall &a, const Walk &wk, uint32_t ring, float *w_m, float *w_l, float *w_o) {
    constexpr int N = D / 32, kStride = kKeys * kWarps, S = kKeys / 16;
    constexpr unsigned kAll = 0xffffffffu;
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int G = a.G, first = wk.first, n = wk.n, key_end = wk.key_end;

    // A stage's keys lie in one page, or in two of 16 tokens: where the rows begin in k and in v, looked up a stage ahead of the copies.
    const bool small = a.c.P < kKeys;
    const int sl = lane % (D / 8);   // of the scales: 16 bytes a lane, K and then V
    const char *const s_pool = (lane < D / 8 ? a.c.k : a.c.v) + wk.head * a.c.s_h + a.c.P * (D / 2) + sl * 16 - (small && sl >= D / 16 ? D : 0);
    const char *const k_pool = a.c.k + wk.head * a.c.s_h + lane * 16, *const v_pool = a.c.v + wk.head * a.c.s_h + lane * 16;
    // where a lane's pieces go: of the lines lane / 8 and that + 4, whose places differ
    const uint32_t code_to[2] = {(lane >> 3) * 128 + ((lane & 7) ^ mix<D>(lane >> 3)) * 16, (lane >> 3) * 128 + ((lane & 7) ^ mix<D>((lane >> 3) + 4)) * 16};
    const uint32_t s_to = ring + (lane < D / 8 ? 0 : stage_bytes(D) / 2) + kKeys * (D / 2) + sl * 16;
    // the row in column 8 t + x of the products, and those in a thread's columns of their results
    auto row_of = [&](int t, int x) { return kFour ? x & 3 : 8 * t + x; };
    auto page_at = [&](int k) { return valid_page(a.c, __ldg(wk.table + (k >> a.c.shift))) * a.c.s_page; };
    long long at0 = 0, at1 = 0;
    auto find = [&](int k0) {
        if (k0 >= key_end) return;
        at0 = page_at(k0);
        if (small) at1 = page_at(min(k0 + 16, n - 1));
    };
    auto fill = [&](int k0, uint32_t st) {
        if (k0 < key_end) {
            const uint32_t to = ring + st * stage_bytes(D), v_to = to + stage_bytes(D) / 2;
            if (!small) {
                const int t0 = k0 & (a.c.P - 1);
                const char *const k_src = k_pool + at0 + t0 * (D / 2), *const v_src = v_pool + at0 + t0 * (D / 2);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    ptx::cp_async16(to + code_to[j & (N / 2 - 1)] + j * 512, k_src + j * 512);
                    ptx::cp_async16(v_to + code_to[j & (N / 2 - 1)] + j * 512, v_src + j * 512);
                }
                if (D == 128 || lane < D / 4) ptx::cp_async16(s_to + st * stage_bytes(D), s_pool + at0 + t0 * (D / 16));
            } else {
                const bool two = k0 + 16 < n;   // what lies beyond n is not copied where it has a page of its own
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j < N / 2 || two) {
                        const long long from = (j < N / 2 ? at0 : at1) + (j & (N / 2 - 1)) * 512;
                        ptx::cp_async16(to + code_to[j & (N / 2 - 1)] + j * 512, k_pool + from);
                        ptx::cp_async16(v_to + code_to[j & (N / 2 - 1)] + j * 512, v_pool + from);
                    }
                if (lane < D / 4 && (sl < D / 16 || two)) ptx::cp_async16(s_to + st * stage_bytes(D), s_pool + (sl < D / 16 ? at0 : at1));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int key = wk.key;
#pragma unroll
    for (int st = 0; st < kStages; ++st) {
        find(key + st * kStride);
        fill(key + st * kStride, st);
    }
    find(key + kStages * kStride);
    const uint32_t q_at = ring + kStages * stage_bytes(D) + lane * 16;   // (a lane reads what it wrote)
    // [t][e]: row 8 t + 2 c + e
    float m[NT][2], l[NT][2], lim[NT][2], base[NT][2], mult[NT][2], acc[NT][2 * N][4];
    int top_e[NT], most_e = -2;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        uint32_t qf[N][4];
        const bool on = row_of(t, g) < (kTok ? wk.rows : G);
        const int r = on ? row_of(t, g) : 0, tok = kTok ? r / G : 0;
        const __nv_bfloat16 *src = q + (long long)(wk.row_q + tok) * a.q_st + (long long)(wk.head * G + r - tok * G) * a.q_sh + c * 8;
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < N; ++w) {
            const uint4 v = on ? __ldg(reinterpret_cast<const uint4 *>(src + 32 * w)) : make_uint4(0, 0, 0, 0);
            qf[w][0] = v.x; qf[w][1] = v.y; qf[w][2] = v.z; qf[w][3] = v.w;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = __vmaxu2(top, qf[w][i] & 0x7fff7fffu);
        }
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(kAll, top, 1));
        top = max(top, __shfl_xor_sync(kAll, top, 2));
        // exponent of the row's largest magnitude, kept where F is a number; F = 2^(125 - e)
        const int e = min(max((int)(top >> 7) - 127, -2), 127);
        const float f0 = __uint_as_float((uint32_t)(252 - e) << 23), f1 = __uint_as_float((uint32_t)(248 - e) << 23);
#pragma unroll
        for (int w = 0; w < N; ++w) {
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[w][i] = pack(half_of(qf[w][i], 0) * (i & 1 ? f1 : f0), half_of(qf[w][i], 1) * (i & 1 ? f1 : f0));
            ptx::st_shared_v4(q_at + (t * N + w) * 512, qf[w]);
        }
        top_e[t] = e;
        most_e = max(most_e, e);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            m[t][u] = lim[t][u] = -CUDART_INF_F;
            base[t][u] = kLift;
            l[t][u] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[t][i][u] = 0.f;
    }
    // What a logit's products are multiplied by: scale 2^(8 + e), which is no fp32 number for queries of 2^125 and a scale of 2^-4, say.  Then the
    // products, below 2^44, take 2^72 of it beforehand.  (scale is below 2^64.)
    const float scale2 = a.scale * kLog2e;
    const bool far = __any_sync(kAll, fabsf(scale2) * __uint_as_float((uint32_t)(63 + most_e) << 23) >= 0x1p55f);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float back = far ? scale2 * __uint_as_float((uint32_t)(63 + top_e[t]) << 23) : scale2 * __uint_as_float((uint32_t)(127 + top_e[t]) << 23) * 0x1p8f;
#pragma unroll
        for (int u = 0; u < 2; ++u) mult[t][u] = __shfl_sync(kAll, back, 4 * (2 * c + u));
    }

    const uint32_t ka = 4 * (g >> 1) + (g & 1);
    // (of 16 s + row, where the rows' numbers add up without carries into what mix() looks at: a line is row * D / 256)
    constexpr int kLine = 256 / D;   // rows of a line
    auto code_at = [&](int row, int byte) { return row / kLine * 128u + (((row % kLine * (D / 2) + byte) / 16) ^ mix<D>(row / kLine)) * 16 + byte % 16; };
    const uint32_t k_at[2] = {ring + code_at(ka, c * 4 * N), ring + code_at(ka + 2, c * 4 * N)};
    const uint32_t v_at[2] = {ring + stage_bytes(D) / 2 + code_at(4 * c, g * 2 * N), ring + stage_bytes(D) / 2 + code_at(4 * c + 1, g * 2 * N)};
    const uint32_t s_at = ring + kKeys * (D / 2) + ka * (D / 16);
    const uint32_t four = c < 2 ? 0x1044u : 0x3244u;   // kFour: the columns' scale of a word of two, as a float
    uint32_t st = 0;
#pragma unroll 1
    for (; key < key_end; key += kStride) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();   // every lane's copies are there
        const uint32_t of = st * stage_bytes(D);
        float y[S][NT][4];   // [s][t][2 h + e]: key 16 s + ka + 2 h, row 8 t + 2 c + e
#pragma unroll
        for (int s = 0; s < S; ++s) {
            uint32_t kw[2][N], ks[2][N / 2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                load_shared(k_at[h] + of + 16 * s * (D / 2), kw[h]);
                load_shared(s_at + of + (16 * s + 2 * h) * (D / 16), ks[h]);
            }
#pragma unroll
            for (int w = 0; w < N; ++w) {
                uint32_t qf[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t) load_shared(q_at + (t * N + w) * 512, qf[t]);
                uint32_t ra[4], rb[4];
                pairs(kw[0][w], ra);
                pairs(kw[1][w], rb);
                const float sa = half_of(ks[0][w >> 1], w), sb = half_of(ks[1][w >> 1], w);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float d[4];
                    mma0(d, ra[0], rb[0], ra[1], rb[1], qf[t][0], qf[t][1]);
                    mma(d, ra[2], rb[2], ra[3], rb[3], qf[t][2], qf[t][3]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) y[s][t][u] = w == 0 ? d[u] * (u < 2 ? sa : sb) : fmaf(d[u], u < 2 ? sa : sb, y[s][t][u]);
                }
            }
        }
        if (far) {   // (a jump on its own: selecting the factor for each product took 96.6 us for 32 sequences of 1000 to 65536, this 95.9)
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int u = 0; u < 4; ++u) y[s][t][u] *= 0x1p72f;
        }
        // a logit less what the row's weights are taken from, m - 78 (m: not below the largest so far but by 8; 0 for none)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    y[s][t][u] = fmaf(y[s][t][u], mult[t][u], base[t][u]);
                    y[s][t][u + 2] = fmaf(y[s][t][u + 2], mult[t][u], base[t][u]);
                }
            }
        uint32_t vs[S][2][N / 2];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) load_shared(s_at + of + stage_bytes(D) / 2 + (16 * s + 2 * h) * (D / 16), vs[s][h]);
        const bool edge = kTok ? key < wk.all_first || key + kKeys > wk.all_n : key < first || key + kKeys > n;
        if (edge) {
            uint32_t nan = 0;   // of the keys that some rows see and others do not: bit 8 s + 4 h + group
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = key + 16 * s + (int)ka + 2 * h;
                    int lo = 0, hi = 8 * NT;
                    if constexpr (kTok) wk.rows_of(k, G, lo, hi);
                    if (k < first || k >= n) hi = 0;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            if (row_of(t, 2 * c + u) < lo || row_of(t, 2 * c + u) >= hi) y[s][t][2 * h + u] = -CUDART_INF_F;
                    const bool part = kTok && hi > 0 && (k < wk.all_first || k >= wk.all_n);
#pragma unroll
                    for (int w = 0; w < N; ++w) {
                        const uint32_t mask = w & 1 ? 0xffff0000u : 0xffffu;
                        const bool out = part && is_nan((w & 1 ? vs[s][h][w >> 1] >> 16 : vs[s][h][w >> 1]) & 0xffffu);
                        if (out) nan |= 1u << (8 * s + 4 * h + w);
                        if (hi == 0 || out) vs[s][h][w >> 1] &= ~mask;   // what no row sees may be anything
                    }
                }
            if (kTok && __any_sync(kAll, nan != 0)) {
                // 0 times NaN is NaN: such a group is left out of the product and put into the rows that see its key
#pragma unroll 1
                for (int i = 0; i < kKeys; ++i) {
                    const uint32_t groups = __shfl_sync(kAll, nan, 8 * (i >> 2 & 3) + 4 * (i & 1)) >> (8 * (i >> 4) + 2 * (i & 2));
                    int lo, hi;
                    wk.rows_of(key + i, G, lo, hi);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int w = 0; w < N; ++w)
                                if ((groups >> w & 1) && row_of(t, 2 * c + u) >= lo && row_of(t, 2 * c + u) < hi)
                                    acc[t][2 * w][u] = acc[t][2 * w][u + 2] = acc[t][2 * w + 1][u] = acc[t][2 * w + 1][u + 2] = CUDART_NAN_F;
                }
            }
        }
        bool over = false;
        float up[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                up[t][u] = fmaxf(y[0][t][u], y[0][t][u + 2]);
#pragma unroll
                for (int s = 1; s < S; ++s) up[t][u] = fmaxf(up[t][u], fmaxf(y[s][t][u], y[s][t][u + 2]));
                over |= up[t][u] > lim[t][u];
            }
        if (__any_sync(kAll, over)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float was = kLift - base[t][u];
                    float top = up[t][u];
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(kAll, top, off));
                    const float mx = fmaxf(m[t][u], top - kLift + was);
                    const float keep = m[t][u] == mx ? 1.f : ex2(m[t][u] - mx), by = mx == -CUDART_INF_F ? 0.f : was - mx;
                    m[t][u] = mx;
                    lim[t][u] = mx == -CUDART_INF_F ? mx : kLift + 8.f;
                    base[t][u] = kLift - (mx == -CUDART_INF_F ? 0.f : mx);
                    l[t][u] *= keep;
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        y[s][t][u] += by;
                        y[s][t][u + 2] += by;
                    }
#pragma unroll
                    for (int i = 0; i < 2 * N; ++i) {
                        acc[t][i][u] *= keep;
                        acc[t][i][u + 2] *= keep;
                    }
                }
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    y[s][t][u] = ex2(y[s][t][u]);
                    l[t][u & 1] += y[s][t][u];
                }
            uint32_t vw[4][N / 2];
#pragma unroll
            for (int i = 0; i < 4; ++i) load_shared(D == 128 ? v_at[i & 1] + of + (16 * s + (i & 2)) * (D / 2) : (v_at[i & 1] ^ (i & 2) * 32) + of + 16 * s * (D / 2), vw[i]);
            uint32_t b0[NT], b1[NT];   // P s
#pragma unroll
            for (int w = 0; w < N; ++w) {
                uint32_t ra[4], rb[4];   // codes of keys 4 c, 4 c + 1; of 4 c + 2, 4 c + 3
                const uint32_t sel = w & 1 ? 0x7632u : 0x5410u;
                pairs(__byte_perm(vw[0][w >> 1], vw[1][w >> 1], sel), ra);
                pairs(__byte_perm(vw[2][w >> 1], vw[3][w >> 1], sel), rb);
                if (!kFour || w % 2 == 0) {
                    const float sa = kFour ? __uint_as_float(__byte_perm(vs[s][0][w >> 1], 0, four)) : half_of(vs[s][0][w >> 1], w);
                    const float sb = kFour ? __uint_as_float(__byte_perm(vs[s][1][w >> 1], 0, four)) : half_of(vs[s][1][w >> 1], w);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        b0[t] = transpose(pack(y[s][t][0] * sa, y[s][t][1] * sa));
                        b1[t] = transpose(pack(y[s][t][2] * sb, y[s][t][3] * sb));
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mma(acc[t][2 * w], ra[0], ra[1], rb[0], rb[1], b0[t], b1[t]);
                    mma(acc[t][2 * w + 1], ra[2], ra[3], rb[2], rb[3], b0[t], b1[t]);
                }
            }
        }
        __syncwarp();   // the stage has been read
        fill(key + kStages * kStride, st);
        find(key + (kStages + 1) * kStride);
        st = st + 1 == kStages ? 0 : st + 1;
    }

    // ---- the warp's sums: row g of tile 2 w + i is dimension 32 w + 8 (g / 2) + g % 2 + 4 i, row g + 8 that + 2
    __syncwarp();
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = row_of(t, 2 * c + u);
            float v = l[t][u];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) v += __shfl_xor_sync(kAll, v, off);
            if (g == 0 && (!kFour || c < 2)) { w_m[r] = m[t][u]; w_l[r] = v * 0x1p-78f; }
#pragma unroll
            for (int w = 0; w < N; ++w) {
                if (kFour && (w & 1) != (c >> 1)) continue;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float *o = w_o + r * D + 32 * w + 8 * (g >> 1) + (g & 1) + 4 * i;
                    o[0] = acc[t][2 * w + i][u] * 0x1p55f;
                    o[2] = acc[t][2 * w + i][u + 2] * 0x1p51f;
                }
            }
        }
}

}  // namespace q4
}  // namespace sla
