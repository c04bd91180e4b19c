// Attention of chunks of new tokens over a paged cache, bf16: tcgen05 MMA with TMEM accumulators, pages by TMA.
//
// A unit is up to 256 rows of one (sequence, KV head): 256 / G neighbouring new tokens with all G heads of the group, as two
// streams of 128 rows.  Per tile of 128 keys and stream
//     S = Q K^T (smem x smem -> TMEM),   P = 2^(scale S - m) in registers, as bf16 back over S,   O += P V (TMEM x smem -> TMEM),
// with a reference maximum m per row that moves only when a logit passes it by 2^8 (then O and the sum are rescaled); sums in
// fp32.  While the row warps of one stream work on their S, the tensor pipe does the other's products.
//
// CTA of 512 threads, one per SM: warps 0-3 and 4-7 are the rows of the streams (a thread a row), 8-11 write results, 12 and 13
// issue a stream's MMAs, 14 fetches K and V (a box per page into a ring shared by both streams), 15 goes through the
// CTA's ranges of the plan (sla_paged.cuh), hands the segments on through a ring in shared memory and fetches their Q.
// Shared memory: Q 2 x 32 KB, ring 5 x 32 KB (K and V tiles in turn).  TMEM: O of the streams in columns 0 and 128, S in 256 and 384.
//
// Measured (32/8 heads, D 128, pages of 64 tokens): 8192 tokens that end at 65536 in 7.5 to 7.7 ms = 1070 to 1100 TFLOP/s at the power cap
// (1.59 GHz), 6.7 ms and 1230 in a single call; 1999 at 30011 in 0.95 to 0.98 ms, 990; 512 at 65536 in 0.54 ms, 1010; 64 at 65536 in 83 us, 3.2 TB/s.  D 64:
// four prompts of 2048 tokens in 135 us, 510 TFLOP/s.  Bound by the chain of a row warp: a tile takes a stream about 3400 cycles, of which its products take the tensor pipe
// 1000, so that two streams leave that pipe idle for two fifths of the time.
//
// Roundings to fewer bits: P goes into its product as bf16, which is what the tensor cores take; the denominator adds the weights
// before that rounding, whose errors (2^-9 each) are independent and average out over the keys.  The result is rounded once.
//
// A unit of one stream's rows or fewer -- the end of a chunk, a few tokens of a batch -- goes through both streams all the same, every
// second tile each, and the two sums are joined where the results are written: its tiles take half the time.  (24 sequences of 100 to 4000
// tokens, 1 to 300 new: 60 us, 69 where such a unit keeps to one stream.)
//
// Values in masked places: a masked weight is 0, and 0 times NaN is NaN, so a value that some row must not see may not enter the
// product unless it is finite.  Only the tiles at the edges of the mask hold such keys; there the row warps clear the values
// beyond the sequence's end (a page's stale rest) and look at the others; what is not finite is cleared too, and added to O of the
// rows that see its key when the segment's products are done (add_not_finite).
//
// A cache in four bits (kQ4): warp 14 brings pages of codes and scales (bulk copies) into a ring of their own, and the warps that write results make
// bf16 tiles of them, K and V in turn, where the copies would have put them: values times 2^-48, exact, one product a pair of codes (sla_q4.cuh).
// The ring of tiles is shorter by one.  8192 tokens that end at 65536 in 8.8 to 9.0 ms, 920 TFLOP/s (over bf16 7.4); 1999 at 30011 in 1.08 ms, 880 (0.93);
// 64 at 65536 in 109 us (84); four prompts of about 2000 tokens at D 64 in 180 us (127); 1 to 600 tokens of 16 sequences in 84 us (58).  What costs the
// rest against bf16 is the making: a chain of about 600 instructions a tile, which one warp on each scheduler takes about 3500 cycles for, as long as
// the rows take for theirs, while issue slots are 44 % used; and every unit that reads the same keys makes them again.  A unit of one stream's rows
// or fewer wants a tile every 1700 cycles and waits for it.  (Eight warps of 48 registers: 10.1 ms; codes read from
// global memory into registers a tile ahead: 1999 at 30011 1.18 ms, 1 to 600 tokens of 16 sequences 91 us instead of 84.)
//
// Every wait on an mbarrier is bounded; when one runs out the CTA sets a status bit, drains and leaves.  The ranges that it had not
// finished handing out stay without a cut (paged_plan has set them so): no unit that begins in them is joined.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <math_constants.h>
#include <stddef.h>

#include <type_traits>

#include "sla_paged_attn.h"
#include "sla_q4.cuh"
#include "sla_tc_ptx.cuh"

namespace sla {

namespace {

using bf16 = __nv_bfloat16;

constexpr int kThreads = 512;
constexpr int kRows = 128;          // of a stream
constexpr int kKeys = 128;          // of a tile
constexpr int kTileShift = 7;
constexpr int kTmemCols = 512;
constexpr uint32_t kColO = 0, kColS = 256;   // + 128 per stream
constexpr int kTurnTiles = 128;      // units of as many tiles are begun at a tile that depends on the time
constexpr int kSegs = 2;            // entries of the ring of segments
constexpr float kRescaleThreshold = 8.f;     // log2 units
// The streams' products are kept at least this many cycles apart.  A stream's tile takes about 3400 cycles of which 1000 are products and 1200
// exponentials; where both streams come to the same pipe at the same time it takes 4000, and nothing moves them apart again.  (Found at D 128; at
// D 64, whose products take half, 700 to 1700 were tried and none was better.)
// Over a cache in four bits the making of K and V moves the streams too, and less is better (D 128, 8192 tokens that end at 65536, 1999 at
// 30011 and 512 at 65536: 8.77 ms, 1097 and 629 us with 1300; 8.81, 1075 and 614 with 1100; 8.85, 1067 and 611 with 1000; 8.98, 1060 and 618 with
// 900.  D 64, one prompt of 8192 and four of about 2000: 544 and 185 us with 1300; 510 and 180 with 900; 508 and 179 with 700; 509 and 179 with 500).
template <int D, bool kQ4> constexpr uint32_t kApart = !kQ4 ? 1300 : D == 128 ? 1100 : 700;
constexpr uint32_t kPolyPairs = 0x10;        // of every eight pairs of columns, those whose exponentials go to the FMA pipe
// Tiles whose products a stream adds up in TMEM before O is moved to a sum in memory: the tensor cores cut what does not fit into 24 bits, always
// towards zero, so that values of one sign come out too small by about 2^-24 for every 16 keys.  Over 2^20, 2^22 and 2^24 keys of like weight
// that was 0.6, 2.6 and 5 % where a range went on so long; it is 0.03 % after 65536 keys, below the rounding of the result to bf16.  Only calls
// whose tables and windows reach further take the kernel that does so (kLong): its loop costs 1 to 3 % (1 to 600 tokens of 16 sequences 61.9 us
// instead of 60.2, 1999 at 30011 988 instead of 980, 2400 at 2^20 nothing that can be told from noise).
constexpr int kFoldTiles = 512;
constexpr int kRegsRow = 184, kRegsRest = 72;
static_assert(2 * kRegsRow + 2 * kRegsRest <= 4 * 128, "more registers than the block is launched with");

template <int D, bool kQ4> struct Layout {
    static constexpr int kHalves = D / 64;                  // 64-column halves of a tile, 128 rows x 128 B each
    static constexpr int kTileBytes = kKeys * D * 2, kHalfBytes = kKeys * 128;
    static constexpr int kStages = D == 128 ? (kQ4 ? 4 : 5) : 10;
    // four bits: codes and scales of a tile of K or V, as its pages have them
    static constexpr int kSlots = D == 128 ? 3 : 6, kSlotBytes = kQ4 ? kKeys * (D / 2 + D / 16) : 0;
    static constexpr int kOffQ = 0, kOffKV = 2 * kTileBytes, kOffCodes = kOffKV + kStages * kTileBytes, kOffMeta = kOffCodes + kSlots * kSlotBytes;
    static constexpr int kSmem = kOffMeta + 3072;
    static_assert(kStages >= 4, "the waits for a stream's tile before look up to four stages back");
};

// What a segment is to the warps of the CTA.
struct Seg {
    int lo, hi, n, q;                 // tiles; tokens and new tokens of the sequence
    int lo_x[2], hi_x[2];             // tiles that the streams take theirs from: at hi_x a stream goes on at lo_x
    int t0, t1, row0, head;
    int part, slot, valid;
    int both;                         // both streams have the unit's rows, of at most one stream, and every second tile each
    int begin;                        // the tile to begin with: at hi the order goes on at lo
    int begin_x[2], own[2];           // the same of the streams, and how many tiles they take
    int pad[3];
    // the tile behind j; its place in the order; whether stream x takes the i-th tile, j
    __device__ __forceinline__ int next(int j) const { return j + 1 < hi ? j + 1 : lo; }
    __device__ __forceinline__ int place(int j) const { return j >= begin ? j - begin : j - begin + hi - lo; }
    __device__ __forceinline__ bool has(int x, int i, int j) const { return both ? (i & 1) == x : j >= lo_x[x] && j < hi_x[x]; }
};
static_assert(sizeof(Seg) == 96, "six 16-byte words");

struct Meta {
    unsigned long long q_full[2], q_empty[2], kv_full[10], kv_empty[2][10], s_full[2], p_ready[2][2], l_full[2], o_full[2], o_empty[2],
        seg_full[kSegs], seg_empty[kSegs], checked[2], code_full[6], code_empty[6];
    uint32_t tmem_base;
    int abort_flag;
    uint32_t s_time[2];               // clock at the stream's last S
    // [stream][segment & 7]: the segment (counted from 1) if values that are not finite were cleared in it.  Whoever finds one says so
    // to both streams before it clears it; the ring of ten stages at most (a tile of K and of V each) keeps the streams less than eight segments with tiles apart.
    int odd[2][8];
    alignas(16) Seg seg[kSegs];
    float2 stats[2][kRows];           // {1 / sum, log2-sum-exp} of the segment's rows
};
static_assert(sizeof(Meta) <= 3072, "meta block too large");

struct TileParams {
    PagedCall a;
    Plan plan;
    Parts parts;
    const bf16 *q;
    bf16 *out;
    float *lse;
    float *fold;                      // [CTAs][8 warps] sums of O, for segments of more than kFoldTiles tiles (kLong)
    int TS;                           // tokens of a stream
    int t_inner;                      // row i is token i % TS, head i / TS (else token i / G, head i % G), as Q's strides nest
    int slot_t, slot_h, slot_p;       // (token, head, page) among the tensor-map coordinates 1..3 of K and V
    int box_rows;                     // keys of a box: the smaller of a page and a tile
    int out32;                        // every row of the output starts at a multiple of 32 bytes
};

__device__ __forceinline__ float max3(float a, float b, float c) {   // NaN where one of them is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ unsigned long long pack2(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(unsigned long long r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ unsigned long long ffma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long fadd2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^x of two arguments at most 128, on the FMA pipe: 2^n p(r) with n the nearest whole number, |r| <= 1/2, and p the polynomial
// 1 + r (c1 + ..) of degree 4 with the smallest relative error (2.8e-6, fitted on Chebyshev nodes).  Arguments below -127, -inf among
// them, give 0 exactly: n = -127, r = 0, and the exponent field of p(0) = 1 less 127 is that of zero.
__device__ __forceinline__ void ex2_poly(unsigned long long x, float &p0, float &p1) {
    float x0, x1, t0, t1;
    unpack2(x, x0, x1);
    x = pack2(fmaxf(x0, -127.f), fmaxf(x1, -127.f));
    const unsigned long long round = pack2(12582912.f, 12582912.f);   // 1.5 2^23: the sum's low bits are n
    const unsigned long long t = fadd2(x, round), n = fadd2(t, pack2(-12582912.f, -12582912.f)), r = ffma2(n, pack2(-1.f, -1.f), x);
    unsigned long long p = ffma2(r, pack2(0.00958285294f, 0.00958285294f), pack2(0.0559064262f, 0.0559064262f));
    p = ffma2(r, p, pack2(0.240240991f, 0.240240991f));
    p = ffma2(r, p, pack2(0.693124175f, 0.693124175f));
    p = ffma2(r, p, pack2(1.f, 1.f));
    unpack2(p, p0, p1);
    unpack2(t, t0, t1);
    p0 = __int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23));
    p1 = __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23));
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    uint32_t y;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ uint64_t desc_advance(uint64_t desc, uint32_t bytes) {   // the address field, units of 16 bytes
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(desc));
    lo += bytes >> 4;
    asm("mov.b64 %0, {%1, %2};" : "=l"(desc) : "r"(lo), "r"(hi));
    return desc;
}

// Polls of a wait that lasts as long as a segment: its tiles take some 2 us each (a poll at most 1.4 us), and the plain limit is the time of
// half a million of them, 70 million keys.
__device__ __forceinline__ uint32_t segment_polls(int tiles) { return ptx::kSpinLimit + 16u * (uint32_t)tiles; }

// Of every bf16 of a pair of two: all bits of the half where the exponent is all ones, an infinity or a NaN.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((((w & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xffffu; }

// Clears what is not finite in the row of 128 bytes at v (and in the next half's).
template <int D, bool kQ4>
__device__ __noinline__ void clear_not_finite(uint4 *v) {
#pragma unroll 1
    for (int h = 0; h < D / 64; ++h)
#pragma unroll 1
        for (int c = 0; c < 8; ++c) {
            uint4 &w = v[h * (Layout<D, kQ4>::kHalfBytes / 16) + c];
            w = make_uint4(w.x & ~not_finite(w.x), w.y & ~not_finite(w.y), w.z & ~not_finite(w.z), w.w & ~not_finite(w.w));
        }
}

// O of a warp's rows and its sum in memory, [D / 4] pieces of 16 bytes a lane and the maximum that they refer to, by a converged warp
// when the products so far are complete.  first: the sum is O; else the sum and O together, by the present maximum.  last: into O, which stays;
// otherwise into memory, and O is zero again.
template <int D>
__device__ __noinline__ void fold_rows(float *fold, uint32_t o_addr, float m, bool first, bool last) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;   // (rows of stream warp / 4)
    float4 *sum = reinterpret_cast<float4 *>(fold + ((long long)blockIdx.x * 8 + warp) * 32 * (D + 4)) + lane;
    float4 *m_at = sum + 32 * (D / 4);
    float f = 0.f;
    if (!first) {
        const float m_sum = m_at->x;
        f = m_sum == m ? 1.f : ex2_approx(m_sum - m);
    }
#pragma unroll 1
    for (int c = 0; c < D; c += 16) {
        uint32_t o[16];
        float4 w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = first ? make_float4(0.f, 0.f, 0.f, 0.f) : sum[32 * (c / 4 + u)];
        ptx::tmem_ld16(o_addr + c, o);
        ptx::tmem_wait_ld();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            w[u].x = fmaf(w[u].x, f, __uint_as_float(o[4 * u])); w[u].y = fmaf(w[u].y, f, __uint_as_float(o[4 * u + 1]));
            w[u].z = fmaf(w[u].z, f, __uint_as_float(o[4 * u + 2])); w[u].w = fmaf(w[u].w, f, __uint_as_float(o[4 * u + 3]));
            if (!last) sum[32 * (c / 4 + u)] = w[u];
            o[4 * u] = last ? __float_as_uint(w[u].x) : 0u; o[4 * u + 1] = last ? __float_as_uint(w[u].y) : 0u;
            o[4 * u + 2] = last ? __float_as_uint(w[u].z) : 0u; o[4 * u + 3] = last ? __float_as_uint(w[u].w) : 0u;
        }
        ptx::tmem_st16(o_addr + c, o);
    }
    if (!last) m_at->x = m;
    ptx::tmem_wait_st();
    ptx::tc_fence_before();
}

// Adds the values that the row warps have cleared to the rows of O that see them: those that are not finite, of the keys of stream x
// that not every row of the unit sees.  Whatever a row's sums and maxima are, such a value makes the result infinite or NaN, so that
// its weight counts only as positive or (a logit of -inf) zero.  A converged warp with a row of O a lane; a lane looks at one of 32
// keys.  The keys lie at the two ends of the mask, at most the unit's tokens and a tile at each, however long the segment is.
// (The row's address and bounds are worked out again in here, off the way of the segments that have no such value: 1 to 600 tokens of
// 16 sequences take 60.5 us so, 61.2 with them as arguments.)
template <int D, bool kQ4>
__device__ __noinline__ void add_not_finite(const TileParams &p, const Seg &s, int x, uint32_t tmem) {
    const int lane = threadIdx.x & 31, row = threadIdx.x & 127, TS = p.TS, G = p.a.G, end = min(s.hi * kKeys, s.n);
    const uint32_t o_addr = tmem + (static_cast<uint32_t>(row & 96) << 16) + kColO + x * 128;
    // the row, as the row warps have it
    const int t = p.t_inner ? row % TS : row / G, g = p.t_inner ? row / TS : row % G, tok = s.t0 + (s.both ? 0 : x * TS) + t;
    const int last = t < TS && g < G && tok < s.t1 ? s.n - s.q + tok : -1, first = p.a.window > 0 ? max(minus(last, p.a.window - 1), 0) : 0;
    const int all_hi = s.n - s.q + s.t0, all_lo = p.a.window > 0 ? minus(s.n - s.q + s.t1, p.a.window) : 0;   // keys that every row sees
    const bf16 *q = p.q + (s.row0 + tok) * p.a.q_st + (long long)(s.head * G + g) * p.a.q_sh;
    const int *table = p.a.c.table + (long long)max(s.slot, 0) * p.a.c.width;
    auto at = [&](int j) {   // of its row; in four bits of its plane
        return valid_page(p.a.c, __ldg(table + (j >> p.a.c.shift))) * p.a.c.s_page + s.head * p.a.c.s_h + (kQ4 ? 0 : (long long)(j & (p.a.c.P - 1)) * p.a.c.s_t);
    };
    // eight values from dimension d on of the key j, whose row or plane lies at `off`
    auto k_piece = [&](long long off, int j, int d, float (&f)[8]) {
        if constexpr (kQ4) q4::load_values<false>(p.a.c.k + off, p.a.c.P, D, j & (p.a.c.P - 1), d / 8, f);
        else Vec16<bf16>::load(reinterpret_cast<const bf16 *>(p.a.c.k) + off + d, f);
    };
    auto v_piece = [&](long long off, int j, int d, float (&f)[8]) {
        if constexpr (kQ4) q4::load_values<true>(p.a.c.v + off, p.a.c.P, D, j & (p.a.c.P - 1), d / 8, f);
        else Vec16<bf16>::load(reinterpret_cast<const bf16 *>(p.a.c.v) + off + d, f);
    };
#pragma unroll 1
    for (int j0 = s.lo * kKeys; j0 < end; j0 += 32) {
        if (j0 >= all_lo && j0 + 31 <= all_hi) {   // every row sees these 32 keys, and all up to all_hi: the product has them
            j0 += (all_hi + 1 - j0) / 32 * 32 - 32;
            continue;
        }
        const int j = j0 + lane;
        uint32_t bad = 0;
        if (j < end && (j < all_lo || j > all_hi) && (!s.both || (s.place(j / kKeys) & 1) == x)) {
            if constexpr (kQ4) {
                for (int d = 0; d < D; d += 32) bad |= q4::is_nan(q4::scale_of(p.a.c.v + at(j), p.a.c.P, D, j & (p.a.c.P - 1), d));
            } else {
                const uint4 *v = reinterpret_cast<const uint4 *>(reinterpret_cast<const bf16 *>(p.a.c.v) + at(j));
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 w = __ldg(v + c);
                    bad |= not_finite(w.x) | not_finite(w.y) | not_finite(w.z) | not_finite(w.w);
                }
            }
        }
#pragma unroll 1
        for (unsigned left = __ballot_sync(0xffffffffu, bad != 0); left; left &= left - 1) {
            const int key = j0 + __ffs(left) - 1;
            const long long off = at(key);
            const bool sees = key >= first && key <= last;
            float weight = 1.f;
            if (sees) {
                float dot = 0.f;
#pragma unroll 2
                for (int d = 0; d < D; d += 8) {
                    float a[8], b[8];
                    Vec16<bf16>::load(q + d, a);
                    k_piece(off, key, d, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = fmaf(a[e], b[e], dot);
                }
                if (dot == -CUDART_INF_F) weight = 0.f;   // (a NaN, or +inf, is in the row's sum)
            }
            __syncwarp();
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
                float f[2][8];
                v_piece(off, key, c, f[0]);
                v_piece(off, key, c + 8, f[1]);
                uint32_t o[16];
                ptx::tmem_ld16(o_addr + c, o);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float u = f[e >> 3][e & 7];
                    if (sees && !(fabsf(u) < CUDART_INF_F)) o[e] = __float_as_uint(fmaf(weight, u, __uint_as_float(o[e])));
                }
                ptx::tmem_st16(o_addr + c, o);
                ptx::tmem_wait_st();
            }
        }
    }
    ptx::tc_fence_before();
}

// A cache in four bits: bulk copies bring a tile's codes and scales to shared memory, page after page; the warps that write results make K and V of them
// in the ring.  A warp has 32 rows of a tile; a lane takes 16 bytes of codes of kItems of them, neighbouring lanes a row's pieces.  The
// rows of eight neighbouring lanes are such that both their loads and, through the swizzle of the tiles, their 16-byte stores meet all banks.
template <int D> struct Codes {
    static constexpr int kItems = D / 32, kLanes = D / 32, kRows = 32 / kLanes, kHalf = kItems / 2;   // of a lane; lanes of a row; rows of an item; items of 16 rows
    uint32_t codes[2], scales[2];   // where the lane's first row of either half of its warp's 32 has them, from the slot's start
    uint32_t to;                    // where its first piece goes, from the tile's start
    int row0;

    __device__ __forceinline__ Codes(int page, int warp) {   // (warp: of the four)
        const int lane = threadIdx.x & 31, idx = lane / kLanes, chunk = min(page, kKeys), bytes = q4::plane_bytes(chunk, D);
        row0 = D == 128 ? 5 * (idx & 1) ^ (idx & 2) ^ (idx >> 2 & 1) : 5 * (idx & 1) ^ 3 * (idx & 2) ^ (idx >> 2 & 1) ^ (idx & 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 32 * warp + 16 * h + row0, t = r & (chunk - 1);
            codes[h] = r / chunk * bytes + q4::codes_at(D, t) + lane % kLanes * 16;
            scales[h] = r / chunk * bytes + q4::scales_at(chunk, D, t);
        }
        to = (32 * warp + row0) * 128 + ((D == 128 ? lane % 4 : 2 * (lane % 2)) ^ (row0 & 7)) * 16;
    }
    uint32_t w[kItems][4], sc[kItems][D / 64];

    // A tile's codes and scales out of the slot at `slot`.  left: rows of the warp that count; those behind them may be anything and become zero.
    __device__ __forceinline__ void load(uint32_t slot, int left) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int h = i / kHalf, e = i % kHalf * kRows;
            q4::load_shared(slot + codes[h] + e * (D / 2), w[i]);
            q4::load_shared(slot + scales[h] + e * (D / 16), sc[i]);
        }
        if (left < 32) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
#pragma unroll
                for (int x = 0; x < D / 64; ++x) sc[i][x] = i * kRows + row0 < left ? sc[i][x] : 0;
        }
    }
    // K or V of it to the tile at `tile`.
    template <bool kValues> __device__ __forceinline__ void store(uint32_t tile) const {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                // the piece of eight dimensions: group, and which of the group's four
                const int g = D == 128 ? x : x & 1, up = D == 128 ? 0 : x >> 1;
                const uint32_t sel = x & 1 ? 0x7632u : 0x5410u;
                const uint32_t word = !kValues ? w[i][x] : D == 128 ? __byte_perm(w[i][x >> 1], w[i][2 + (x >> 1)], sel) : __byte_perm(w[i][2 * (x >> 1)], w[i][2 * (x >> 1) + 1], sel);
                uint32_t v[4];
                q4::small_values(word, __byte_perm(sc[i][g >> 1], 0, g & 1 ? 0x3232 : 0x1010), v);
                ptx::st_shared_v4(((tile + to) ^ ((g & 1) * 64 + up * 16)) + (g >> 1) * Layout<D, true>::kHalfBytes + i * kRows * 128, v);
            }
    }
};

template <int D, bool kLong, bool kQ4>
__global__ void __launch_bounds__(kThreads, 1)
paged_tiles(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
            const __grid_constant__ TileParams p) {
    using L = Layout<D, kQ4>;
    constexpr int kStages = L::kStages, kHalves = L::kHalves;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = ptx::smem_u32(smem);
    Meta *meta = reinterpret_cast<Meta *>(smem + L::kOffMeta);
    volatile int *abort_flag = &meta->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (base & 1023u) {   // the swizzled tiles need a 1024-byte aligned window: refuse rather than corrupt
        if (tid == 0) atomicOr(p.a.c.status, kStatusTimeout);
        return;
    }
    const uint32_t mbase = base + L::kOffMeta;
    const uint32_t bar_q_full = mbase + offsetof(Meta, q_full), bar_q_empty = mbase + offsetof(Meta, q_empty);
    const uint32_t bar_kv_full = mbase + offsetof(Meta, kv_full), bar_kv_empty = mbase + offsetof(Meta, kv_empty);
    const uint32_t bar_s_full = mbase + offsetof(Meta, s_full), bar_p_ready = mbase + offsetof(Meta, p_ready);
    const uint32_t bar_l_full = mbase + offsetof(Meta, l_full), bar_o_full = mbase + offsetof(Meta, o_full);
    const uint32_t bar_o_empty = mbase + offsetof(Meta, o_empty), bar_checked = mbase + offsetof(Meta, checked);
    const uint32_t bar_code_full = mbase + offsetof(Meta, code_full), bar_code_empty = mbase + offsetof(Meta, code_empty);
    const uint32_t bar_seg_full = mbase + offsetof(Meta, seg_full), bar_seg_empty = mbase + offsetof(Meta, seg_empty);

    if (tid == 0) {
#pragma unroll 1
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(bar_q_full + 8 * x, 1);
            ptx::mbar_init(bar_q_empty + 8 * x, 1);
            ptx::mbar_init(bar_s_full + 8 * x, 1);
            ptx::mbar_init(bar_p_ready + 16 * x, 4);       // a row warp each
            ptx::mbar_init(bar_p_ready + 16 * x + 8, 4);
            ptx::mbar_init(bar_l_full + 8 * x, 4);
            ptx::mbar_init(bar_checked + 8 * x, 4);
            ptx::mbar_init(bar_o_full + 8 * x, 1);
            ptx::mbar_init(bar_o_empty + 8 * x, 4);        // an epilogue warp each
        }
#pragma unroll 1
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(bar_kv_full + 8 * s, kQ4 ? 4 : 1);   // four bits: a filling warp each
            ptx::mbar_init(bar_kv_empty + 8 * s, 1);
            ptx::mbar_init(bar_kv_empty + 80 + 8 * s, 1);
        }
#pragma unroll 1
        for (int s = 0; s < kSegs; ++s) {
            ptx::mbar_init(bar_seg_full + 8 * s, 1);
            ptx::mbar_init(bar_seg_empty + 8 * s, 13 + 2 * 32);   // rows, epilogue, K/V: a warp each; the issuers a lane each
        }
        if constexpr (kQ4) {
#pragma unroll 1
            for (int s = 0; s < L::kSlots; ++s) {
                ptx::mbar_init(bar_code_full + 8 * s, 1);
                ptx::mbar_init(bar_code_empty + 8 * s, 4);
            }
        }
        meta->abort_flag = 0;
        meta->s_time[0] = meta->s_time[1] = clock();
        for (int s = 0; s < 8; ++s) meta->odd[0][s] = meta->odd[1][s] = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 12) {
        ptx::tmem_alloc(mbase + offsetof(Meta, tmem_base), kTmemCols);
        ptx::tmem_relinquish();
    }
    chain_wait();      // the set-up above runs beside the kernel before this one
    chain_release();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = meta->tmem_base;
    const int G = p.a.G, TS = p.TS;

    // the CTA's k-th segment is there, for a whole warp; the warp has done with it
    auto take_seg = [&](uint32_t k) {
        return ptx::mbar_wait_warp(bar_seg_full + 8 * (k % kSegs), (k / kSegs) & 1u, abort_flag) && meta->seg[k % kSegs].valid != 0;
    };
    auto free_seg = [&](uint32_t k) {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar_seg_empty + 8 * (k % kSegs));
    };

    if (warp >= 12) {
        ptx::setmaxnreg_dec<kRegsRest>();
        if (warp < 14) {
            // ---------------- MMA issuer of stream x: a whole warp, its elected lane issues.  S of the next tile goes right behind
            // the PV of this one, which reads the P that lies over it (the tensor pipe keeps a thread's order).
            const bool leader = ptx::elect_one();
            const int x = warp - 12;
            constexpr uint32_t kIdescS = ptx::idesc_bf16_f32(kRows, kKeys, false, false);   // both K-major
            constexpr uint32_t kIdescO = ptx::idesc_bf16_f32(kRows, D, false, true);        // V is N-major
            const uint32_t s_col = tmem + kColS + x * 128, o_col = tmem + kColO + x * 128;
            const uint64_t dq = ptx::smem_desc_sw128(base + L::kOffQ + x * L::kTileBytes, 16, 1024);
            const uint64_t dk0 = ptx::smem_desc_sw128(base + L::kOffKV, 16, 1024);
            const uint64_t dv0 = ptx::smem_desc_sw128(base + L::kOffKV, L::kHalfBytes, 1024);
            uint32_t i = 0, nt = 0, ns = 0;   // ring position; tiles and segments of the stream so far
            bool ok = true;
#pragma unroll 1
            for (uint32_t k = 0; ok; ++k) {
                if (!ptx::mbar_wait(bar_seg_full + 8 * (k % kSegs), (k / kSegs) & 1u, abort_flag)) break;
                const Seg &s = meta->seg[k % kSegs];
                if (!s.valid) break;
                const int tiles = s.hi - s.lo, own = s.own[x];
                int done = 0, j = s.begin;   // done: of the stream's own
                bool k_there = false;   // K of the tile has been waited for
#pragma unroll 1
                for (int t = 0; t < tiles; ++t) {
                    const bool on = s.has(x, t, j);
                    j = s.next(j);
                    uint32_t st = i % kStages;
                    if (!k_there && !(ok = ptx::mbar_wait(bar_kv_full + 8 * st, (i / kStages) & 1u, abort_flag))) break;
                    k_there = false;
                    if (on) {
                        if (done == 0 && !(ok = ptx::mbar_wait(bar_q_full + 8 * x, ns & 1u, abort_flag))) break;
                        ptx::tc_fence_after();
                        {
                            volatile uint32_t *s_time = meta->s_time;
                            const uint32_t other = s_time[1 - x];
                            uint32_t now;
                            do now = clock(); while (now - other < kApart<D, kQ4>);
                            s_time[x] = now;
                        }
                        const uint64_t dk = desc_advance(dk0, st * L::kTileBytes);
                        if (leader) {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t off = (kk >> 2) * L::kHalfBytes + (kk & 3) * 32;
                                ptx::mma_ss(s_col, desc_advance(dq, off), desc_advance(dk, off), kIdescS, kk > 0);
                            }
                            ptx::mma_commit(bar_s_full + 8 * x);
                            ptx::mma_commit(bar_kv_empty + 80 * x + 8 * st);
                            if (done == own - 1) ptx::mma_commit(bar_q_empty + 8 * x);
                        }
                    } else if (leader) {
                        ptx::mbar_arrive(bar_kv_empty + 80 * x + 8 * st);
                    }
                    ++i;
                    st = i % kStages;
                    if (!(ok = ptx::mbar_wait(bar_kv_full + 8 * st, (i / kStages) & 1u, abort_flag))) break;
                    if (on) {
                        // the first PV of a segment overwrites O: the results of the segment before have been read
                        if (done == 0 && ns > 0 && !(ok = ptx::mbar_wait(bar_o_empty + 8 * x, (ns - 1u) & 1u, abort_flag))) break;
                        if (t + 1 < tiles) {   // off the way from P to the next S
                            k_there = true;
                            if (!(ok = ptx::mbar_wait(bar_kv_full + 8 * ((i + 1) % kStages), ((i + 1) / kStages) & 1u, abort_flag))) break;
                        }
                        const uint64_t dv = desc_advance(dv0, st * L::kTileBytes);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!(ok = ptx::mbar_wait(bar_p_ready + 16 * x + 8 * half, nt & 1u, abort_flag))) break;
                            ptx::tc_fence_after();
                            if (leader) {
#pragma unroll
                                for (int kk = 4 * half; kk < 4 * half + 4; ++kk)
                                    ptx::mma_ts(o_col, s_col + kk * 8, desc_advance(dv, kk * 2048), kIdescO, (done > 0 || kk > 0) ? 1u : 0u);
                            }
                        }
                        if (!ok) break;
                        if (leader) {
                            ptx::mma_commit(bar_kv_empty + 80 * x + 8 * st);
                            if (done == own - 1) ptx::mma_commit(bar_o_full + 8 * x);
                        }
                        ++nt;
                        ++done;
                    } else if (leader) {
                        ptx::mbar_arrive(bar_kv_empty + 80 * x + 8 * st);
                    }
                    ++i;
                }
                ns += own > 0;
                ptx::mbar_arrive(bar_seg_empty + 8 * (k % kSegs));
            }
        } else if (warp == 14) {
            if constexpr (kQ4) {
            // ---------------- codes and scales of K and V: a lane per page that the tile has
            const Pages &c = p.a.c;
            const int chunk = min(c.P, kKeys), bytes = q4::plane_bytes(chunk, D), chunks = kKeys / chunk;
            uint32_t i = 0;
            bool ok = true;
#pragma unroll 1
            for (uint32_t k = 0; ok && take_seg(k); free_seg(k++)) {
                const Seg &s = meta->seg[k % kSegs];
                const int tiles = s.hi - s.lo, n = s.n;
                const int *table = c.table + (long long)max(s.slot, 0) * c.width;
                auto page_of = [&](int j) {   // -1: no page
                    const int key = j * kKeys + lane * chunk;
                    return lane < chunks && key < n ? valid_page(c, __ldg(table + (key >> c.shift))) : -1;
                };
                int next = tiles > 0 ? page_of(s.begin) : -1, j_next = s.begin;
#pragma unroll 1
                for (int t = 0; t < tiles && ok; ++t) {
                    const int page = next, t0 = j_next * kKeys & (c.P - 1);   // (pages of 256 tokens: the half)
                    j_next = s.next(j_next);
                    next = page_of(j_next);
                    const uint32_t all = __popc(__ballot_sync(0xffffffffu, page >= 0)) * bytes;
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv, ++i) {
                        const uint32_t slot = i % L::kSlots, full = bar_code_full + 8 * slot;
                        if (!(ok = ptx::mbar_wait_warp(bar_code_empty + 8 * slot, ((i / L::kSlots) & 1u) ^ 1u, abort_flag))) break;
                        if (lane == 0) ptx::mbar_arrive_expect_tx(full, all);
                        __syncwarp();
                        if (page >= 0) {
                            const char *plane = (kv ? c.v : c.k) + page * c.s_page + s.head * c.s_h;
                            const uint32_t dst = base + L::kOffCodes + slot * L::kSlotBytes + lane * bytes;
                            if (chunk == c.P) {
                                ptx::bulk_load(dst, plane, bytes, full);
                            } else {
                                ptx::bulk_load(dst, plane + q4::codes_at(D, t0), chunk * (D / 2), full);
                                ptx::bulk_load(dst + chunk * (D / 2), plane + q4::scales_at(c.P, D, t0), chunk * (D / 16), full);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            } else {
            // ---------------- K and V: a lane per box, as many as the tile has pages with tokens
            ptx::prefetch_tensormap(&tm_k);
            ptx::prefetch_tensormap(&tm_v);
            const bool leader = ptx::elect_one();
            const int boxes = kKeys / p.box_rows, shift = p.a.c.shift;
            const uint32_t box_bytes = p.box_rows * 128;
            uint32_t i = 0;
            bool ok = true;
#pragma unroll 1
            for (uint32_t k = 0; ok && take_seg(k); free_seg(k++)) {
                const Seg &s = meta->seg[k % kSegs];
                const int tiles = s.hi - s.lo, n = s.n, head = s.head;
                const int *table = p.a.c.table + (long long)max(s.slot, 0) * p.a.c.width;
                auto key_of = [&](int j) { return j * kKeys + lane * p.box_rows; };
                auto page_of = [&](int j) {   // -1: no box
                    const int key = key_of(j);
                    return lane < boxes && key < n ? valid_page(p.a.c, __ldg(table + (key >> shift))) : -1;
                };
                int next = tiles > 0 ? page_of(s.begin) : -1, j_next = s.begin;
#pragma unroll 1
                for (int t = 0; t < tiles && ok; ++t) {
                    const int page = next, j = j_next;
                    j_next = s.next(j);
                    next = page_of(j_next);
                    int c[4];
                    c[1 + p.slot_t] = key_of(j) & (p.a.c.P - 1);
                    c[1 + p.slot_h] = head;
                    c[1 + p.slot_p] = page;
                    const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, page >= 0)) * box_bytes * kHalves;
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv, ++i) {
                        const uint32_t st = i % kStages, ph = ((i / kStages) & 1u) ^ 1u, full = bar_kv_full + 8 * st;
                        ok = ptx::mbar_wait_warp(bar_kv_empty + 8 * st, ph, abort_flag) && ptx::mbar_wait_warp(bar_kv_empty + 80 + 8 * st, ph, abort_flag);
                        if (!ok) break;
                        if (leader) ptx::mbar_arrive_expect_tx(full, bytes);
                        __syncwarp();
                        if (page >= 0) {
                            const uint32_t dst = base + L::kOffKV + st * L::kTileBytes + lane * box_bytes;
                            const CUtensorMap *tm = kv ? &tm_v : &tm_k;
                            ptx::tma_load_4d(dst, tm, full, 0, c[1], c[2], c[3]);
                            if (kHalves == 2) ptx::tma_load_4d(dst + L::kHalfBytes, tm, full, 64, c[1], c[2], c[3]);
                        }
                        __syncwarp();
                    }
                }
            }
            }
        } else {
            // ---------------- the CTA's ranges, segment after segment, and their Q
            ptx::prefetch_tensormap(&tm_q);
            const bool leader = ptx::elect_one();
            uint32_t k = 0, nq[2] = {0, 0};
            int at = 0;   // tiles so far
            uint32_t polls = ptx::kSpinLimit;   // of a wait for the segments before
            bool ok = !p.a.expire;
            if (!ok) *abort_flag = 1;
            auto put = [&](const Seg &s) {
                ok = ptx::mbar_wait_warp(bar_seg_empty + 8 * (k % kSegs), ((k / kSegs) & 1u) ^ 1u, abort_flag, polls);
                if (ok && leader) {
                    meta->seg[k % kSegs] = s;
                    ptx::mbar_arrive(bar_seg_full + 8 * (k % kSegs));
                }
                __syncwarp();
                ++k;
            };
            Seg s;
            for (int range = blockIdx.x; ok; range += gridDim.x) {
                Cursor cur;
                Segment g;
                int last_range;
                Cut cut = {0, 0, 0, -1};
                if (!cur.open(p.plan, range, g, last_range)) break;
                do {
                    if (last_range >= 0) cut = {g.row0 + g.t0, g.t1 - g.t0, g.head, last_range};
                    s.lo = g.lo; s.hi = g.hi; s.n = g.n; s.q = g.q;
                    s.t0 = g.t0; s.t1 = g.t1; s.row0 = g.row0; s.head = g.head;
                    s.part = g.part; s.slot = g.slot; s.valid = 1;
                    s.both = g.t1 - g.t0 <= TS;
                    const int tiles = g.hi - g.lo;
                    // CTAs that read the same keys read them at about the same time, so that they find them in L2: after t tiles each is at
                    // the tile t of its unit, or, where a unit is shared by several, at one that is t modulo their share.  512 tokens at
                    // 65536 (64 units over 148 CTAs): 540 us instead of 620, which read 1.86 GB out of DRAM for 0.27 GB of keys; 1999 at
                    // 30011: 920 instead of 985.  Short units keep their order: their keys stay in L2 in any order, and four prompts of
                    // 2048 tokens (D 64) took 162 us instead of 154 with turns.
                    int turn = 0;
                    if (g.all >= kTurnTiles) {
                        const int period = max(1, min(g.all, (int)min(cur.ranges.each, (long long)0x3fffffff)));
                        turn = (at - g.lo) % period;
                        turn += turn < 0 ? period : 0;
                    }
                    s.begin = turn < tiles ? g.lo + turn : g.lo;
                    at = (at + tiles) & 0x3fffffff;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int a0 = min(g.t0 + x * TS, g.t1), a1 = min(a0 + TS, g.t1);
                        int lo = g.lo, hi = g.hi;
                        if (!s.both) unit_tiles(g.n, g.q, a0, a1, p.a.window, kTileShift, lo, hi);
                        lo = max(lo, g.lo);
                        hi = min(hi, g.hi);
                        const int at_x = s.begin + (s.both ? x : 0);
                        s.lo_x[x] = lo;
                        s.hi_x[x] = hi;
                        s.own[x] = s.both ? (tiles + 1 - x) >> 1 : max(hi - lo, 0);
                        s.begin_x[x] = s.both ? (at_x < hi ? at_x : at_x - tiles) : at_x >= lo && at_x < hi ? at_x : lo;
                    }
                    put(s);
#pragma unroll 1
                    for (int x = 0; x < 2 && ok; ++x) {
                        if (s.own[x] == 0) continue;
                        ok = ptx::mbar_wait_warp(bar_q_empty + 8 * x, (nq[x] & 1u) ^ 1u, abort_flag, polls);
                        ++nq[x];
                        if (!ok) break;
                        if (leader) {
                            const uint32_t full = bar_q_full + 8 * x, dst = base + L::kOffQ + x * L::kTileBytes;
                            ptx::mbar_arrive_expect_tx(full, TS * G * 128 * kHalves);
                            const int tok = g.row0 + g.t0 + (s.both ? 0 : x * TS), c1 = p.t_inner ? tok : g.head * G, c2 = p.t_inner ? g.head * G : tok;
#pragma unroll
                            for (int h = 0; h < kHalves; ++h) ptx::tma_load_4d(dst + h * L::kHalfBytes, &tm_q, full, 64 * h, c1, c2, 0);
                        }
                        __syncwarp();
                    }
                    polls = max(polls, segment_polls(tiles));
                } while (ok && cur.next(p.a, p.plan, Shape{2 * TS, kTileShift, TS}, g, last_range));
                if (leader && ok) p.parts.cut[range] = cut;
            }
            s = Seg{};
            if (ok) put(s);
        }
    } else if (warp >= 8) {
        // ---------------- results: a thread a row
        ptx::setmaxnreg_dec<kRegsRest>();
        const int row = tid & 127;
        const int t = p.t_inner ? row % TS : row / G, g = p.t_inner ? row / TS : row % G, canon = t * G + g;
        const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        uint32_t ns[2] = {0, 0};
        bool ok = true;
        auto results = [&](uint32_t k) {
            const Seg &s = meta->seg[k % kSegs];
#pragma unroll 1
            for (int x = 0; x < 2 && ok; ++x) {
                const int tok = s.t0 + x * TS + t;
                const bool has = s.own[x] > 0, second = s.both && s.own[1] > 0;
                const bool write = t < TS && g < G && tok < s.t1;
                const int h = s.head * G + g;
                const long long r = s.row0 + tok;
                bf16 *dst = p.out + r * p.a.q_st + (long long)h * p.a.q_sh;
                float2 stat = make_float2(0.f, -CUDART_INF_F);   // factor of O, log2-sum-exp
                float f1 = 0.f;                                  // factor of the other stream's O
                if (has) {
                    ok = ptx::mbar_wait_warp(bar_l_full + 8 * x, ns[x] & 1u, abort_flag, segment_polls(s.hi - s.lo)) &&
                         ptx::mbar_wait_warp(bar_o_full + 8 * x, ns[x] & 1u, abort_flag);
                    if (!ok) break;
                    ++ns[x];
                    ptx::tc_fence_after();
                    stat = meta->stats[x][row];
                }
                if (second) {   // two sums over every second tile each
                    ok = ptx::mbar_wait_warp(bar_l_full + 8, ns[1] & 1u, abort_flag) && ptx::mbar_wait_warp(bar_o_full + 8, ns[1] & 1u, abort_flag);
                    if (!ok) break;
                    ++ns[1];
                    ptx::tc_fence_after();
                    const float2 other = meta->stats[1][row];
                    const float top = fmaxf(stat.y, other.y), ref = top == -CUDART_INF_F ? 0.f : top;
                    const float w0 = ex2_approx(stat.y - ref), w1 = ex2_approx(other.y - ref), sum = w0 + w1;
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    stat.x *= w0 * inv;
                    f1 = other.x * w1 * inv;
                    stat.y = sum == 0.f ? -CUDART_INF_F : ref + log2f(sum);
                }
                const bool none = stat.y == -CUDART_INF_F;
                if (has) {
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 16) {   // (32 columns at a time spill)
                        uint32_t o[16];
                        ptx::tmem_ld16(lane_addr + kColO + x * 128 + c0, o);
                        if (second) {
                            uint32_t o1[16];
                            ptx::tmem_ld16(lane_addr + kColO + 128 + c0, o1);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(fmaf(__uint_as_float(o1[e]), f1, __uint_as_float(o[e]) * stat.x));
                        } else {
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * stat.x);
                        }
                        if (c0 == D - 16) {   // O is in registers: the next segment's first PV may overwrite it
                            ptx::tc_fence_before();
                            __syncwarp();
                            if (lane == 0) {
                                ptx::mbar_arrive(bar_o_empty + 8 * x);
                                if (second) ptx::mbar_arrive(bar_o_empty + 8);
                            }
                        }
                        if (!write) continue;
                        if (s.part < 0) {   // (rows may start at any 16 bytes)
                            uint32_t w[8];
#pragma unroll
                            for (int u = 0; u < 8; ++u) w[u] = none ? 0u : bf16x2(__uint_as_float(o[2 * u]), __uint_as_float(o[2 * u + 1]));
                            if (p.out32) {
                                ptx::st_global_v8(dst + c0, w);
                            } else {
                                *reinterpret_cast<uint4 *>(dst + c0) = make_uint4(w[0], w[1], w[2], w[3]);
                                *reinterpret_cast<uint4 *>(dst + c0 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                            }
                        } else if (!none) {
#pragma unroll
                            for (int e = 0; e < 16; e += 8) {
                                const uint32_t w[8] = {o[e], o[e + 1], o[e + 2], o[e + 3], o[e + 4], o[e + 5], o[e + 6], o[e + 7]};
                                ptx::st_global_v8(p.parts.at(s.part, 256, D, x * kRows + canon, c0 + e), w);
                            }
                        }
                    }
                } else if (write && s.part < 0) {
#pragma unroll 1
                    for (int e = 0; e < D; e += 8) *reinterpret_cast<uint4 *>(dst + e) = make_uint4(0, 0, 0, 0);
                }
                if (write) {
                    if (s.part < 0) p.lse[r * p.a.Hq + h] = stat.y * kLn2;
                    else p.parts.lse2[(long long)s.part * 256 + x * kRows + canon] = stat.y;
                }
                if (s.both) break;
            }
        };
        if constexpr (!kQ4) {
#pragma unroll 1
            for (uint32_t k = 0; ok && take_seg(k); free_seg(k++)) results(k);
        } else {
            Codes<D> codes(p.a.c.P, warp - 8);
            uint32_t i = 0;   // tiles of K and V so far
            auto make = [&](auto values, int left) {
                const uint32_t st = i % kStages, ph = ((i / kStages) & 1u) ^ 1u, slot = i % L::kSlots;
                if (!ptx::mbar_wait_warp(bar_code_full + 8 * slot, (i / L::kSlots) & 1u, abort_flag)) return false;
                codes.load(base + L::kOffCodes + slot * L::kSlotBytes, left);
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_code_empty + 8 * slot);
                if (!ptx::mbar_wait_warp(bar_kv_empty + 8 * st, ph, abort_flag) || !ptx::mbar_wait_warp(bar_kv_empty + 80 + 8 * st, ph, abort_flag)) return false;
                codes.template store<decltype(values)::value>(base + L::kOffKV + st * L::kTileBytes);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_kv_full + 8 * st);
                ++i;
                return true;
            };
            auto make_tiles = [&](uint32_t k, int from, int until) {
                const Seg &s = meta->seg[k % kSegs];
                const int n = s.n, lo = s.lo, hi = s.hi;
                int j = s.begin + from;
                if (j >= hi) j -= hi - lo;
#pragma unroll 1
                for (int t = from; t < until; ++t) {
                    const int left = n - j * kKeys - 32 * (warp - 8);
                    if (!make(std::false_type{}, left) || !make(std::true_type{}, left)) return false;
                    j = j + 1 < hi ? j + 1 : lo;
                }
                return true;
            };
            auto tiles_of = [&](uint32_t k) { return meta->seg[k % kSegs].hi - meta->seg[k % kSegs].lo; };
            // The first two tiles of the next segment are made before the results of this one are written: they wait for nothing but this segment's
            // products.
            uint32_t k = 0;
            int from = 0;
            bool first = true;   // in turn: what is left of segment k; the first tiles of the next k, and the results of the one before
#pragma unroll 1
            for (bool more = take_seg(0); ok && more;) {   // (one call of make_tiles, which is long)
                const int until = first ? tiles_of(k) : min(2, tiles_of(k));
                ok = make_tiles(k, from, until);
                from = until;
                if (first) {
                    more = ok && take_seg(k + 1);
                    if (more) {
                        ++k;
                        from = 0;
                        first = false;
                        continue;
                    }
                    if (ok) results(k);
                    free_seg(k);
                } else {
                    if (ok) results(k - 1);
                    free_seg(k - 1);
                    first = true;
                }
            }
        }
    } else {
        // ---------------- rows of stream x: a thread a row
        ptx::setmaxnreg_inc<kRegsRow>();
        const int x = warp >> 2, row = tid & 127;
        const int t = p.t_inner ? row % TS : row / G, g = p.t_inner ? row / TS : row % G;
        const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t o_addr = lane_addr + kColO + x * 128, s_col = lane_addr + kColS + x * 128;
        const float scale2 = p.a.scale * kLog2e * (kQ4 ? q4::kSmall : 1.f);   // (K and V of codes are 2^-48 of what they are)
        uint32_t nt = 0, ns = 0, tiles = 0;   // tiles and segments of the stream, tiles of the CTA so far
        bool ok = true;
#pragma unroll 1
        for (uint32_t k = 0; ok && take_seg(k); free_seg(k++)) {
            const Seg &s = meta->seg[k % kSegs];
            const int tok = s.t0 + (s.both ? 0 : x * TS) + t;
            const bool valid = t < TS && g < G && tok < s.t1;
            const int last = valid ? s.n - s.q + tok : -1, first = p.a.window > 0 ? max(minus(last, p.a.window - 1), 0) : 0;   // keys seen
            // keys that not every row of the unit sees lie outside [all_lo, all_hi]
            const int all_hi = s.n - s.q + s.t0, all_lo = p.a.window > 0 ? minus(s.n - s.q + s.t1, p.a.window) : 0;
            if (s.own[x] > 0) {
                const int lx = s.lo_x[x], hx = s.hi_x[x], step = s.both ? 2 : 1;
                int j = s.begin_x[x];
                float m_ref = -CUDART_INF_F, l = 0.f;
                bool fresh = true;   // no logit above -inf so far
#pragma unroll 1
                for (int left = s.own[x]; left > 0; --left, ++nt) {
                    const int k0 = j * kKeys;
                    if (kLong && s.own[x] > kFoldTiles && left != s.own[x] && (s.own[x] - left) % kFoldTiles == 0) {   // (the wait as before a rescale, below)
                        const int before = j - step;
                        const uint32_t v = 2 * (tiles + s.place(before < lx ? before + hx - lx : before)) + 1u;
                        if (!(ok = ptx::mbar_wait_warp(bar_kv_empty + 80 * x + 8 * (v % kStages), (v / kStages) & 1u, abort_flag))) break;
                        ptx::tc_fence_after();
                        fold_rows<D>(p.fold, o_addr, fresh ? -CUDART_INF_F : m_ref, s.own[x] - left == kFoldTiles, false);
                    }
                    if (!(ok = ptx::mbar_wait_warp(bar_s_full + 8 * x, nt & 1u, abort_flag))) break;
                    ptx::tc_fence_after();
                    uint32_t sr[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) ptx::tmem_ld32(s_col + c * 32, sr[c]);
                    ptx::tmem_wait_ld();
                    if (k0 < first || k0 + kKeys - 1 > last) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int a = k0 + c * 32;   // bits [first - a, last - a] of the 32 columns
                            const int lo = max(first - a, 0), hi = min(last - a, 31);
                            const uint32_t inside = lo <= hi ? (0xffffffffu >> (31 - (hi - lo))) << lo : 0u;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(inside & (1u << e))) sr[c][e] = 0xff800000u;   // -inf
                        }
                    }
                    float bm;   // (scale > 0)
                    {
                        float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
#pragma unroll
                                for (int u = 0; u < 4; ++u)
                                    mx[u] = max3(mx[u], __uint_as_float(sr[c][e + 2 * u]), __uint_as_float(sr[c][e + 2 * u + 1]));
                        bm = max3(max3(mx[0], mx[1], mx[2]), mx[3], mx[3]) * scale2;
                    }
                    // a logit that is NaN or +inf makes the row NaN: the sum says so, whatever the weights below become
                    if (!(bm < CUDART_INF_F)) {
                        l = CUDART_NAN_F;
                        bm = m_ref;
                    }
                    const bool need = !fresh && bm > m_ref + kRescaleThreshold;
                    if (__any_sync(0xffffffffu, need)) {
                        // the PV of the stream's tile before must have landed before O is touched
                        // (a stream has every tile of the unit but at most one, or every second one, so that the tile before lies at most two
                        // places, four stages, back.  Its stage may hold V of the present tile by now, but no later one: the stream
                        // gives that up when P of the present tile, which this warp still owes, has met it.  So the parity is that of the tile before.)
                        const int before = j - step;
                        const uint32_t v = 2 * (tiles + s.place(before < lx ? before + hx - lx : before)) + 1u;
                        if (!(ok = ptx::mbar_wait_warp(bar_kv_empty + 80 * x + 8 * (v % kStages), (v / kStages) & 1u, abort_flag))) break;
                        ptx::tc_fence_after();
                        const float f = need ? ex2_approx(m_ref - bm) : 1.f;
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            ptx::tmem_ld16(o_addr + c * 16, o);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            ptx::tmem_st16(o_addr + c * 16, o);
                        }
                        if (need) {
                            l *= f;
                            m_ref = bm;
                        }
                    }
                    if (fresh && bm > -CUDART_INF_F) {
                        m_ref = bm;
                        fresh = false;
                    }
                    const float neg_m = fresh ? 0.f : -m_ref;   // a row with no key so far: -inf stays -inf
                    const unsigned long long sc2 = pack2(scale2, scale2), nm2 = pack2(neg_m, neg_m);
                    unsigned long long acc2[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) acc2[u] = pack2(0.f, 0.f);
                    const bool edge = k0 + kKeys - 1 > all_hi || k0 < all_lo;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t pk[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int c = 2 * half + (e >> 4), c2 = (e & 15) * 2;
                            const unsigned long long y = ffma2(pack2(__uint_as_float(sr[c][c2]), __uint_as_float(sr[c][c2 + 1])), sc2, nm2);
                            float p0, p1;
                            if (kPolyPairs >> (e & 7) & 1) {
                                ex2_poly(y, p0, p1);
                            } else {
                                unpack2(y, p0, p1);
                                p0 = ex2_approx(p0);
                                p1 = ex2_approx(p1);
                            }
                            acc2[e & 3] = fadd2(acc2[e & 3], pack2(p0, p1));
                            pk[e] = bf16x2(p0, p1);
                        }
                        ptx::tmem_st32(s_col + half * 32, pk);
                        if (half == 0 && edge) {
                            // this thread's key of the tile: beyond the sequence it is cleared, else looked at
                            const uint32_t v = 2 * (tiles + s.place(j)) + 1u;
                            if (!(ok = ptx::mbar_wait_warp(bar_kv_full + 8 * (v % kStages), (v / kStages) & 1u, abort_flag))) break;
                            const int key = k0 + row;
                            uint4 *vr = reinterpret_cast<uint4 *>(smem + L::kOffKV + (v % kStages) * L::kTileBytes + row * 128);
                            const bool clear = key >= s.n;
                            if (!clear && (key > all_hi || key < all_lo)) {
                                uint32_t bad = 0;
#pragma unroll
                                for (int h = 0; h < kHalves; ++h)
#pragma unroll 4
                                    for (int c = 0; c < 8; ++c) {
                                        const uint4 w = vr[h * (L::kHalfBytes / 16) + (c ^ (row & 7))];
                                        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                                        for (int u = 0; u < 4; ++u) bad |= ((ws[u] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // exponent all ones
                                    }
                                if (bad) {
                                    *(volatile int *)&meta->odd[0][k & 7] = *(volatile int *)&meta->odd[1][k & 7] = (int)k + 1;
                                    __threadfence_block();
                                    clear_not_finite<D, kQ4>(vr);
                                }
                            }
                            if (clear) {
#pragma unroll
                                for (int h = 0; h < kHalves; ++h)
#pragma unroll
                                    for (int c = 0; c < 8; ++c) vr[h * (L::kHalfBytes / 16) + c] = make_uint4(0, 0, 0, 0);
                            }
                            ptx::fence_proxy_async_smem();
                        }
                        ptx::tmem_wait_st();
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(bar_p_ready + 16 * x + 8 * half);
                    }
                    if (!ok) break;
                    float s0, s1, s2, s3;
                    unpack2(fadd2(acc2[0], acc2[1]), s0, s1);
                    unpack2(fadd2(acc2[2], acc2[3]), s2, s3);
                    l += (s0 + s1) + (s2 + s3);
                    j += step;
                    if (j >= hx) j -= hx - lx;
                }
                if (!ok) break;
                // all four warps have looked at their keys
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_checked + 8 * x);
                if (!(ok = ptx::mbar_wait_warp(bar_checked + 8 * x, ns & 1u, abort_flag))) break;
                const bool odd = __any_sync(0xffffffffu, *(volatile int *)&meta->odd[x][k & 7] == (int)k + 1);
                if (odd || (kLong && s.own[x] > kFoldTiles)) {
                    // O is complete, and stays: the next segment's first PV waits for the epilogue, which waits for this warp
                    if (!(ok = ptx::mbar_wait_warp(bar_o_full + 8 * x, ns & 1u, abort_flag))) break;
                    ptx::tc_fence_after();
                    if (kLong && s.own[x] > kFoldTiles) fold_rows<D>(p.fold, o_addr, fresh ? -CUDART_INF_F : m_ref, false, true);
                    if (odd) add_not_finite<D, kQ4>(p, s, x, tmem);
                }
                // the epilogue has read the statistics (and O) of the segment before
                if (ns > 0 && !(ok = ptx::mbar_wait_warp(bar_o_empty + 8 * x, (ns - 1u) & 1u, abort_flag))) break;
                ++ns;
                const bool none = l == 0.f && fresh;   // (a row of NaN logits has a sum that is NaN)
                meta->stats[x][row] = make_float2(none ? 0.f : (kQ4 ? q4::kSmall : 1.f) / l, none ? -CUDART_INF_F : (fresh ? 0.f : m_ref) + log2f(l));
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_l_full + 8 * x);
            }
            tiles += s.hi - s.lo;
        }
    }

    // ---- teardown
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) atomicOr(p.a.c.status, kStatusTimeout);
        __nanosleep(200000);   // let copies and MMAs that may still be in flight land
        __syncthreads();
    }
    if (warp == 12) {
        __syncwarp();
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, kTmemCols);
    }
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    if (!fn) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
    }
    return fn;
}

// The outer dimensions of a tensor in the order of their strides (bytes), those of size 1 last.  False when two overlap in memory:
// such a layout is not a tiled tensor.
struct Dim { unsigned long long size, stride; int which; };
bool order_dims(Dim *d, int n, unsigned long long inner_bytes) {
    for (int a = 0; a < n; ++a)
        for (int b = a + 1; b < n; ++b) {
            const bool swap = (d[b].size > 1 && d[a].size == 1) ? true : (d[a].size > 1 && d[b].size == 1) ? false : d[b].stride < d[a].stride;
            if (swap) { const Dim t = d[a]; d[a] = d[b]; d[b] = t; }
        }
    unsigned long long extent = inner_bytes;
    for (int a = 0; a < n; ++a) {
        if (d[a].size == 1) d[a].stride = extent;
        else if (d[a].stride < extent || d[a].stride >= (1ull << 40)) return false;
        extent = d[a].stride * d[a].size;
        if (extent >= (1ull << 46)) return false;
    }
    return true;
}

bool kv_dims(const PagedCall &a, Dim (&d)[3]) {
    d[0] = {(unsigned long long)a.c.P, (unsigned long long)a.c.s_t * 2, 0};
    d[1] = {(unsigned long long)a.c.Hkv, (unsigned long long)a.c.s_h * 2, 1};
    d[2] = {(unsigned long long)a.c.n_pages, (unsigned long long)a.c.s_page * 2, 2};
    return order_dims(d, 3, (unsigned long long)a.c.D * 2);
}
bool q_dims(const PagedCall &a, Dim (&d)[2]) {
    d[0] = {(unsigned long long)a.Hq, (unsigned long long)a.q_sh * 2, 0};
    d[1] = {(unsigned long long)a.b.n_new, (unsigned long long)a.q_st * 2, 1};
    return order_dims(d, 2, (unsigned long long)a.c.D * 2);
}

bool make_map(CUtensorMap *tm, const void *ptr, int D, const Dim *d, int n, const cuuint32_t *box_outer) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t gdim[4] = {(cuuint64_t)D, 1, 1, 1}, gstr[3];
    cuuint32_t box[4] = {64, 1, 1, 1}, estr[4] = {1, 1, 1, 1};
    for (int a = 0; a < 3; ++a) {
        gdim[1 + a] = a < n ? d[a].size : 1;
        gstr[a] = a < n ? d[a].stride : d[n - 1].stride * d[n - 1].size;
        box[1 + a] = a < n ? box_outer[a] : 1;
    }
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(ptr), gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kLong, bool kQ4>
cudaError_t tiles_of(const void *q, const PagedCall &a, const PagedPlan &pl, char *scratch, void *out, float *lse, cudaStream_t st) {
    static bool allowed[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev]) {
        e = cudaFuncSetAttribute(paged_tiles<D, kLong, kQ4>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D, kQ4>::kSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev] = true;
    }
    TileParams p;
    p.a = a;
    p.plan = plan_at(pl, scratch);
    p.parts = parts_at(pl, scratch);
    p.q = (const bf16 *)q;
    p.out = (bf16 *)out;
    p.lse = lse;
    p.fold = pl.fold_bytes ? reinterpret_cast<float *>(scratch + pl.off_fold) : nullptr;
    p.TS = pl.TS;
    p.out32 = (reinterpret_cast<uintptr_t>(out) & 31u) == 0 && a.q_st % 16 == 0 && a.q_sh % 16 == 0;
    p.box_rows = a.c.P < kKeys ? a.c.P : kKeys;
    Dim kd[3] = {}, qd[2];
    if ((!kQ4 && !kv_dims(a, kd)) || !q_dims(a, qd)) return cudaErrorInvalidValue;
    int *slot[3] = {&p.slot_t, &p.slot_h, &p.slot_p};
    cuuint32_t kbox[3] = {1, 1, 1}, qbox[2];
    p.slot_t = p.slot_h = p.slot_p = 0;
    for (int i = 0; i < 3 && !kQ4; ++i) {
        *slot[kd[i].which] = i;
        if (kd[i].which == 0) kbox[i] = p.box_rows;
    }
    p.t_inner = qd[0].which == 1;
    for (int i = 0; i < 2; ++i) qbox[i] = qd[i].which == 1 ? pl.TS : a.G;
    CUtensorMap tq, tk, tv;
    if (!make_map(&tq, q, D, qd, 2, qbox)) return cudaErrorInvalidValue;
    tk = tv = tq;   // (four bits: not looked at)
    if (!kQ4 && (!make_map(&tk, a.c.k, D, kd, 3, kbox) || !make_map(&tv, a.c.v, D, kd, 3, kbox))) return cudaErrorInvalidValue;
    return launch_chained(paged_tiles<D, kLong, kQ4>, dim3(pl.n_ctas), dim3(kThreads), Layout<D, kQ4>::kSmem, st, tq, tk, tv, p);
}

}  // namespace

// bf16, strides that nest in memory (no broadcast views), a scale that keeps the order of the logits and -inf what it is
bool paged_tiles_supported(const PagedCall &a, int dtype) {
    Dim kd[3], qd[2];
    return dtype == SLA_BF16 && a.scale > 0.f && (q4::is(a.c) || kv_dims(a, kd)) && q_dims(a, qd);
}

void plan_paged_tiles(const PagedCall &a, PagedPlan &p, int sm_count) {
    p.R = 2 * kRows;
    p.RS = kRows;
    p.TS = kRows / a.G;
    p.TQ = 2 * p.TS;
    p.kt_shift = kTileShift;
    p.small = p.TS;
    p.n_ctas = sm_count;
    // (a bound that does not ask the number of SMs, so that the workspace can be sized without a device)
    const long long units = a.b.n_new / p.TQ + a.b.n_seqs, weight = units * a.c.Hkv * (((long long)a.c.width << a.c.shift) / kKeys + 1 + kUnitWeight);
    const long long bytes = (long long)a.c.n_pages * a.c.P * a.c.Hkv * row_bytes(a.c) * 2, groups = bytes / kGroupBytes + 1;
    const long long most = groups < weight / (128 * kGroupWeight) ? groups : weight / (128 * kGroupWeight);
    p.max_groups = most < 1 ? 1 : most < 8 ? (int)most : 8;
    p.min_weight = 3;
    // A unit's keys at most: of a table row, or of its tokens' windows, with the tiles at either end.  (A warp's 32 rows of O and a maximum each, in
    // 16-byte pieces.)
    const long long row = (long long)a.c.width << a.c.shift, keys = a.window > 0 && a.window < row ? (long long)a.window + p.TQ + 2 * kKeys : row;
    p.fold_bytes = keys > (long long)kFoldTiles * kKeys ? (size_t)sm_count * 8 * 32 * (a.c.D + 4) * sizeof(float) : 0;
}

template <bool kQ4>
static cudaError_t tiles_for(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    if (p.fold_bytes) return a.c.D == 64 ? tiles_of<64, true, kQ4>(q, a, p, scratch, out, lse, st) : tiles_of<128, true, kQ4>(q, a, p, scratch, out, lse, st);
    return a.c.D == 64 ? tiles_of<64, false, kQ4>(q, a, p, scratch, out, lse, st) : tiles_of<128, false, kQ4>(q, a, p, scratch, out, lse, st);
}

cudaError_t launch_paged_tiles(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st) {
    return q4::is(a.c) ? tiles_for<true>(q, a, p, scratch, out, lse, st) : tiles_for<false>(q, a, p, scratch, out, lse, st);
}

}  // namespace sla
