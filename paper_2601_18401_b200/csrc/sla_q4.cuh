// A paged cache in four bits: its format, and the device code that takes it apart (internal; the public interface is include/sla.h).
//
// A row (token, KV head) is held in groups of 32 consecutive dimensions.  With a = max |x| of the group
//     s = the smallest number of five significant bits with 7.5 s >= a, at least 2^-40,      c = x / s rounded, halves away from zero, |c| <= 7,
// and x is read as c s, off by at most s / 2.  Three and five bits make eight: c s is a bf16 number, so that reading back rounds nothing and the
// tensor cores get the very values that the cache holds.  A group with an infinity or a NaN, or whose s would be 2^40 or more, has s = NaN: it
// reads as NaN.  The bounds of s keep every product below with the powers of two that the kernels carry along inside the range of fp32.
//
// A plane is a page's rows of one head: P rows of codes, D / 2 bytes each, then P rows of scales, D / 32 bf16 each.
// Four codes make a 16-bit unit.  Dimension d = 32 g + 8 c + 2 i + h is code i of the unit (g, c, h).  The units of a row lie in the order
//     keys:   (c, g, h)      a 32-bit word has a group's eight neighbouring dimensions 32 g + 8 c ..
//     values: (c, h, g)      8 bytes have four codes of each of the four groups (D 64: 4 bytes of two)
// which is what a thread of an MMA needs: of a key (a column of B) every fourth piece of eight dimensions, one group after the other; of values
// (rows of A) four dimensions of every group, to be paired with the neighbouring token's.
// In a unit, code i is a sign and a magnitude of three bits:
//     bit  15 14 13 12 11 10  9  8  7  6  5  4  3  2  1  0
//          s0 s1 m3 m3 m3 m2 m2 m2 s2 s3 m1 m1 m1 m0 m0 m0
// so that one AND, behind a shift by one and a swap of bytes where these are needed, leaves a bf16: sign, exponent zero, and the magnitude
// in the fraction, a subnormal of value c 2^-133 (codes 0 and 2) or 16 c 2^-133 (codes 1 and 3).  Products with it are exact, and the power of two
// leaves with a factor that is applied anyway.  Seven instructions for eight codes; offset codes that are subtracted take eleven.
#pragma once

#include "sla_paged.cuh"

namespace sla {
namespace q4 {

// (strides of such a cache are in bytes)
__host__ __device__ inline bool is(const Pages &p) { return p.es == 1; }
__host__ __device__ inline int plane_bytes(int P, int D) { return P * (D / 2 + D / 16); }

// The eight codes of two units (the halves of w), pairs of equal place: r[i] = {code i of the low unit, of the high unit} as bf16 subnormals.
__device__ __forceinline__ void pairs(uint32_t w, uint32_t (&r)[4]) {
    const uint32_t x = __byte_perm(w, 0, 0x2301);   // bytes of the halves swapped
    r[0] = w & 0x80078007u;
    r[1] = (w << 1) & 0x80708070u;
    r[2] = x & 0x80078007u;
    r[3] = (x << 1) & 0x80708070u;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// A scale as the factor of values(): 2^13 s in both halves.
__device__ __forceinline__ uint32_t factor(uint32_t s) { return mul_bf16x2(s * 0x10001u, 0x46004600u); }   // (s: the 16 bits of a bf16)
// The values of those codes in bf16, exact: c 2^-133 times 2^120 (16 c 2^-133 times 2^116) is c 2^-13.
__device__ __forceinline__ void values(uint32_t w, uint32_t f, uint32_t (&r)[4]) {
    pairs(w, r);
    r[0] = mul_bf16x2(mul_bf16x2(r[0], 0x7b807b80u), f);
    r[1] = mul_bf16x2(mul_bf16x2(r[1], 0x79807980u), f);
    r[2] = mul_bf16x2(mul_bf16x2(r[2], 0x7b807b80u), f);
    r[3] = mul_bf16x2(mul_bf16x2(r[3], 0x79807980u), f);
}
// The values times 2^-48, from the scale in both halves of s: one product a pair, with 2^85 s or 2^81 s (which are bf16 numbers, s being below 2^40).
constexpr float kSmall = 0x1p48f;
__device__ __forceinline__ void small_values(uint32_t w, uint32_t s, uint32_t (&r)[4]) {
    const uint32_t f0 = mul_bf16x2(s, 0x6a006a00u), f1 = mul_bf16x2(s, 0x68006800u);   // 2^85, 2^81
    pairs(w, r);
    r[0] = mul_bf16x2(r[0], f0);
    r[1] = mul_bf16x2(r[1], f1);
    r[2] = mul_bf16x2(r[2], f0);
    r[3] = mul_bf16x2(r[3], f1);
}

// N words of shared memory, as wide as they are
template <int N> __device__ __forceinline__ void load_shared(uint32_t at, uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    } else if constexpr (N == 2) {
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at + 4 * i));
    }
}
// Where a row of a plane has what: bytes from the plane's start.
__device__ __forceinline__ int codes_at(int D, int t) { return t * (D / 2); }
__device__ __forceinline__ int scales_at(int P, int D, int t) { return P * (D / 2) + t * (D / 16); }
// The piece of eight dimensions 8 j .. of a row: its two units as a word (even dimensions in the low half, odd ones in the high half), and its scale.
template <bool kValues>
__device__ __forceinline__ void load_piece(const char *plane, int P, int D, int t, int j, uint32_t &w, uint32_t &s) {
    const int n = D / 32, g = j >> 2, c = j & 3;
    const char *row = plane + codes_at(D, t);
    s = __ldg(reinterpret_cast<const unsigned short *>(plane + scales_at(P, D, t)) + g);
    if (kValues) {
        const unsigned short *u = reinterpret_cast<const unsigned short *>(row) + 2 * c * n + g;
        w = __ldg(u) | (uint32_t)__ldg(u + n) << 16;
    } else {
        w = __ldg(reinterpret_cast<const uint32_t *>(row) + c * n + g);
    }
}
// Its values in fp32.
template <bool kValues>
__device__ __forceinline__ void load_values(const char *plane, int P, int D, int t, int j, float (&f)[8]) {
    uint32_t w, s, r[4];
    load_piece<kValues>(plane, P, D, t, j, w, s);
    values(w, factor(s), r);
    Vec16<__nv_bfloat16>::unpack(make_uint4(r[0], r[1], r[2], r[3]), f);
}
// The 16 bits of the scale of dimension d.
__device__ __forceinline__ uint32_t scale_of(const char *plane, int P, int D, int t, int d) {
    return __ldg(reinterpret_cast<const unsigned short *>(plane + scales_at(P, D, t)) + d / 32);
}
__device__ __forceinline__ bool is_nan(uint32_t s) { return (s & 0x7fffu) > 0x7f80u; }

// The scale of a group whose largest magnitude has the bits a (fp32, no sign): bits of a bf16.  The quotient is cut to five bits, and goes up
// by one of them where it is too small; 7.5 s has nine bits, so that the comparison is exact.
__device__ __forceinline__ uint32_t scale_for(uint32_t a) {
    const float x = __uint_as_float(a);
    uint32_t s = __float_as_uint(x * (2.f / 15.f)) & 0xfff80000u;
    if (7.5f * __uint_as_float(s) < x) s += 0x80000u;
    s = max(s, 0x2b800000u);                                      // 2^-40
    return a >= 0x7f800000u || s >= 0x53800000u ? 0x7fc0u : s >> 16;   // 2^40
}

}  // namespace q4
}  // namespace sla
