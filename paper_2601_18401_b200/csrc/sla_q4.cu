// A paged cache in four bits (format: sla_q4.cuh): quantising new tokens as they are written, and reading rows of a cache back.
//
//   append_q4     a warp per new token (or 1024 values of it): loads its K and V, finds its place meanwhile, a scale per four lanes, codes
//   cache_read    a warp per row (or 128 pieces of it): values of a four-bit cache in bf16 or fp32, or the rows of another cache as they are
#include "sla_q4.cuh"

namespace sla {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr unsigned kFull = 0xffffffffu;

// The last x with cu[x] <= r, 32 ways a step; a converged warp.
__device__ __forceinline__ int sequence_of(const Batch &b, int r) {
    if (!b.cu) return r;
    const int lane = threadIdx.x & 31;
    int lo = 0, n = b.n_seqs;
    while (n > 1) {
        const int step = (n + 31) / 32, probe = lo + min(lane * step, n - 1);
        const unsigned le = __ballot_sync(kFull, b.cu[probe] <= r && lane * step < n);
        const int at = le ? 31 - __clz(le) : 0;
        lo += at * step;
        n = min(step, n - at * step);
    }
    return lo;
}

// Page and row of the call's row r; false where there is none.  first NULL: rows count from the sequence's start.  held: positions the
// sequence has not are no place.
__device__ __forceinline__ bool place_of(const Pages &p, const Batch &b, const int *first, int r, bool held, int &page, int &t) {
    const int x = sequence_of(b, r);
    if (x >= b.n_seqs) return false;
    int lo, hi;
    new_rows(b, x, lo, hi);
    const int f = first ? first[x] : 0;
    if (r < lo || r >= hi || f < 0) return false;
    const int s = slot_of(p, b, x);
    const long long pos = (long long)f + (r - lo);
    if (s < 0 || pos >= (held ? tokens_of(p, s) : (long long)p.width << p.shift)) {
        atomicOr(p.status, kStatusBadIndex);
        return false;
    }
    page = p.table[(long long)s * p.width + (pos >> p.shift)];
    t = (int)(pos & (p.P - 1));
    if ((unsigned)page < (unsigned)p.n_pages) return true;
    atomicOr(p.status, kStatusBadIndex);
    return false;
}

// ---- quantising --------------------------------------------------------------------------------------------------------------------
// Eight values in fp32 and the bits of the largest magnitude among them.
template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const char *p) { v = __ldg(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ uint32_t top() const {   // of pairs of 15-bit magnitudes
        const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
    __device__ __forceinline__ float at(int i) const {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <> struct Piece<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const char *p) {
        a = __ldg(reinterpret_cast<const float4 *>(p));
        b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float at(int i) const {
        const float4 &w = i < 4 ? a : b;
        return (i & 3) == 0 ? w.x : (i & 3) == 1 ? w.y : (i & 3) == 2 ? w.z : w.w;
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(at(i)) & 0x7fffffffu);
        return m;
    }
};

// The two units of a piece, even dimensions in the low half.  2^23 + |x| / s has the code in its lowest bits.  Halves go up: a bf16 x that is
// not exactly half way between two codes is at least 2^-9 of its size away (eight bits against nine), so that a quotient made 2^-16 larger rounds
// as the exact one does; an fp32 x may be nearer, and the rest x - c s, which is exact, decides.
template <typename T>
__device__ __forceinline__ uint32_t codes_of(const Piece<T> &p, uint32_t scale) {
    constexpr bool kExact = sizeof(T) == 4;
    constexpr int kAt[4] = {0, 3, 8, 11}, kSign[4] = {15, 14, 7, 6};
    const float s = __uint_as_float(scale << 16), inv = __frcp_rn(s) * (kExact ? 1.f : 1.f + 0x1p-16f);
    uint32_t w = 0, signs = 0, base = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = p.at(2 * i + h);
            float z = fmaf(fabsf(x), inv, 0x1p23f);
            if (kExact) {
                const float rest = fmaf(0x1p23f - z, s, fabsf(x));
                if (rest >= 0.5f * s) z += 1.f;
                if (rest < -0.5f * s) z -= 1.f;
            }
            z = fminf(z, 0x1p23f + 7.f);
            w += __float_as_uint(z) << (kAt[i] + 16 * h);
            base += 0x4b000000u << (kAt[i] + 16 * h);
            signs |= (__float_as_uint(x) >> 31) << (kSign[i] + 16 * h);
        }
    return q4::is_nan(scale) ? 0u : (w - base) | signs;
}

// Stores the piece of a group (four lanes, eight lanes' worth for values): all lanes of a warp call it.
template <bool kValues>
__device__ __forceinline__ void store_units(char *plane, int P, int D, int t, int j, uint32_t w, uint32_t s, bool on) {
    const int n = D / 32, g = j >> 2, c = j & 3;
    if (kValues) {   // the units of two neighbouring groups make a word: the even group takes those of h = 0
        const uint32_t other = __shfl_xor_sync(kFull, w, 4);
        w = g & 1 ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
    }
    if (!on) return;
    uint32_t *row = reinterpret_cast<uint32_t *>(plane + q4::codes_at(D, t));
    row[kValues ? (2 * c + (g & 1)) * (n / 2) + (g >> 1) : c * n + g] = w;
    if (c == 0) reinterpret_cast<unsigned short *>(plane + q4::scales_at(P, D, t))[g] = (unsigned short)s;
}
template <bool kValues>
__device__ __forceinline__ uint32_t load_units(const char *plane, int D, int t, int j, bool on) {
    const int n = D / 32, g = j >> 2, c = j & 3;
    const uint32_t *row = reinterpret_cast<const uint32_t *>(plane + q4::codes_at(D, t));
    uint32_t w = on ? __ldg(row + (kValues ? (2 * c + (g & 1)) * (n / 2) + (g >> 1) : c * n + g)) : 0;
    if (kValues) {
        const uint32_t other = __shfl_xor_sync(kFull, w, 4);
        w = g & 1 ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
    }
    return w;
}

template <typename T, int U>
__global__ void __launch_bounds__(kThreads) append_q4(Pages p, Batch b, const int *__restrict__ first, const char *__restrict__ k_new,
                                                      const char *__restrict__ v_new, long long s_t, long long s_h, int parts) {
    chain_wait();
    chain_release();
    const int lane = threadIdx.x & 31, per_head = p.D / 8, pieces = p.Hkv * per_head;
    const long long items = (long long)b.n_new * parts;
    for (long long it = blockIdx.x * (long long)kWarps + (threadIdx.x >> 5); it < items; it += gridDim.x * (long long)kWarps) {
        const int r = (int)(it / parts), c0 = (int)(it - (long long)r * parts) * 32 * U + lane;
        Piece<T> kk[U], vv[U];
        int head[U], j[U];
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int c = c0 + 32 * e;
            head[e] = c / per_head;
            j[e] = c - head[e] * per_head;
            const long long from = (r * s_t + head[e] * s_h + j[e] * 8) * (long long)sizeof(T);
            if (c < pieces) {
                kk[e].load(k_new + from);
                vv[e].load(v_new + from);
            } else {
                kk[e].clear();
                vv[e].clear();
            }
        }
        int page, t;
        if (!place_of(p, b, first, r, false, page, t)) continue;
#pragma unroll
        for (int e = 0; e < U; ++e) {
            uint32_t ka = kk[e].top(), va = vv[e].top();
#pragma unroll
            for (int off = 1; off < 4; off <<= 1) {
                ka = max(ka, __shfl_xor_sync(kFull, ka, off));
                va = max(va, __shfl_xor_sync(kFull, va, off));
            }
            const uint32_t ks = q4::scale_for(ka), vs = q4::scale_for(va);
            const long long plane = page * p.s_page + head[e] * p.s_h;
            const bool on = c0 + 32 * e < pieces;
            store_units<false>(p.k + plane, p.P, p.D, t, j[e], codes_of(kk[e], ks), ks, on);
            store_units<true>(p.v + plane, p.P, p.D, t, j[e], codes_of(vv[e], vs), vs, on);
        }
    }
}

// ---- reading back --------------------------------------------------------------------------------------------------------------------
struct Out {
    char *k, *v;
    long long s_t, s_h;   // elements
};
template <typename T> __device__ __forceinline__ void store_values(char *to, const uint32_t (&r)[4]);
template <> __device__ __forceinline__ void store_values<__nv_bfloat16>(char *to, const uint32_t (&r)[4]) {
    *reinterpret_cast<uint4 *>(to) = make_uint4(r[0], r[1], r[2], r[3]);
}
template <> __device__ __forceinline__ void store_values<float>(char *to, const uint32_t (&r)[4]) {
    *reinterpret_cast<uint4 *>(to) = make_uint4(r[0] << 16, r[0] & 0xffff0000u, r[1] << 16, r[1] & 0xffff0000u);
    *reinterpret_cast<uint4 *>(to + 16) = make_uint4(r[2] << 16, r[2] & 0xffff0000u, r[3] << 16, r[3] & 0xffff0000u);
}

template <typename T, int U>
__global__ void __launch_bounds__(kThreads) read_q4(Pages p, Batch b, const int *__restrict__ first, Out out, int parts) {
    chain_wait();
    chain_release();
    const int lane = threadIdx.x & 31, per_head = p.D / 8, pieces = p.Hkv * per_head;
    const long long items = (long long)b.n_new * parts;
    for (long long it = blockIdx.x * (long long)kWarps + (threadIdx.x >> 5); it < items; it += gridDim.x * (long long)kWarps) {
        const int r = (int)(it / parts), c0 = (int)(it - (long long)r * parts) * 32 * U + lane;
        int page, t;
        if (!place_of(p, b, first, r, true, page, t)) continue;
        uint32_t kw[U], vw[U], ks[U], vs[U];
        long long to[U];
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int c = c0 + 32 * e, head = c / per_head, j = c - head * per_head;
            const bool on = c < pieces;
            const long long plane = page * p.s_page + head * p.s_h;
            kw[e] = load_units<false>(p.k + plane, p.D, t, j, on);
            vw[e] = load_units<true>(p.v + plane, p.D, t, j, on);
            ks[e] = on ? q4::scale_of(p.k + plane, p.P, p.D, t, 8 * j) : 0;
            vs[e] = on ? q4::scale_of(p.v + plane, p.P, p.D, t, 8 * j) : 0;
            to[e] = (r * out.s_t + head * out.s_h + j * 8) * (long long)sizeof(T);
        }
#pragma unroll
        for (int e = 0; e < U; ++e) {
            if (c0 + 32 * e >= pieces) continue;
            uint32_t w[4];
            q4::values(kw[e], q4::factor(ks[e]), w);
            store_values<T>(out.k + to[e], w);
            q4::values(vw[e], q4::factor(vs[e]), w);
            store_values<T>(out.v + to[e], w);
        }
    }
}

// Rows of a cache that is not in four bits, as they are: pieces of 16 bytes.
template <int U>
__global__ void __launch_bounds__(kThreads) read_rows(Pages p, Batch b, const int *__restrict__ first, Out out, int parts) {
    chain_wait();
    chain_release();
    const int lane = threadIdx.x & 31, per_head = p.D * p.es / 16, pieces = p.Hkv * per_head;
    const long long items = (long long)b.n_new * parts;
    for (long long it = blockIdx.x * (long long)kWarps + (threadIdx.x >> 5); it < items; it += gridDim.x * (long long)kWarps) {
        const int r = (int)(it / parts), c0 = (int)(it - (long long)r * parts) * 32 * U + lane;
        int page, t;
        if (!place_of(p, b, first, r, true, page, t)) continue;
        uint4 kk[U], vv[U];
        long long to[U];
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int c = c0 + 32 * e, head = c / per_head, j = c - head * per_head;
            const long long from = (page * p.s_page + head * p.s_h + t * p.s_t) * p.es + j * 16;
            to[e] = (r * out.s_t + head * out.s_h) * p.es + j * 16;
            if (c < pieces) {
                kk[e] = __ldg(reinterpret_cast<const uint4 *>(p.k + from));
                vv[e] = __ldg(reinterpret_cast<const uint4 *>(p.v + from));
            }
        }
#pragma unroll
        for (int e = 0; e < U; ++e)
            if (c0 + 32 * e < pieces) {
                *reinterpret_cast<uint4 *>(out.k + to[e]) = kk[e];
                *reinterpret_cast<uint4 *>(out.v + to[e]) = vv[e];
            }
    }
}

constexpr int kPieces = 4;   // of a lane: 1024 values of K and of V a warp
struct Grid {
    int parts;
    unsigned ctas;
};
Grid grid_for(const Batch &b, int pieces, int sm_count) {
    const int parts = (pieces + 32 * kPieces - 1) / (32 * kPieces);
    const long long ctas = ((long long)b.n_new * parts + kWarps - 1) / kWarps, most = (long long)sm_count * 8;
    return {parts, (unsigned)(ctas < most ? ctas : most)};
}

}  // namespace

cudaError_t launch_append_q4(const Pages &p, const Batch &b, const int *first, bool f32, const void *k_new, const void *v_new,
                             long long s_t, long long s_h, int sm_count, cudaStream_t st) {
    if (b.n_new == 0) return cudaSuccess;
    const Grid g = grid_for(b, p.Hkv * p.D / 8, sm_count);
    return f32 ? launch_chained(append_q4<float, kPieces>, dim3(g.ctas), dim3(kThreads), 0, st, p, b, first, (const char *)k_new, (const char *)v_new, s_t, s_h, g.parts)
               : launch_chained(append_q4<__nv_bfloat16, kPieces>, dim3(g.ctas), dim3(kThreads), 0, st, p, b, first, (const char *)k_new, (const char *)v_new, s_t, s_h, g.parts);
}

cudaError_t launch_cache_read(const Pages &p, const Batch &b, const int *first, bool f32, void *k_out, void *v_out, long long s_t,
                              long long s_h, int sm_count, cudaStream_t st) {
    if (b.n_new == 0) return cudaSuccess;
    const bool four = q4::is(p);
    const Grid g = grid_for(b, four ? p.Hkv * p.D / 8 : p.Hkv * p.D * p.es / 16, sm_count);
    const Out out = {(char *)k_out, (char *)v_out, s_t, s_h};
    if (!four) return launch_chained(read_rows<kPieces>, dim3(g.ctas), dim3(kThreads), 0, st, p, b, first, out, g.parts);
    return f32 ? launch_chained(read_q4<float, kPieces>, dim3(g.ctas), dim3(kThreads), 0, st, p, b, first, out, g.parts)
               : launch_chained(read_q4<__nv_bfloat16, kPieces>, dim3(g.ctas), dim3(kThreads), 0, st, p, b, first, out, g.parts);
}

}  // namespace sla
