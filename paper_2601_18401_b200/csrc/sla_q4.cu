// A paged cache in four bits (format: sla_q4.cuh): quantising new tokens as they are written, and reading rows of a cache back.
//
//   append_q4     a warp per new token, or several (and 1024 values of each): loads their K and V, finds their places meanwhile, a scale per four lanes, codes
//   read_q4       a warp per row, or several (and 512 values of each): values of a cache in four bits, in bf16 or fp32
//   read_rows     the same of other caches, whose rows are copied
//
// A lane has eight neighbouring dimensions, four lanes a group.  What appending takes are instructions (245 for eight values of K and of V; issue slots
// 70 %, ALU pipe 61 %), reading the latency of a row's loads behind its lookups.  Measured in a graph (8 heads, D 128, the rate of a copy being 6.5 TB/s):
// 18.7 thousand tokens in bf16 appended in 24 us, 4.1 TB/s, in fp32 in 48 us, 3.6 TB/s; 65536 rows read into bf16 in 64 us, 5.4 TB/s, into fp32 in 127 to
// 132 us, 4.7 TB/s; as many of a cache in bf16 in 88 us, 6.1 TB/s, in fp32 in 172 us, 6.2 TB/s.
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

// Pages and rows in them of rows of the call that a warp goes through one after another: what it looked up stays while the rows stay in the
// sequence, and in the page.  first NULL: rows count from the sequence's start.  held: positions the sequence has not are no place.
struct Places {
    int lo = 0, hi = 0, f = 0, most = 0, col = -1;
    long long plane = 0;         // of the page, in elements
    const int *row = nullptr;

    // false where there is none; t: its row of the page
    __device__ __forceinline__ bool at(const Pages &p, const Batch &b, const int *first, bool held, int r, int &t) {
        if (r >= hi) {
            const int x = sequence_of(b, r);
            col = -1;
            f = -1;
            if (x < b.n_seqs) {
                new_rows(b, x, lo, hi);
                f = first ? first[x] : 0;
                const int s = slot_of(p, b, x);
                if (s >= 0) {
                    row = p.table + (long long)s * p.width;
                    most = held ? tokens_of(p, s) : p.width << p.shift;
                } else if (f >= 0) {
                    f = -1;
                    atomicOr(p.status, kStatusBadIndex);
                }
            }
        }
        if (r < lo || r >= hi || f < 0) return false;
        const long long pos = (long long)f + (r - lo);
        if (pos >= most) {
            atomicOr(p.status, kStatusBadIndex);
            return false;
        }
        t = (int)(pos & (p.P - 1));
        if (col != (int)(pos >> p.shift)) {
            col = (int)(pos >> p.shift);
            const int page = row[col];
            const bool there = (unsigned)page < (unsigned)p.n_pages;
            plane = there ? page * p.s_page : -1;
            if (!there) atomicOr(p.status, kStatusBadIndex);
        }
        return plane >= 0;
    }
};
// A lane's pieces of a row (K's and V's alike): piece j of the heads head, head + by, ..; those below Hkv exist.
struct Pieces {
    int j, head, by;
    __device__ __forceinline__ Pieces(int per_head, int part, int U) {   // (8, 16 or 32 pieces a head)
        const int lane = threadIdx.x & 31;
        by = 32 / per_head;
        j = lane & (per_head - 1);
        head = part * U * by + (unsigned)lane / per_head;
    }
};

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
    __device__ __forceinline__ uint32_t signs() const {   // where the codes have them
        return (v.x & 0x80008000u) | (v.y >> 1 & 0x40004000u) | (v.z >> 8 & 0x00800080u) | (v.w >> 9 & 0x00400040u);
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
    __device__ __forceinline__ uint32_t signs() const {
        constexpr int kSign[4] = {15, 14, 7, 6};
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= __float_as_uint(at(i)) >> (31 - kSign[i / 2] - 16 * (i & 1)) & 1u << (kSign[i / 2] + 16 * (i & 1));
        return w;
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(at(i)) & 0x7fffffffu);
        return m;
    }
};

// The two units of a piece, even dimensions in the low half.  2^23 + |x| / s has the code in its lowest bits; the quotient is held below 7.5 by the
// saturation of its product with 1 / 7.4999, which needs no instruction.  Halves go up: a bf16 x that is not exactly half way between two codes is at
// least 2^-9 of its size away (eight bits against nine), so that a quotient made 2^-16 larger rounds as the exact one does, also where the reciprocal
// is off by 2^-22; an fp32 x may be nearer, and the rest x - c s, which is exact, decides.
__device__ __forceinline__ float mul_sat(float a, float b) {
    float d;
    asm("mul.rn.sat.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float reciprocal(float a) {
    float d;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(a));
    return d;
}
__device__ __forceinline__ uint32_t shift_add(uint32_t a, int k, uint32_t b) {   // on the pipe of the multiplications: the other one is the busier
    uint32_t d;
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(1u << k), "r"(b));
    return d;
}
template <typename T>
__device__ __forceinline__ uint32_t codes_of(const Piece<T> &p, uint32_t scale) {
    constexpr bool kExact = sizeof(T) == 4;
    constexpr int kAt[4] = {0, 3, 8, 11};
    constexpr float kMost = 7.4999f;
    const float s = __uint_as_float(scale << 16), inv = reciprocal(s) * ((kExact ? 1.f : 1.f + 0x1p-16f) / kMost);
    uint32_t base = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) base += (0x4b000000u << kAt[i]) + (0x4b000000u << (kAt[i] + 16));
    uint32_t w = 0u - base;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = fabsf(p.at(2 * i + h));
            float z = fmaf(mul_sat(x, inv), kMost, 0x1p23f);
            if (kExact) {
                const float rest = fmaf(0x1p23f - z, s, x);
                if (rest >= 0.5f * s && z < 0x1p23f + 7.f) z += 1.f;
                if (rest < -0.5f * s) z -= 1.f;
            }
            w = shift_add(__float_as_uint(z), kAt[i] + 16 * h, w);
        }
    return q4::is_nan(scale) ? 0u : w | p.signs();
}

// Of values, the words that lie in memory have a unit of two neighbouring groups; the lane of the even group has those of h = 0.  From a piece's two
// units (h = 0 low) to such a word and back, by a whole warp: lanes of neighbouring groups are four apart.
__device__ __forceinline__ uint32_t exchange_units(uint32_t w, int j) {
    const uint32_t other = __shfl_xor_sync(kFull, w, 4);
    return j >> 2 & 1 ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
}
template <bool kValues>
__device__ __forceinline__ void store_units(char *plane, int P, int D, int t, int j, uint32_t w, uint32_t s, bool on) {
    const int n = D / 32, g = j >> 2, c = j & 3;
    if (kValues) w = exchange_units(w, j);
    if (!on) return;
    uint32_t *row = reinterpret_cast<uint32_t *>(plane + q4::codes_at(D, t));
    row[kValues ? (2 * c + (g & 1)) * (n / 2) + (g >> 1) : c * n + g] = w;
    if (c == 0) reinterpret_cast<unsigned short *>(plane + q4::scales_at(P, D, t))[g] = (unsigned short)s;
}
template <bool kValues>
__device__ __forceinline__ uint32_t load_units(const char *plane, int D, int t, int j, bool on) {
    const int n = D / 32, g = j >> 2, c = j & 3;
    const uint32_t *row = reinterpret_cast<const uint32_t *>(plane + q4::codes_at(D, t));
    return on ? __ldg(row + (kValues ? (2 * c + (g & 1)) * (n / 2) + (g >> 1) : c * n + g)) : 0;   // (values: for exchange_units)
}

template <typename T, int U>
__global__ void __launch_bounds__(kThreads) append_q4(Pages p, Batch b, const int *__restrict__ first, const char *__restrict__ k_new,
                                                      const char *__restrict__ v_new, long long s_t, long long s_h, int rows) {
    chain_wait();
    chain_release();
    const Pieces l(p.D / 8, blockIdx.y, U);
    const long long from_head = (l.head * s_h + l.j * 8) * (long long)sizeof(T), by = l.by * s_h * (long long)sizeof(T);
    for (long long r0 = (blockIdx.x * (long long)kWarps + (threadIdx.x >> 5)) * rows; r0 < b.n_new; r0 += gridDim.x * (long long)kWarps * rows) {
        Places places;
#pragma unroll 1
        for (int r = (int)r0, end = (int)min(r0 + rows, (long long)b.n_new); r < end; ++r) {
            Piece<T> kk[U], vv[U];
            const long long from = r * s_t * (long long)sizeof(T) + from_head;
#pragma unroll
            for (int e = 0; e < U; ++e) {
                if (l.head + e * l.by < p.Hkv) {
                    kk[e].load(k_new + from + e * by);
                    vv[e].load(v_new + from + e * by);
                } else {
                    kk[e].clear();
                    vv[e].clear();
                }
            }
            int t;
            if (!places.at(p, b, first, false, r, t)) continue;
#pragma unroll
            for (int e = 0; e < U; ++e) {
                uint32_t ka = kk[e].top(), va = vv[e].top();
#pragma unroll
                for (int off = 1; off < 4; off <<= 1) {
                    ka = max(ka, __shfl_xor_sync(kFull, ka, off));
                    va = max(va, __shfl_xor_sync(kFull, va, off));
                }
                const uint32_t ks = q4::scale_for(ka), vs = q4::scale_for(va);
                const long long plane = places.plane + (l.head + e * l.by) * p.s_h;
                const bool on = l.head + e * l.by < p.Hkv;
                store_units<false>(p.k + plane, p.P, p.D, t, l.j, codes_of(kk[e], ks), ks, on);
                store_units<true>(p.v + plane, p.P, p.D, t, l.j, codes_of(vv[e], vs), vs, on);
            }
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
__global__ void __launch_bounds__(kThreads) read_q4(Pages p, Batch b, const int *__restrict__ first, Out out, int rows) {
    chain_wait();
    chain_release();
    const Pieces l(p.D / 8, blockIdx.y, U);
    const long long to_head = (l.head * out.s_h + l.j * 8) * (long long)sizeof(T), by = l.by * out.s_h * (long long)sizeof(T);
    for (long long r0 = (blockIdx.x * (long long)kWarps + (threadIdx.x >> 5)) * rows; r0 < b.n_new; r0 += gridDim.x * (long long)kWarps * rows) {
        Places places;
#pragma unroll 1
        for (int r = (int)r0, end = (int)min(r0 + rows, (long long)b.n_new); r < end; ++r) {
            int t;
            if (!places.at(p, b, first, true, r, t)) continue;
            uint32_t kw[U], vw[U], ks[U], vs[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const bool on = l.head + e * l.by < p.Hkv;
                const long long plane = places.plane + (l.head + e * l.by) * p.s_h;
                kw[e] = load_units<false>(p.k + plane, p.D, t, l.j, on);
                vw[e] = load_units<true>(p.v + plane, p.D, t, l.j, on);
                ks[e] = on ? q4::scale_of(p.k + plane, p.P, p.D, t, 8 * l.j) : 0;
                vs[e] = on ? q4::scale_of(p.v + plane, p.P, p.D, t, 8 * l.j) : 0;
            }
            const long long to = r * out.s_t * (long long)sizeof(T) + to_head;
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const uint32_t vwe = exchange_units(vw[e], l.j);
                if (l.head + e * l.by >= p.Hkv) continue;
                uint32_t w[4];
                q4::values(kw[e], q4::factor(ks[e]), w);
                store_values<T>(out.k + to + e * by, w);
                q4::values(vwe, q4::factor(vs[e]), w);
                store_values<T>(out.v + to + e * by, w);
            }
        }
    }
}

// Rows of a cache that is not in four bits, as they are: pieces of 16 bytes.
template <int U>
__global__ void __launch_bounds__(kThreads) read_rows(Pages p, Batch b, const int *__restrict__ first, Out out, int rows) {
    chain_wait();
    chain_release();
    const Pieces l(p.D * p.es / 16, blockIdx.y, U);
    for (long long r0 = (blockIdx.x * (long long)kWarps + (threadIdx.x >> 5)) * rows; r0 < b.n_new; r0 += gridDim.x * (long long)kWarps * rows) {
        Places places;
#pragma unroll 1
        for (int r = (int)r0, end = (int)min(r0 + rows, (long long)b.n_new); r < end; ++r) {
            int t;
            if (!places.at(p, b, first, true, r, t)) continue;
            uint4 kk[U], vv[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int head = l.head + e * l.by;
                const long long from = (places.plane + head * p.s_h + t * p.s_t) * p.es + l.j * 16;
                if (head < p.Hkv) {
                    kk[e] = __ldg(reinterpret_cast<const uint4 *>(p.k + from));
                    vv[e] = __ldg(reinterpret_cast<const uint4 *>(p.v + from));
                }
            }
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int head = l.head + e * l.by;
                const long long to = (r * out.s_t + head * out.s_h) * p.es + l.j * 16;
                if (head < p.Hkv) {
                    *reinterpret_cast<uint4 *>(out.k + to) = kk[e];
                    *reinterpret_cast<uint4 *>(out.v + to) = vv[e];
                }
            }
        }
    }
}

// A warp for every `rows` rows and 32 U pieces of them: single rows until the chip is full of warps, then several, so that what is looked up
// serves them all.
// Pieces of a lane: one where there are not enough of them for every warp that the chip holds (a token of each of 48 sequences appended and read
// 9.9 us, 10.3 with two, 11.1 with four); else two to read and four to append, of which more are on their way together (18.7 thousand
// tokens of 8 heads of 128: appended in 24.0 us, 24.1 with two, 26.9 with one; 65536 read head by head in 64.5 us, 68 with four or one).  Appending
// in fp32 takes one, as many bytes as two in bf16: 74 us for three chunks of 4000 to 8192 tokens written and read, 77 with four.
constexpr int kReadPieces = 2, kAppendPieces = 4;
struct Grid {
    dim3 ctas;
    int rows;
};
bool few_pieces(const Batch &b, int pieces, int sm_count) { return (long long)b.n_new * pieces <= (long long)sm_count * 64 * 32; }
Grid grid_for(const Batch &b, int pieces, int U, int sm_count) {
    const int parts = (pieces + 32 * U - 1) / (32 * U);
    const long long warps = (long long)sm_count * 64, items = (long long)b.n_new * parts;
    const int rows = items > 8 * warps ? 8 : items > warps ? (int)((items + warps - 1) / warps) : 1;
    const long long ctas = ((b.n_new + rows - 1) / rows + kWarps - 1) / kWarps;
    return {dim3((unsigned)(ctas < (1 << 20) ? ctas : 1 << 20), parts), rows};
}

}  // namespace

template <typename T, int U>
static cudaError_t append_of(const Pages &p, const Batch &b, const int *first, const void *k_new, const void *v_new, long long s_t, long long s_h,
                             int sm_count, cudaStream_t st) {
    const Grid g = grid_for(b, p.Hkv * p.D / 8, U, sm_count);
    return launch_chained(append_q4<T, U>, g.ctas, dim3(kThreads), 0, st, p, b, first, (const char *)k_new, (const char *)v_new, s_t, s_h, g.rows);
}
cudaError_t launch_append_q4(const Pages &p, const Batch &b, const int *first, bool f32, const void *k_new, const void *v_new,
                             long long s_t, long long s_h, int sm_count, cudaStream_t st) {
    if (b.n_new == 0) return cudaSuccess;
    if (f32) return append_of<float, 1>(p, b, first, k_new, v_new, s_t, s_h, sm_count, st);
    return few_pieces(b, p.Hkv * p.D / 8, sm_count) ? append_of<__nv_bfloat16, 1>(p, b, first, k_new, v_new, s_t, s_h, sm_count, st)
                                                    : append_of<__nv_bfloat16, kAppendPieces>(p, b, first, k_new, v_new, s_t, s_h, sm_count, st);
}

template <int U>
static cudaError_t read_of(const Pages &p, const Batch &b, const int *first, bool f32, const Out &out, int pieces, int sm_count, cudaStream_t st) {
    const Grid g = grid_for(b, pieces, U, sm_count);
    if (!q4::is(p)) return launch_chained(read_rows<U>, g.ctas, dim3(kThreads), 0, st, p, b, first, out, g.rows);
    return f32 ? launch_chained(read_q4<float, U>, g.ctas, dim3(kThreads), 0, st, p, b, first, out, g.rows)
               : launch_chained(read_q4<__nv_bfloat16, U>, g.ctas, dim3(kThreads), 0, st, p, b, first, out, g.rows);
}
cudaError_t launch_cache_read(const Pages &p, const Batch &b, const int *first, bool f32, void *k_out, void *v_out, long long s_t,
                              long long s_h, int sm_count, cudaStream_t st) {
    if (b.n_new == 0) return cudaSuccess;
    const int pieces = q4::is(p) ? p.Hkv * p.D / 8 : p.Hkv * p.D * p.es / 16;
    const Out out = {(char *)k_out, (char *)v_out, s_t, s_h};
    return few_pieces(b, pieces, sm_count) ? read_of<1>(p, b, first, f32, out, pieces, sm_count, st) : read_of<kReadPieces>(p, b, first, f32, out, pieces, sm_count, st);
}

}  // namespace sla
