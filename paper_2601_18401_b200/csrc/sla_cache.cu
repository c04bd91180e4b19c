// Paged key/value cache of libsla: handing out, sharing, moving and freeing pages, and writing new tokens into them.
// The bookkeeping (table, n_tokens, ref) lives on the device, so that no call waits for a length.
//
//   cache_extend     one CTA: pages each sequence lacks, a prefix sum of them, the free pages of lowest index
//   cache_append     a warp per (token, KB of its row): copies k_new and v_new to their places
//   cache_release    a thread per table entry: an exchange takes the entry, so that it loses its reference once
//   fork_plan, fork_share   one CTA hands out the pages for the partly filled ones; the grid shares the full ones and copies
//   compact_count, compact_rank, compact_move   pages in use per chunk; ranks of movers and holes; data, tables, ref
//
// All are bound by the latency of a few dependent loads except the copies of tokens and pages, which are bound by HBM.  Measured (8 KV
// heads, D 128, bf16): extend and append of a token to each of 48 sequences 7.4 us, of 18.7 thousand tokens to 3 sequences 33 us (153 MB
// moved, 23 us at the rate of a copy); 6 sequences forked to 48 9.4 us; a pool of 1 GB whose holes take 304 MB compacted in 114 us, 94 of
// them the copies at 6.5 TB/s.
#include "sla_q4.cuh"

namespace sla {

namespace {

constexpr int kPlanThreads = 1024;

// Inclusive prefix sum over the CTA (1024 threads); `total` receives the sum.  Every thread calls it.
__device__ inline int cta_scan(int v, int *s_warp, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v += y;
    }
    __syncthreads();   // s_warp is free
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    int w = s_warp[lane];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, off);
        if (lane >= off) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    return v + (warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0);
}

// The free pages (ref = 0) of lowest index, ascending, until `want` are found: free_list[0 .. found).  One CTA.
__device__ inline int find_free(const int *ref, int n_pages, int want, int *free_list, int *s_warp) {
    int found = 0;
    for (int p0 = 0; p0 < n_pages && found < want; p0 += 4 * kPlanThreads) {
        const int p = p0 + 4 * threadIdx.x;
        int is_free = 0;   // a bit per page
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (p + e < n_pages && ref[p + e] == 0) is_free |= 1 << e;
        int total;
        int at = found + cta_scan(__popc(is_free), s_warp, total) - __popc(is_free);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (is_free >> e & 1) {
                if (at < want) free_list[at] = p + e;
                ++at;
            }
        found += total;
    }
    __syncthreads();
    return min(found, want);
}

__device__ __forceinline__ int pages_for(const Pages &p, long long tokens) { return (int)((tokens + p.P - 1) >> p.shift); }

// free_list [n_pages], upto [n_seqs]: inclusive prefix sums of the pages wanted
__global__ void __launch_bounds__(kPlanThreads) cache_extend(Pages p, Batch b, int *__restrict__ first, int *__restrict__ free_list,
                                                             int *__restrict__ upto) {
    __shared__ int s_warp[32];
    chain_wait();
    chain_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = 0;
    for (int x0 = 0; x0 < b.n_seqs; x0 += kPlanThreads) {
        const int x = x0 + threadIdx.x;
        int need = 0;
        if (x < b.n_seqs) {
            const int s = slot_of(p, b, x);
            int lo, hi, at = -1;
            new_rows(b, x, lo, hi);
            if (s < 0) {
                atomicOr(p.status, kStatusBadIndex);
            } else {
                const long long n = p.n_tokens[s], want = n + (hi - lo);
                if (n < 0 || n > (long long)p.width << p.shift) atomicOr(p.status, kStatusBadIndex);
                else if (want > (long long)p.width << p.shift) atomicOr(p.status, kStatusCacheFull);
                else {
                    need = pages_for(p, want) - pages_for(p, n);
                    at = (int)n;
                }
            }
            first[x] = at;
        }
        int total;
        const int incl = sum + cta_scan(need, s_warp, total);
        if (x < b.n_seqs) upto[x] = incl;
        sum += total;
    }
    const int found = sum > 0 ? find_free(p.ref, p.n_pages, sum, free_list, s_warp) : 0;
    __syncthreads();
    // a warp per sequence: table entries, references, the new length
    for (int x = warp; x < b.n_seqs; x += kPlanThreads / 32) {
        const int at = first[x];
        const int end = upto[x], begin = x ? upto[x - 1] : 0;
        __syncwarp();
        if (at < 0) continue;
        if (end > begin && end > found) {
            if (lane == 0) {
                first[x] = -1;
                atomicOr(p.status, kStatusCacheFull);
            }
            continue;
        }
        const int s = slot_of(p, b, x);
        int lo, hi;
        new_rows(b, x, lo, hi);
        int *row = p.table + (long long)s * p.width + pages_for(p, at);
        for (int j = begin + lane; j < end; j += 32) {
            const int page = free_list[j];
            row[j - begin] = page;
            p.ref[page] = 1;
        }
        if (lane == 0) p.n_tokens[s] = at + (hi - lo);
    }
}

// A token's row [Hkv, D] of k and of v in pieces of 1 KB or less; a warp takes a piece of both at a time.
__global__ void __launch_bounds__(256) cache_append(Pages p, Batch b, const int *__restrict__ first, const char *__restrict__ k_new,
                                                    const char *__restrict__ v_new, long long s_t, long long s_h, int parts) {
    chain_wait();
    chain_release();
    const int lane = threadIdx.x & 31;
    const int per_head = p.D * p.es / 16, chunks = p.Hkv * per_head, part_len = (chunks + parts - 1) / parts;   // 16-byte chunks
    const long long items = (long long)b.n_new * parts;
    for (long long it = blockIdx.x * 8ll + (threadIdx.x >> 5); it < items; it += gridDim.x * 8ll) {
        const int r = (int)(it / parts), part = (int)(it - (long long)r * parts);
        // the last x with cu[x] <= r, 32 ways a step
        int x = r;
        if (b.cu) {
            int lo = 0, n = b.n_seqs;
            while (n > 1) {
                const int step = (n + 31) / 32, probe = lo + min(lane * step, n - 1);
                const unsigned le = __ballot_sync(0xffffffffu, b.cu[probe] <= r && lane * step < n);
                const int at = le ? 31 - __clz(le) : 0;
                lo += at * step;
                n = min(step, n - at * step);
            }
            x = lo;
        }
        if (x >= b.n_seqs) continue;
        int lo, hi;
        new_rows(b, x, lo, hi);
        const int f = first[x];
        if (r < lo || r >= hi || f < 0) continue;
        const int s = slot_of(p, b, x);
        const long long pos = (long long)f + (r - lo);
        if (s < 0 || pos >= (long long)p.width << p.shift) {
            if (lane == 0) atomicOr(p.status, kStatusBadIndex);
            continue;
        }
        const int page = p.table[(long long)s * p.width + (pos >> p.shift)];
        if ((unsigned)page >= (unsigned)p.n_pages) {
            if (lane == 0) atomicOr(p.status, kStatusBadIndex);
            continue;
        }
        const long long to = (page * p.s_page + (pos & (p.P - 1)) * p.s_t) * p.es, from = r * s_t * p.es;
        const int end = min(chunks, (part + 1) * part_len);
        for (int c0 = part * part_len + lane; c0 < end; c0 += 64) {
            uint4 kk[2], vv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = c0 + 32 * e, h = c / per_head, d = c - h * per_head;
                if (c < end) {
                    kk[e] = __ldg(reinterpret_cast<const uint4 *>(k_new + from + (long long)h * s_h * p.es + d * 16));
                    vv[e] = __ldg(reinterpret_cast<const uint4 *>(v_new + from + (long long)h * s_h * p.es + d * 16));
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = c0 + 32 * e, h = c / per_head, d = c - h * per_head;
                if (c < end) {
                    *reinterpret_cast<uint4 *>(p.k + to + (long long)h * p.s_h * p.es + d * 16) = kk[e];
                    *reinterpret_cast<uint4 *>(p.v + to + (long long)h * p.s_h * p.es + d * 16) = vv[e];
                }
            }
        }
    }
}

__global__ void __launch_bounds__(256) cache_release(Pages p, const int *__restrict__ seq) {
    chain_wait();
    chain_release();
    const int s = seq[blockIdx.x];
    if ((unsigned)s >= (unsigned)p.n_slots) {
        if (threadIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, kStatusBadIndex);
        return;
    }
    for (int c = blockIdx.y * 256 + threadIdx.x; c < p.width; c += gridDim.y * 256) {
        int *at = p.table + (long long)s * p.width + c;
        if (*at == -1) continue;
        const int page = atomicExch(at, -1);
        if (page == -1) continue;
        if ((unsigned)page >= (unsigned)p.n_pages) atomicOr(p.status, kStatusBadIndex);
        else if (atomicSub(p.ref + page, 1) <= 0) {   // the counts did not match the table
            atomicAdd(p.ref + page, 1);
            atomicOr(p.status, kStatusBadIndex);
        }
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) p.n_tokens[s] = 0;
}

// ---- copying pages ---------------------------------------------------------------------------------
// Where the 16-byte chunk c of a page lies, from the page's start, in bytes.  A page whose heads and tokens leave no gaps is one
// run of bytes; otherwise chunks go through (outer, inner, d) in the order of the strides.
struct PageShape {
    int chunks;         // of a page
    int dense;
    int per_row, inner; // 16-byte chunks of a (head, token) row; rows of the inner dimension
    long long s_outer, s_inner;   // bytes
};
__host__ __device__ inline PageShape page_shape(const Pages &p) {
    PageShape f;
    if (q4::is(p)) {   // a plane of each head
        f.per_row = q4::plane_bytes(p.P, p.D) / 16;
        f.chunks = p.Hkv * f.per_row;
        f.inner = p.Hkv;
        f.s_inner = p.s_h;
        f.s_outer = 0;
        f.dense = p.s_h == f.per_row * 16ll || p.Hkv == 1;
        return f;
    }
    f.per_row = p.D * p.es / 16;
    f.chunks = p.Hkv * p.P * f.per_row;
    const bool head_inner = p.Hkv > 1 && p.s_h < p.s_t;
    f.inner = head_inner ? p.Hkv : p.P;
    f.s_inner = (head_inner ? p.s_h : p.s_t) * p.es;
    f.s_outer = (head_inner ? p.s_t : p.s_h) * p.es;
    f.dense = f.s_inner == f.per_row * 16ll && (f.s_outer == f.s_inner * f.inner || p.Hkv == 1);
    return f;
}
__device__ __forceinline__ long long chunk_at(const PageShape &f, int c) {
    if (f.dense) return c * 16ll;
    const int row = c / f.per_row, d = c - row * f.per_row, o = row / f.inner;
    return o * f.s_outer + (row - o * f.inner) * f.s_inner + d * 16;
}

// Chunks [c0, c1) of page `from` to page `to`, k and v, by the threads of a CTA: four 16-byte loads of each in flight.
constexpr int kCopyThreads = 256, kCopyChunks = 4 * kCopyThreads;   // chunks of k and of v that one CTA copies in one go
__device__ inline void copy_page_part(const Pages &p, const PageShape &f, int from, int to, int part) {
    const char *ks = p.k + from * p.s_page * p.es, *vs = p.v + from * p.s_page * p.es;
    char *kd = p.k + to * p.s_page * p.es, *vd = p.v + to * p.s_page * p.es;
    uint4 a[4], b[4];
    long long at[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = part * kCopyChunks + e * kCopyThreads + threadIdx.x;
        at[e] = c < f.chunks ? chunk_at(f, c) : -1;
        if (at[e] >= 0) {
            a[e] = *reinterpret_cast<const uint4 *>(ks + at[e]);
            b[e] = *reinterpret_cast<const uint4 *>(vs + at[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (at[e] >= 0) {
            *reinterpret_cast<uint4 *>(kd + at[e]) = a[e];
            *reinterpret_cast<uint4 *>(vd + at[e]) = b[e];
        }
}

__global__ void __launch_bounds__(kCopyThreads) cache_copy(Pages p, PageShape f, const int *__restrict__ pairs, int n) {
    chain_wait();
    chain_release();
    const int from = pairs[blockIdx.x], to = pairs[n + blockIdx.x];
    if (from < 0 || to < 0) return;
    if (from >= p.n_pages || to >= p.n_pages) {
        if (threadIdx.x == 0) atomicOr(p.status, kStatusBadIndex);
        return;
    }
    if (from != to) copy_page_part(p, f, from, to, blockIdx.y);
}

// ---- fork -------------------------------------------------------------------------------------------
// free_list [n_pages], upto [n], full [n]: pages to share, 0 for a refused pair
__global__ void __launch_bounds__(kPlanThreads) fork_plan(Pages p, const int *__restrict__ src, const int *__restrict__ dst, int n,
                                                          int *__restrict__ pairs, int *__restrict__ free_list, int *__restrict__ upto, int *__restrict__ full) {
    __shared__ int s_warp[32];
    chain_wait();
    chain_release();
    int sum = 0;
    for (int x0 = 0; x0 < n; x0 += kPlanThreads) {
        const int x = x0 + threadIdx.x;
        int part = 0;
        if (x < n) {
            const int s = src[x], d = dst[x];
            int f = -1;   // tokens to share, -1: refused
            if ((unsigned)s >= (unsigned)p.n_slots || (unsigned)d >= (unsigned)p.n_slots || p.n_tokens[d] != 0) {
                atomicOr(p.status, kStatusBadIndex);
            } else {
                f = tokens_of(p, s);
                part = (f & (p.P - 1)) != 0;
            }
            full[x] = f;
        }
        int total;
        const int incl = sum + cta_scan(part, s_warp, total);
        if (x < n) upto[x] = incl;
        sum += total;
    }
    const int found = sum > 0 ? find_free(p.ref, p.n_pages, sum, free_list, s_warp) : 0;
    __syncthreads();
    for (int x = threadIdx.x; x < n; x += kPlanThreads) {
        int tokens = full[x], old = -1, to = -1;
        if (tokens >= 0 && (tokens & (p.P - 1))) {
            const int j = upto[x] - 1;
            old = p.table[(long long)src[x] * p.width + (tokens >> p.shift)];
            if (j >= found || (unsigned)old >= (unsigned)p.n_pages) {
                atomicOr(p.status, j >= found ? kStatusCacheFull : kStatusBadIndex);
                old = tokens = -1;
            } else {
                to = free_list[j];
                p.table[(long long)dst[x] * p.width + (tokens >> p.shift)] = to;
                p.ref[to] = 1;
            }
        }
        if (tokens > 0) p.n_tokens[dst[x]] = tokens;
        full[x] = tokens > 0 ? tokens >> p.shift : 0;
        pairs[x] = old;
        pairs[n + x] = to;
    }
}

// blockIdx.x: the pair; blockIdx.y < share_ctas: its table row, above: its partly filled page
__global__ void __launch_bounds__(kCopyThreads) fork_share(Pages p, PageShape f, const int *__restrict__ src, const int *__restrict__ dst,
                                                           int n, const int *__restrict__ pairs, const int *__restrict__ full,
                                                           int share_ctas) {
    chain_wait();
    chain_release();
    const int x = blockIdx.x;
    if ((int)blockIdx.y >= share_ctas) {
        const int from = pairs[x], to = pairs[n + x];
        if (to >= 0) copy_page_part(p, f, from, to, blockIdx.y - share_ctas);
        return;
    }
    const int pages = full[x];
    if (pages == 0) return;
    const int *from = p.table + (long long)src[x] * p.width;
    int *to = p.table + (long long)dst[x] * p.width;
    for (int c = blockIdx.y * kCopyThreads + threadIdx.x; c < pages; c += share_ctas * kCopyThreads) {
        const int page = from[c];
        to[c] = page;
        if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(p.ref + page, 1);
        else atomicOr(p.status, kStatusBadIndex);
    }
}

// ---- compact ----------------------------------------------------------------------------------------
// The pool in at most 1024 chunks of a multiple of 4096 pages.  count [kMaxChunks], behind it the number of moves; rank [n_pages]: of a
// mover among the movers, -1 otherwise
__host__ __device__ inline int chunk_pages(int n_pages) {
    const long long quantum = 4ll * kPlanThreads;
    return (int)(quantum * ((n_pages + quantum * kMaxChunks - 1) / (quantum * kMaxChunks)));
}

__device__ inline int count_live(const int *ref, int lo, int hi, int *s_warp) {
    int mine = 0;
#pragma unroll 4
    for (int q = lo + threadIdx.x; q < hi; q += kPlanThreads) mine += ref[q] > 0;
    int total;
    cta_scan(mine, s_warp, total);
    return total;
}

__global__ void __launch_bounds__(kPlanThreads) compact_count(Pages p, int per, int *__restrict__ count) {
    __shared__ int s_warp[32];
    chain_wait();
    chain_release();
    const int lo = blockIdx.x * per, hi = min(lo + per, p.n_pages);
    const int total = count_live(p.ref, lo, hi, s_warp);
    if (threadIdx.x == 0) count[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kPlanThreads) compact_rank(Pages p, int per, int *__restrict__ count, int *__restrict__ rank, int *__restrict__ pairs) {
    __shared__ int s_warp[32], s_before, s_below;
    chain_wait();
    chain_release();
    const int n_chunks = gridDim.x, c = threadIdx.x;
    // pages in use in all; before this chunk; in the whole chunks below page `live`
    const int mine = c < n_chunks ? count[c] : 0;
    int live;
    const int incl = cta_scan(mine, s_warp, live);
    if (c == (int)blockIdx.x) s_before = incl - mine;
    const int edge = live / per;   // the chunk that page `live` lies in (none of it when live == n_pages)
    if (c == 0) s_below = live;
    __syncthreads();
    if (c == edge && c < n_chunks) s_below = incl - mine;
    __syncthreads();
    const int below = s_below + (edge < n_chunks ? count_live(p.ref, edge * per, live, s_warp) : 0);
    const int n_moves = live - below;   // pages in use at or above `live`: as many as are free below it
    if (blockIdx.x == 0 && c == 0) count[kMaxChunks] = n_moves;
    int upto = s_before;
    for (int p0 = blockIdx.x * per; p0 < min((int)(blockIdx.x + 1) * per, p.n_pages); p0 += 4 * kPlanThreads) {
        const int q0 = p0 + 4 * c;   // four pages a thread
        int on = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (q0 + e < p.n_pages && p.ref[q0 + e] > 0) on |= 1 << e;
        int total;
        int before = upto + cta_scan(__popc(on), s_warp, total) - __popc(on);   // pages in use below q
        upto += total;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int q = q0 + e, is = on >> e & 1;
            if (q < p.n_pages) {
                if (q >= n_moves) pairs[q] = pairs[p.n_pages + q] = -1;
                rank[q] = is && q >= live ? before - below : -1;
                if (is && q >= live) pairs[before - below] = q;
                if (!is && q < live) pairs[p.n_pages + q - before] = q;
            }
            before += is;
        }
    }
}

__global__ void __launch_bounds__(kCopyThreads) compact_move(Pages p, PageShape f, const int *__restrict__ count, const int *__restrict__ rank,
                                                             const int *__restrict__ pairs, int table_ctas) {
    chain_wait();
    chain_release();
    const int n_moves = count[kMaxChunks];
    if ((int)blockIdx.x < table_ctas) {
        if (n_moves == 0) return;
        const long long entries = (long long)p.n_slots * p.width;
        for (long long e = blockIdx.x * (long long)kCopyThreads + threadIdx.x; e < entries; e += table_ctas * (long long)kCopyThreads) {
            const int page = p.table[e];
            if ((unsigned)page >= (unsigned)p.n_pages) {
                if (page != -1) atomicOr(p.status, kStatusBadIndex);
                continue;
            }
            const int r = rank[page];
            if (r >= 0) p.table[e] = pairs[p.n_pages + r];
        }
        return;
    }
    const int parts = (f.chunks + kCopyChunks - 1) / kCopyChunks;
    const long long items = (long long)n_moves * parts;
    for (long long it = blockIdx.x - table_ctas; it < items; it += gridDim.x - table_ctas) {
        const int j = (int)(it / parts), part = (int)(it - (long long)j * parts);
        const int from = pairs[j], to = pairs[p.n_pages + j];
        copy_page_part(p, f, from, to, part);
        if (part == 0 && threadIdx.x == 0) {
            p.ref[to] = p.ref[from];
            p.ref[from] = 0;
        }
    }
}

int parts_of(const PageShape &f) { return (f.chunks + kCopyChunks - 1) / kCopyChunks; }

}  // namespace

CacheScratch plan_cache(const Pages &p, int n_seqs, size_t gap) {
    CacheScratch s;
    size_t off = 0;
    auto take = [&](size_t ints) {
        if (gap) { s.canaries.add(off); off += gap; }
        const size_t at = off;
        off = (off + ints * sizeof(int) + 255) & ~(size_t)255;
        return at;
    };
    const size_t n = n_seqs > 0 ? n_seqs : 0;
    s.off_pages = take(p.n_pages);
    s.off_seqs = take(n);
    s.off_seqs2 = take(n);
    s.off_chunks = take(kMaxChunks + 1);
    if (gap) { s.canaries.add(off); off += gap; }
    s.bytes = off;
    return s;
}

cudaError_t launch_cache_extend(const Pages &p, const Batch &b, int *first, const CacheScratch &s, char *scratch, cudaStream_t st) {
    return launch_chained(cache_extend, dim3(1), dim3(kPlanThreads), 0, st, p, b, first, reinterpret_cast<int *>(scratch + s.off_pages),
                          reinterpret_cast<int *>(scratch + s.off_seqs));
}

cudaError_t launch_cache_append(const Pages &p, const Batch &b, const int *first, const void *k_new, const void *v_new,
                                long long s_t, long long s_h, int sm_count, cudaStream_t st) {
    if (b.n_new == 0) return cudaSuccess;
    const int parts = (p.Hkv * p.D * p.es + 1023) / 1024;
    const long long items = (long long)b.n_new * parts, most = (long long)sm_count * 8;
    const long long ctas = (items + 7) / 8 < most ? (items + 7) / 8 : most;
    return launch_chained(cache_append, dim3((unsigned)ctas), dim3(256), 0, st, p, b, first, (const char *)k_new, (const char *)v_new, s_t, s_h, parts);
}

cudaError_t launch_cache_release(const Pages &p, const int *seq, int n, cudaStream_t st) {
    if (n == 0) return cudaSuccess;
    const int ctas = (p.width + 1023) / 1024;
    return launch_chained(cache_release, dim3(n, ctas < 64 ? ctas : 64), dim3(256), 0, st, p, seq);
}

cudaError_t launch_cache_copy(const Pages &p, const int *pairs, int n, cudaStream_t st) {
    if (n == 0) return cudaSuccess;
    const PageShape f = page_shape(p);
    return launch_chained(cache_copy, dim3(n, parts_of(f)), dim3(kCopyThreads), 0, st, p, f, pairs, n);
}

cudaError_t launch_cache_fork(const Pages &p, const int *src, const int *dst, int n, int *pairs, const CacheScratch &s, char *scratch, cudaStream_t st) {
    if (n == 0) return cudaSuccess;
    const PageShape f = page_shape(p);
    int *full = reinterpret_cast<int *>(scratch + s.off_seqs2);
    cudaError_t e = launch_chained(fork_plan, dim3(1), dim3(kPlanThreads), 0, st, p, src, dst, n, pairs, reinterpret_cast<int *>(scratch + s.off_pages),
                                   reinterpret_cast<int *>(scratch + s.off_seqs), full);
    const int share = p.width < 16 * kCopyThreads ? (p.width + kCopyThreads - 1) / kCopyThreads : 16;
    if (e == cudaSuccess)
        e = launch_chained(fork_share, dim3(n, share + parts_of(f)), dim3(kCopyThreads), 0, st, p, f, src, dst, n, (const int *)pairs,
                           (const int *)full, share);
    return e;
}

cudaError_t launch_cache_compact(const Pages &p, int *pairs, const CacheScratch &s, char *scratch, int sm_count, cudaStream_t st) {
    const PageShape f = page_shape(p);
    int *count = reinterpret_cast<int *>(scratch + s.off_chunks), *rank = reinterpret_cast<int *>(scratch + s.off_pages);
    const int per = chunk_pages(p.n_pages), chunks = (p.n_pages + per - 1) / per;
    cudaError_t e = launch_chained(compact_count, dim3(chunks), dim3(kPlanThreads), 0, st, p, per, count);
    if (e == cudaSuccess) e = launch_chained(compact_rank, dim3(chunks), dim3(kPlanThreads), 0, st, p, per, count, rank, pairs);
    const long long entries = (long long)p.n_slots * p.width;
    const int table_ctas = (int)(entries < 64ll * 4 * kCopyThreads ? (entries + 4 * kCopyThreads - 1) / (4 * kCopyThreads) : 64);
    if (e == cudaSuccess)
        e = launch_chained(compact_move, dim3(table_ctas + sm_count * 8), dim3(kCopyThreads), 0, st, p, f, (const int *)count, (const int *)rank,
                           (const int *)pairs, table_ctas);
    return e;
}

}  // namespace sla
