// Paged key/value cache: what its kernels share (internal; the public interface is include/sla.h).
#pragma once

#include "sla_common.cuh"
#include "sla_kernels.h"

namespace sla {

// A cache by value, as the kernels take it.
struct Pages {
    char *k, *v;
    int *table, *n_tokens, *ref;
    int n_pages, P, shift;          // page_tokens = P = 1 << shift
    int Hkv, D, es;                 // es: bytes of an element
    int n_slots, width;
    long long s_page, s_h, s_t;     // in elements
    int *status;
};

// The sequences of a call.  (Small on purpose: with 160 bytes of arguments a launch of cache_extend takes the host 0.3 us less than with 168.)
struct Batch {
    int n_seqs, n_new, max_new;
    int slot0;                      // 0 where seq is not NULL
    const int *seq, *cu;            // either may be NULL (slots slot0 .. slot0 + n_seqs - 1; one token a sequence)
};

// Rows [lo, hi) of sequence x in the call's tensors, kept inside them whatever cu_new holds.
__device__ __forceinline__ void new_rows(const Batch &b, int x, int &lo, int &hi) {
    lo = b.cu ? min(max(b.cu[x], 0), b.n_new) : min(x, b.n_new);
    hi = b.cu ? min(max(b.cu[x + 1], lo), b.n_new) : min(x + 1, b.n_new);
}
// The slot of sequence x, or -1 (the caller flags it).
__device__ __forceinline__ int slot_of(const Pages &p, const Batch &b, int x) {
    const int s = b.seq ? b.seq[x] : b.slot0 + x;
    return (unsigned)s < (unsigned)p.n_slots ? s : -1;
}
// Tokens of a slot, kept inside its table row.
__device__ __forceinline__ int tokens_of(const Pages &p, int slot) {
    const int n = p.n_tokens[slot], most = p.width << p.shift;
    if (n < 0 || n > most) {
        atomicOr(p.status, kStatusBadIndex);
        return n < 0 ? 0 : most;
    }
    return n;
}
// Tokens of sequence x in its slot, for the calls that attend to them: none of one that cache_extend refused (first: its entry is
// negative; NULL: not asked).
__device__ __forceinline__ int tokens_of(const Pages &p, const int *first, int x, int slot) {
    const bool refused = first && first[x] < 0;
    const int n = tokens_of(p, slot);
    return refused ? 0 : n;
}
// A page number from the table: one outside the pool is flagged and read as page 0, so that no address leaves it.
__device__ __forceinline__ int valid_page(const Pages &p, int page) {
    if ((unsigned)page < (unsigned)p.n_pages) return page;
    atomicOr(p.status, kStatusBadIndex);
    return 0;
}

// ---- launchers (sla_cache.cu)
// Scratch of extend, fork and compact, in bytes from the scratch base: ints [n_pages], twice [n_seqs], [kMaxChunks + 1]
constexpr int kMaxChunks = 1024;   // of a pool, to compact
struct CacheScratch {
    size_t off_pages, off_seqs, off_seqs2, off_chunks, bytes;
    Canaries canaries;
};
CacheScratch plan_cache(const Pages &p, int n_seqs, size_t gap = 0);   // gap: bytes of canary between regions
cudaError_t launch_cache_extend(const Pages &p, const Batch &b, int *first, const CacheScratch &s, char *scratch, cudaStream_t st);
cudaError_t launch_cache_append(const Pages &p, const Batch &b, const int *first, const void *k_new, const void *v_new,
                                long long s_t, long long s_h, int sm_count, cudaStream_t st);
cudaError_t launch_cache_release(const Pages &p, const int *seq, int n, cudaStream_t st);
cudaError_t launch_cache_fork(const Pages &p, const int *src, const int *dst, int n, int *pairs, const CacheScratch &s, char *scratch, cudaStream_t st);
cudaError_t launch_cache_compact(const Pages &p, int *pairs, const CacheScratch &s, char *scratch, int sm_count, cudaStream_t st);
cudaError_t launch_cache_copy(const Pages &p, const int *pairs, int n, cudaStream_t st);

// ---- attention over the cache ---------------------------------------------------------------------
// One call of sla_paged_attention.
struct PagedCall {
    Pages c;
    Batch b;
    const int *first;          // of cache_extend, or NULL
    int Hq, G, window;
    long long q_st, q_sh;      // strides of q and out, in elements
    float scale;
    int expire;                // self-test: the CTAs of paged_tiles leave as if their first wait had run out
};

// Whole part of a / b for 0 <= a < 2^53, b > 0: an estimate put right, where a 64-bit division is a hundred instructions, each
// fetched for the first time at the start of a launch.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    long long q = (long long)((float)a / (float)b);
    long long r = a - q * b;
    while (r < 0) { const long long d = max((long long)((float)-r / (float)b), 1ll); q -= d; r += d * b; }
    while (r >= b) { const long long d = max((long long)((float)r / (float)b), 1ll); q += d; r -= d * b; }
    return q;
}
// The ranges of a list: the first `longer` of them have a weight more than `each`.
struct Ranges {
    long long each;
    int count, longer;
    __device__ __forceinline__ long long at(int r) const { return each * r + min(r, longer); }   // where range r begins
    __device__ __forceinline__ int holding(long long p) const {                                 // the range of position p
        const long long head = (each + 1) * longer;
        return (int)(p < head ? quotient(p, each + 1) : longer + quotient(p - head, each));
    }
};

// The work of a call is a list of units -- (sequence, KV head, TQ consecutive new tokens with all G heads of the group) -- each
// with the tiles of KT keys that its tokens see, written down as a running sum of weights (tiles + kUnitWeight, what a unit costs
// beyond its tiles).  The list is cut into equal ranges, wherever that falls: every CTA gets the same share of the keys whatever the
// lengths are.  A unit that is cut leaves partial results, joined by paged_merge.  Where several units read the same keys and these
// are too many for L2, the ranges are a multiple of the CTAs, who go through the list together: each multiple reads kGroupBytes.
// (Not below kGroupWeight a range, where the cuts cost more: 1999 tokens at 30011, three multiples 980 us and one 925 us; 8192 tokens
// that end at 65536, six multiples 6670 us and one 7180 us.  Claimed ranges of falling sizes for CTAs that are done early gave nothing:
// 945 us and 7100 us.)
struct Start;
struct Plan {
    long long *seq_at;    // [n_seqs + 1] weight before sequence x
    int *unit_at;         // [n_seqs + 1] units of one head before sequence x
    long long *unit_end;  // [units] weight up to and with the unit, from the start of its (sequence, head)
    int4 *seqs;           // [n_seqs] slot (-1: none), tokens, new tokens, first row
    Ranges *ranges;
    Start *starts;        // [ranges]
    int max_units, max_ranges;   // room in unit_end and starts
};
constexpr int kUnitWeight = 2;
constexpr long long kGroupBytes = 48ll << 20, kGroupWeight = 400;
// How a kernel cuts a call up: TQ new tokens a unit, tiles of 1 << kt_shift keys.  Units of at most `small` tokens go through two tiles at
// a time (sla_paged_tiles.cu): their tiles weigh half.
struct Shape {
    int TQ, kt_shift, small;
};

// a - b where the difference of a negative position and a large window may not fit: it wraps, and nobody asks for it there, since a
// negative position sees no key.  (max(a, 0) - b costs paged_rows registers: 200 to 333 new tokens of 2 sequences of 2500 to 3000 in fp32
// take 93.3 us with it and 90.9 so.)
__host__ __device__ __forceinline__ int minus(int a, int b) { return (int)((unsigned)a - (unsigned)b); }
// Keys of the new tokens [t0, t1) of a sequence of n tokens, q of them new: tiles [lo, hi) of KT keys.  (A position is negative where the
// sequence is shorter than its new tokens, and the window may be the largest int: their difference is formed only where it is positive.)
__host__ __device__ __forceinline__ void unit_tiles(int n, int q, int t0, int t1, int window, int kt_shift, int &lo, int &hi) {
    const int p0 = n - q + t0, end = n - q + t1;   // first position, one past the last
    const int first = window > 0 && p0 >= window ? p0 - window + 1 : 0;
    lo = first >> kt_shift;
    hi = end > 0 ? (end + (1 << kt_shift) - 1) >> kt_shift : lo;
    if (hi < lo) hi = lo;
}
__device__ __forceinline__ int unit_weight(int n, int q, int t0, int t1, int window, const Shape &f) {
    int lo, hi;
    unit_tiles(n, q, t0, t1, window, f.kt_shift, lo, hi);
    return (t1 - t0 <= f.small ? (hi - lo + 1) >> 1 : hi - lo) + kUnitWeight;
}

// A CTA builds the plan (all threads call it; the arrays are visible to the CTA on return).
template <int kThreads>
__device__ inline void build_plan(const PagedCall &a, const Shape &f, int n_ctas, int max_groups, int min_weight, const Plan &plan,
                                  long long *s_sum) {
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned full = 0xffffffffu;
    // a warp has as few sequences at a time as it can, so that few of them wait for one another; its first ones are on their way at once
    const int per = min(32, (a.b.n_seqs + kWarps - 1) / kWarps);
    auto sequence = [&](int x) {
        int4 s = make_int4(-1, 0, 0, 0);
        if (lane < per && x < a.b.n_seqs) {
            int r1;
            new_rows(a.b, x, s.w, r1);
            s.z = r1 - s.w;
            s.x = slot_of(a.c, a.b, x);
            if (s.x < 0) atomicOr(a.c.status, kStatusBadIndex);
            else s.y = tokens_of(a.c, a.first, x, s.x);
        }
        return s;
    };
    int4 of = sequence(warp * per + lane);
    // units of every sequence (a cu_new that does not ascend could name more than there is room for: those are left out)
    if (warp == 0) {
        int at = 0;
        for (int x0 = 0; x0 < a.b.n_seqs; x0 += 32) {
            const int x = x0 + lane;
            int units = 0;
            if (x < a.b.n_seqs) {
                int lo, hi;
                new_rows(a.b, x, lo, hi);
                units = (hi - lo + f.TQ - 1) / f.TQ;
            }
            long long all = units;
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) all += __shfl_xor_sync(full, all, off);
            if (at + all > plan.max_units) {
                if (lane == 0) atomicOr(a.c.status, kStatusBadIndex);
                units = 0;
            }
            int v = units;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int y = __shfl_up_sync(full, v, off);
                if (lane >= off) v += y;
            }
            if (x < a.b.n_seqs) plan.unit_at[x] = at + v - units;
            at += __shfl_sync(full, v, 31);
        }
        if (lane == 0) plan.unit_at[a.b.n_seqs] = at;
    }
    __syncthreads();
    // weights of a sequence's units: by a lane where one unit is all there is, else by a warp
    long long reread = 0;   // bytes of keys and values that several units read
    for (int x0 = warp * per; x0 < a.b.n_seqs; x0 += kWarps * per) {
        const int x = x0 + lane;
        const bool on = lane < per && x < a.b.n_seqs;
        if (x0 != warp * per) of = sequence(x);
        const int n = of.y, q = of.z, units = on ? plan.unit_at[x + 1] - plan.unit_at[x] : 0;
        if (on) plan.seqs[x] = of;
        long long total = 0;
        if (units == 1) {
            total = unit_weight(n, q, 0, q, a.window, f);
            plan.unit_end[plan.unit_at[x]] = total;
        }
        for (unsigned many = __ballot_sync(full, units > 1); many; many &= many - 1) {
            const int src = __ffs(many) - 1;
            const int u_n = __shfl_sync(full, units, src), qs = __shfl_sync(full, q, src), ns = __shfl_sync(full, n, src);
            const int base = plan.unit_at[x0 + src];
            long long sum = 0;
            for (int u0 = 0; u0 < u_n; u0 += 32) {
                const int u = u0 + lane;
                long long v = u < u_n ? unit_weight(ns, qs, u * f.TQ, min((u + 1) * f.TQ, qs), a.window, f) : 0;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const long long y = __shfl_up_sync(full, v, off);
                    if (lane >= off) v += y;
                }
                if (u < u_n) plan.unit_end[base + u] = sum + v;
                sum += __shfl_sync(full, v, 31);
            }
            if (lane == src) {
                total = sum;
                reread += (long long)n * a.c.Hkv * a.c.D * a.c.es * 2;
            }
        }
        if (on) plan.seq_at[x + 1] = total * a.c.Hkv;
    }
    __syncthreads();
    if (warp == 0) {
        long long at = 0;
        for (int x0 = 0; x0 < a.b.n_seqs; x0 += 32) {
            const int x = x0 + lane;
            long long v = x < a.b.n_seqs ? plan.seq_at[x + 1] : 0;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const long long y = __shfl_up_sync(full, v, off);
                if (lane >= off) v += y;
            }
            if (x < a.b.n_seqs) plan.seq_at[x + 1] = at + v;
            at += __shfl_sync(full, v, 31);
        }
        if (lane == 0) plan.seq_at[0] = 0;
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) reread += __shfl_xor_sync(full, reread, off);
    if (lane == 0) s_sum[warp] = reread;
    __syncthreads();
    if (tid == 0) {
        long long bytes = 0;
        for (int w = 0; w < kWarps; ++w) bytes += s_sum[w];
        const long long total = plan.seq_at[a.b.n_seqs];
        long long groups = 1;
        if (max_groups > 1) {
            const long long most = quotient(total, n_ctas * kGroupWeight);
            groups = quotient(bytes + kGroupBytes - 1, kGroupBytes);
            groups = groups > most ? most : groups;
            groups = groups < 1 ? 1 : groups > max_groups ? max_groups : groups;
        }
        long long n = groups * n_ctas;
        if (n * min_weight > total) n = quotient(total, min_weight);   // a range of a few tiles at least
        if (n < 1) n = total > 0 ? 1 : 0;
        const long long each = n ? quotient(total, n) : 0;
        *plan.ranges = {each, (int)n, (int)(total - each * n)};
    }
    __syncthreads();
}

// Index of the last entry of the ascending a[0 .. n) that is <= v (a[0] <= v); a converged warp, 32 ways a step.
__device__ __forceinline__ int warp_last_le(const long long *a, int n, long long v) {
    const int lane = threadIdx.x & 31;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 31) / 32;
        const bool le = lane * step < n && a[lo + lane * step] <= v;
        const int at = 31 - __clz(__ballot_sync(0xffffffffu, le));
        lo += at * step;
        n = min(step, n - at * step);
    }
    return lo;
}

// The same by a thread alone.
__device__ __forceinline__ int last_le(const long long *a, int n, long long v) {
    int lo = 0;
    while (n > 1) {
        const int half = n / 2;
        const bool le = a[lo + half] <= v;
        lo += le ? half : 0;
        n = le ? n - half : half;
    }
    return lo;
}

// What one CTA does of one unit.
struct Segment {
    int head;                 // KV head
    int slot, n, q;           // cache slot (-1: none), tokens, new tokens
    int t0, t1, row0;         // new tokens of the unit; row of the sequence's first new token
    int lo, hi;               // tiles to attend to
    int all;                  // tiles of the whole unit
    int part;                 // -1: the whole unit; else the partial result's number
};

// The first segment of a range and where its cursor stands behind it.  The plan has them for every range: to find them takes half a dozen
// loads that wait for one another, which the plan has in shared memory.  (Four prompts of 2048 tokens, D 64: 146 us with the search at
// the start of every CTA, 135 so; 1 to 600 tokens of 16 sequences 59.7 and 59.2; calls of 25 to 40 us the same within 2 %.)
struct alignas(16) Start {
    long long w;
    Segment s;
    int last_range, x, unit, units;
};

// Goes through the segments of range r.
struct Cursor {
    Ranges ranges;
    long long w, end;
    int x, head, unit, units, r;

    // the first segment of range r (in w < end); false beyond the last range
    __device__ __forceinline__ bool open(const Plan &plan, int range, Segment &s, int &last_range) {
        ranges = *plan.ranges;
        r = range;
        const Start b = plan.starts[min(r, plan.max_ranges - 1)];   // (both loads at once)
        if (r >= ranges.count) return false;
        end = ranges.at(r + 1);
        w = b.w; s = b.s; last_range = b.last_range;
        x = b.x; unit = b.unit; units = b.units; head = b.s.head;
        return true;
    }
    // puts the cursor in front of it
    __device__ __forceinline__ void seek(const PagedCall &a, const Plan &plan, const Ranges &of, int range) {
        ranges = of;
        r = range;
        w = ranges.at(r);
        end = ranges.at(r + 1);
        x = last_le(plan.seq_at, a.b.n_seqs, w);
        units = plan.unit_at[x + 1] - plan.unit_at[x];
        const long long *ue = plan.unit_end + plan.unit_at[x];
        const long long rem = w - plan.seq_at[x], per_head = ue[units - 1];
        head = (int)quotient(rem, per_head);
        const long long in = rem - head * per_head;
        unit = ue[0] > in ? 0 : last_le(ue, units, in) + 1;
    }
    // the segment at the cursor; false when the range is done.  *last_range: for a unit that starts in this range and does not
    // end in it, the range it ends in, else -1.
    __device__ __forceinline__ bool next(const PagedCall &a, const Plan &plan, const Shape &f, Segment &s, int &last_range) {
        last_range = -1;
        if (w >= end) return false;
        if (unit == units) {
            unit = 0;
            if (++head == a.c.Hkv) {
                head = 0;
                do ++x; while (plan.unit_at[x + 1] == plan.unit_at[x]);
                units = plan.unit_at[x + 1] - plan.unit_at[x];
            }
        }
        const long long *ue = plan.unit_end + plan.unit_at[x];
        const long long u1 = ue[unit], u0 = unit ? ue[unit - 1] : 0;
        const long long start = plan.seq_at[x] + head * ue[units - 1] + u0, stop = start + (u1 - u0);
        s.head = head;
        const int4 of = plan.seqs[x];
        s.slot = of.x; s.n = of.y; s.q = of.z; s.row0 = of.w;
        s.t0 = unit * f.TQ;
        s.t1 = min(s.t0 + f.TQ, s.q);
        int lo, hi;
        unit_tiles(s.n, s.q, s.t0, s.t1, a.window, f.kt_shift, lo, hi);
        const int per = s.t1 - s.t0 <= f.small ? 2 : 1;   // tiles of a weight
        const int from = (int)(w - start), to = (int)((end < stop ? end : stop) - start);   // weights of the unit in this range
        s.lo = min(lo + per * max(from - kUnitWeight, 0), hi);
        s.hi = min(lo + per * max(to - kUnitWeight, 0), hi);
        s.all = hi - lo;
        const bool begins = from == 0, ends = end >= stop;
        s.part = begins && ends ? -1 : begins ? 2 * r + 1 : 2 * r;
        if (begins && !ends) last_range = ranges.holding(stop - 1);
        w = end < stop ? end : stop;
        ++unit;
        return true;
    }
};

// The unit that starts in a range and ends in the range `last` (-1 where none does): its first row, tokens and KV head.
struct alignas(16) Cut {
    int row0, tokens, head, last;
};
// Partial results: part p of a unit of R rows has its normalised sums at o + p * R * D and its log2-sum-exp at lse2 + p * R (-inf: no
// keys; the sums are then not written).  Eight columns of all rows lie together, row by row: where a thread has a row, the threads of a
// warp write and read 1 KB on end.  (sla_paged_decode.cu joins its own parts and has them as [R, D].)
struct Parts {
    float *o, *lse2;
    Cut *cut;             // [ranges]
    __device__ __forceinline__ float *at(int part, int R, int D, int row, int d) const { return o + (long long)part * R * D + ((d >> 3) * R + row) * 8 + (d & 7); }
};

}  // namespace sla
