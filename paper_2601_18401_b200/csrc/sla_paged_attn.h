// Internal launcher declarations of the attention over a paged cache.
#pragma once

#include "sla_kernels.h"
#include "sla_paged.cuh"

namespace sla {

// Tiles and scratch layout of one call (offsets in bytes from the scratch base).
struct PagedPlan {
    enum Kind { kRows, kDecode, kTiles } kind;
    int R, RS, TS, TQ;      // rows of a unit, rows and tokens of its sub-tiles, tokens of the unit
    int kt_shift;           // log2 of the keys of a tile
    int small;              // tokens of a unit whose tiles weigh half
    int n_ctas, max_groups, min_weight, max_units, max_ranges;
    size_t off_seq_at, off_unit_at, off_unit_end, off_ranges, off_seqs, off_starts, off_cut, off_lse2, off_o, off_fold, bytes;
    size_t fold_bytes;      // sums of O beside TMEM (sla_paged_tiles.cu)
    Canaries canaries;
};

inline Plan plan_at(const PagedPlan &p, char *scratch) {
    return {reinterpret_cast<long long *>(scratch + p.off_seq_at), reinterpret_cast<int *>(scratch + p.off_unit_at),
            reinterpret_cast<long long *>(scratch + p.off_unit_end), reinterpret_cast<int4 *>(scratch + p.off_seqs),
            reinterpret_cast<Ranges *>(scratch + p.off_ranges), reinterpret_cast<Start *>(scratch + p.off_starts), p.max_units, p.max_ranges};
}
inline Parts parts_at(const PagedPlan &p, char *scratch) {
    return {reinterpret_cast<float *>(scratch + p.off_o), reinterpret_cast<float *>(scratch + p.off_lse2),
            reinterpret_cast<Cut *>(scratch + p.off_cut)};
}

PagedPlan plan_paged(const PagedCall &a, int dtype, int sm_count, size_t gap = 0);   // gap: bytes of canary between regions
cudaError_t launch_paged_plan(const PagedCall &a, const PagedPlan &p, char *scratch, cudaStream_t st);
cudaError_t launch_paged_merge(const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st);
// counters: p.n_ctas ints, zero on entry and again on exit
cudaError_t launch_paged_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                   float *lse, cudaStream_t st, long long *launches);

// ---- one new token a sequence (sla_paged_decode.cu)
bool paged_decode_supported(const PagedCall &a);
void plan_paged_decode(const PagedCall &a, PagedPlan &p, int sm_count);
cudaError_t launch_paged_decode_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                          float *lse, cudaStream_t st, long long *launches);

// ---- chunks of new tokens, bf16 (sla_paged_tiles.cu)
bool paged_tiles_supported(const PagedCall &a, int dtype);
void plan_paged_tiles(const PagedCall &a, PagedPlan &p, int sm_count);
cudaError_t launch_paged_tiles(const void *q, const PagedCall &a, const PagedPlan &p, char *scratch, void *out, float *lse, cudaStream_t st);

}  // namespace sla
