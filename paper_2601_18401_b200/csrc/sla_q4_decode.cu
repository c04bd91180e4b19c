// Attention of few new tokens a sequence over a paged cache in four bits: the kernels of sla_paged_decode.cuh.
#include "sla_paged_decode.cuh"

namespace sla {

cudaError_t launch_paged_decode_q4(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                   float *lse, cudaStream_t st, long long *launches) {
    if (dtype == SLA_F32)
        return a.c.D == 64 ? decode_for<float, 64, true>(q, a, p, scratch, counters, out, lse, st, launches) : decode_for<float, 128, true>(q, a, p, scratch, counters, out, lse, st, launches);
    return a.c.D == 64 ? decode_for<__nv_bfloat16, 64, true>(q, a, p, scratch, counters, out, lse, st, launches)
                       : decode_for<__nv_bfloat16, 128, true>(q, a, p, scratch, counters, out, lse, st, launches);
}

}  // namespace sla
