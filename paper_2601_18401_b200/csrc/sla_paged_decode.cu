// Attention of few new tokens a sequence over a paged cache (sla_paged_decode.cuh): the choice of the kernel, and the kernels over rows of bf16 and fp32.
#include "sla_paged_decode.cuh"

namespace sla {

bool paged_decode_supported(const PagedCall &a) { return (long long)a.b.max_new * a.G <= 16; }

void plan_paged_decode(const PagedCall &a, PagedPlan &p, int sm_count) {
    p.R = p.RS = 16;
    p.TS = p.TQ = 1;
    p.n_ctas = ctas_per_sm(a.c.D, a.b.max_new * a.G <= 8 ? 1 : 2, q4::is(a.c)) * sm_count;
}

cudaError_t launch_paged_decode_attention(const void *q, const PagedCall &a, int dtype, const PagedPlan &p, char *scratch, int *counters, void *out,
                                          float *lse, cudaStream_t st, long long *launches) {
    if (q4::is(a.c)) return launch_paged_decode_q4(q, a, dtype, p, scratch, counters, out, lse, st, launches);
    if (dtype == SLA_F32)
        return a.c.D == 64 ? decode_for<float, 64, false>(q, a, p, scratch, counters, out, lse, st, launches) : decode_for<float, 128, false>(q, a, p, scratch, counters, out, lse, st, launches);
    return a.c.D == 64 ? decode_for<__nv_bfloat16, 64, false>(q, a, p, scratch, counters, out, lse, st, launches)
                       : decode_for<__nv_bfloat16, 128, false>(q, a, p, scratch, counters, out, lse, st, launches);
}

}  // namespace sla
