#include "sar_ln.cuh"

namespace sar {
sar_status ln_backward_grouped_bf16(const LnShape &s, const LnArgs &a, bool ckpt, unsigned *records, cudaStream_t st) {
    return ckpt ? ln_backward_of<__nv_bfloat16, true, true>(s, a, records, st) : ln_backward_of<__nv_bfloat16, false, true>(s, a, records, st);
}
}  // namespace sar
