#include "sar_ln.cuh"

namespace sar {
sar_status ln_forward_bf16(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st) {
    return ckpt ? ln_forward_of<__nv_bfloat16, true>(s, a, st) : ln_forward_of<__nv_bfloat16, false>(s, a, st);
}
}  // namespace sar
