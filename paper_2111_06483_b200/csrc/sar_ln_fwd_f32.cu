#include "sar_ln.cuh"

namespace sar {
sar_status ln_forward_f32(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st) {
    return ckpt ? ln_forward_of<float, true>(s, a, st) : ln_forward_of<float, false>(s, a, st);
}
}  // namespace sar
