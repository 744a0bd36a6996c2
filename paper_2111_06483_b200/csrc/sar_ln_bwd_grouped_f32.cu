#include "sar_ln.cuh"

namespace sar {
sar_status ln_backward_grouped_f32(const LnShape &s, const LnGroupedArgs &a, bool ckpt, unsigned *records, cudaStream_t st) {
    return ckpt ? ln_backward_of<float, true>(s, a, records, st) : ln_backward_of<float, false>(s, a, records, st);
}
}  // namespace sar
