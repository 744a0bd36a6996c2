#include "sar_ln.cuh"

namespace sar {
sar_status ln_checkpoint_bf16(const LnShape &s, const LnArgs &a, bool unpack, cudaStream_t st) {
    return ln_dispatch<__nv_bfloat16, kLnCkpt>(s, [&](auto cfg) -> sar_status {
        using Row = typename decltype(cfg)::row;
        if (unpack) {
            static const unsigned most = ln_resident(ln_unpack_kernel<Row>, 0);
            return ln_launch("ckpt8_unpack", ln_unpack_kernel<Row>, ln_grid<Row::G>(a.n), most, 0, a, st);
        }
        if constexpr (Row::kShifted && Row::E * Row::G * Row::V <= kPackShiftedFrom) {
            return SAR_ERR_UNSUPPORTED;   // shapes of narrower rows than are packed shifted
        } else {
            static const unsigned most = ln_resident(ln_pack_kernel<Row>, 0);
            return ln_launch("ckpt8_pack", ln_pack_kernel<Row>, ln_grid<Row::G>(a.n), most, 0, a, st);
        }
    });
}
}  // namespace sar
