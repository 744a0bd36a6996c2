// Checkpoints of node arrays in 8 bits: x[n, C] -> codes and block scales, and back (include/sar.h has the format and the
// contracts).  Each is one pass over its arrays.  Whole blocks are counted through the array here, whatever the rows; rows whose last
// block is short go row by row through the layer normalisation's kernels, without a division for every block (a million rows
// of 100, us, here and by rows: float32 packed 108 and 101, unpacked 125 and 87; bf16 97 and 95, 106 and 68; of 72 bf16 70 and 44, 54
// and 43), unless they are longer than a block's registers.
#include "sar_ckpt8.cuh"
#include "sar_ln.cuh"

#include <type_traits>

namespace sar {

// Division by the blocks of a row, as a product: exact for numerators below 2^31 (q = (n * ceil(2^(31 + l) / d)) >> (31 + l) with
// l = ceil(log2 d): the product's excess is below n / 2^31 of a unit).
struct RowDivide {
    unsigned long long mul;
    int shift;
    int d;
};
static RowDivide row_divide(int d) {
    int l = 0;
    while ((1ll << l) < d) ++l;
    return {((1ull << (31 + l)) + d - 1) / d, 31 + l, d};
}

// A block's 32 columns are S slots of E columns for each of LPB = 32 / (E S) consecutive threads: slot i of thread `sub` starts at
// column (i LPB + sub) E of the block, E being 8 bf16 (16 bytes), 4 of either type, or one column for rows that allow no more.  Several
// slots rather than more threads: a block's maximum is then joined in 2 or 3 steps.  Rows whose columns are no multiple of 32 end in a
// shorter block, where some slots have no columns; with whole blocks the rows do not matter and the blocks are counted through.
template <typename T, int E, int S>
struct CkptBlock {
    using Vec = ColVec<T, E>;
    using raw_t = typename Vec::type;
    static constexpr int P = (E + 1) / 2, LPB = kCkptBlock / (E * S);
    long long at;   // flat index of the thread's first slot
    int left;       // columns from there to the end of the row or the block; none for a block behind the last
    __device__ __forceinline__ CkptBlock(long long b, long long blocks, int sub, int C, const RowDivide &nb, bool whole) {
        if (whole) {
            at = b * kCkptBlock + sub * E;
            left = kCkptBlock - sub * E;
        } else {
            const long long row = b < (1ll << 31) ? (long long)((unsigned long long)b * nb.mul >> nb.shift) : b / nb.d;
            const int col = (int)(b - row * nb.d) * kCkptBlock + sub * E;
            at = row * C + col;
            left = C - col;
        }
        if (b >= blocks) left = 0;
    }
    // E divides C: a slot has all its columns or none
    __device__ __forceinline__ bool ok(int i) const { return i * LPB * E < left; }
    __device__ __forceinline__ long long slot(int i) const { return at + i * LPB * E; }
};

// Each thread asks for its columns of several blocks before it uses the first: 64 bytes in flight of x, 32 of codes.
template <int BYTES, int E, int S>
constexpr int ckpt_ahead = BYTES == 1 ? (32 / (E * S) < 4 ? 4 : 32 / (E * S)) : 64 / (E * S * BYTES) < 1 ? 1 : 64 / (E * S * BYTES) > 4 ? 4 : 64 / (E * S * BYTES);

template <typename T, int E, int S>
__global__ void __launch_bounds__(256, 4) ckpt8_pack_kernel(long long blocks, int C, RowDivide nb, const T *__restrict__ x, int8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales) {
    after_predecessor();
    using B = CkptBlock<T, E, S>;
    constexpr int P = B::P, LPB = B::LPB, U = ckpt_ahead<sizeof(T), E, S>;
    const int sub = threadIdx.x % LPB;
    const bool whole = C == nb.d * kCkptBlock;
    // b0: the warp's first block, the same for all its lanes (the shuffles need every lane); a warp's blocks follow one another
    const long long stride = (long long)gridDim.x * (256 / LPB) * U;
    for (long long b0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (32 / LPB) * U; b0 < blocks; b0 += stride) {
        typename B::raw_t raw[U][S];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const B p(b0 + u * (32 / LPB) + (threadIdx.x & 31) / LPB, blocks, sub, C, nb, whole);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                raw[u][i] = typename B::raw_t{};
                if (p.ok(i)) raw[u][i] = __ldg(reinterpret_cast<const typename B::raw_t *>(x + p.slot(i)));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long b = b0 + u * (32 / LPB) + (threadIdx.x & 31) / LPB;
            const B p(b, blocks, sub, C, nb, whole);
            float2 v[S][P];
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                B::Vec::get(raw[u][i], v[i]);
#pragma unroll
                for (int q = 0; q < P; ++q) top = ckpt_top(top, v[i][q].x, v[i][q].y);
            }
#pragma unroll
            for (int d = 1; d < LPB; d <<= 1) top = ckpt_top(top, __shfl_xor_sync(0xffffffffu, top, d), 0.f);
            const float inv = ckpt_inverse(top);
            const bool bad = ckpt_bad(top), cut = __any_sync(0xffffffffu, ckpt_cut(top, inv));
#pragma unroll
            for (int i = 0; i < S; ++i) {
                if (!p.ok(i)) continue;
                int8_t *to = codes + p.slot(i);
                if constexpr (E == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(ckpt_code4(v[i][0], v[i][1], inv, bad, cut), ckpt_code4(v[i][2], v[i][3], inv, bad, cut));
                else if constexpr (E == 4) *reinterpret_cast<unsigned *>(to) = ckpt_code4(v[i][0], v[i][1], inv, bad, cut);
                else *to = ckpt_code1(v[i][0].x, inv, bad, cut);
            }
            if (sub == 0 && b < blocks) scales[b] = (uint8_t)ckpt_scale_byte(top);
        }
    }
}

template <typename T, int E, int S>
__global__ void __launch_bounds__(256, 4) ckpt8_unpack_kernel(long long blocks, int C, RowDivide nb, const int8_t *__restrict__ codes,
                                                              const uint8_t *__restrict__ scales, T *__restrict__ x) {
    after_predecessor();
    using B = CkptBlock<T, E, S>;
    using W = typename std::conditional<E == 8, uint2, typename std::conditional<E == 4, unsigned, signed char>::type>::type;
    constexpr int P = B::P, LPB = B::LPB, U = ckpt_ahead<1, E, S>;
    const int sub = threadIdx.x % LPB;
    const bool whole = C == nb.d * kCkptBlock;
    const long long stride = (long long)gridDim.x * (256 / LPB) * U;
    for (long long b0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (32 / LPB) * U + (threadIdx.x & 31) / LPB; b0 < blocks; b0 += stride) {
        W raw[U][S];
        unsigned s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long b = b0 + u * (32 / LPB);
            const B p(b, blocks, sub, C, nb, whole);
            s[u] = b < blocks ? __ldg(scales + b) : 0u;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                raw[u][i] = W{};
                if (p.ok(i)) raw[u][i] = __ldg(reinterpret_cast<const W *>(codes + p.slot(i)));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const B p(b0 + u * (32 / LPB), blocks, sub, C, nb, whole);
            const float scale = ckpt_scale(s[u]);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                if (!p.ok(i)) continue;
                float2 v[P];
                if constexpr (E == 1) {
                    v[0] = make_float2((float)raw[u][i] * scale, 0.f);
                } else {
                    unsigned w[2];
                    memcpy(w, &raw[u][i], E);
#pragma unroll
                    for (int q = 0; q < P; ++q) v[q] = ckpt_decode2(w[q / 2] ^ 0x80808080u, 2 * q & 3, make_float2(scale, scale));
                }
                *reinterpret_cast<typename B::raw_t *>(x + p.slot(i)) = B::Vec::put(v);
            }
        }
    }
}

// columns per access for these sizes and addresses
static int ckpt_width(int32_t C, sar_dtype t, const void *x, const void *codes) {
    const size_t es = sar_elem_size(t);
    for (int e : {8, 4})
        if (e * es <= 16 && C % e == 0 && sar_aligned(x, e * es) && sar_aligned(codes, e)) return e;
    return 1;
}

template <typename T, typename Fn>
static sar_status ckpt_dispatch(int e, Fn &&f) {
    if constexpr (sizeof(T) == 2) {
        if (e == 8) return f(Cfg<T, 8, 1, 0>{});
    }
    if (e == 4) return f(Cfg<T, 4, 2, 0>{});
    return f(Cfg<T, 1, 4, 0>{});
}

static sar_status ckpt_check(int64_t n, int32_t C, sar_dtype t, const void *x, const void *codes, const void *scales) {
    if (n < 0 || C < 1 || (t != SAR_F32 && t != SAR_BF16)) return SAR_ERR_INVALID_ARG;
    if (C > (1 << 20)) return SAR_ERR_UNSUPPORTED;
    if (n > 0 && (!x || !codes || !scales)) return SAR_ERR_INVALID_ARG;
    return check_elem_align({x}, sar_elem_size(t));
}

// blocks of 256 threads for so many blocks of columns, per warp and step `per`: as many as run at once walk the array
static unsigned ckpt_grid(long long blocks, int per) {
    const long long want = (blocks + 8ll * per - 1) / (8ll * per);
    return (unsigned)(want < 148 * 4 ? want : 148 * 4);
}

}  // namespace sar

using namespace sar;

extern "C" {

sar_status sar_ckpt8_pack(int64_t n, int32_t C, sar_dtype t, const void *x, int8_t *codes, uint8_t *scales, void *stream) {
    SAR_TRY(ckpt_check(n, C, t, x, codes, scales));
    if (n == 0) return SAR_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LnShape s = ln_shape(C, t, kLnPack, ln_alignment({x}), ln_alignment({codes}));
    if (C % kCkptBlock != 0 && s.E > 0) {
        LnArgs a = ln_args(n, C);
        a.x = x;
        a.codes = codes;
        a.scales = scales;
        return (t == SAR_F32 ? ln_checkpoint_f32 : ln_checkpoint_bf16)(s, a, false, st);
    }
    const int nb = (int)ckpt_blocks(C), e = ckpt_width(C, t, x, codes);
    const long long blocks = n * nb;
    auto go = [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        using T = typename K::type;
        SAR_LAUNCH("ckpt8_pack", st, launch_if(n * C <= kOverlapElems, ckpt8_pack_kernel<T, K::g, K::v>, ckpt_grid(blocks, K::g * K::v * ckpt_ahead<sizeof(T), K::g, K::v>), 256, 0, st,
                                               blocks, C, row_divide(nb), static_cast<const T *>(x), codes, scales));
        return sar_after_launch();
    };
    return t == SAR_F32 ? ckpt_dispatch<float>(e, go) : ckpt_dispatch<__nv_bfloat16>(e, go);
}

sar_status sar_ckpt8_unpack(int64_t n, int32_t C, sar_dtype t, const int8_t *codes, const uint8_t *scales, void *x, void *stream) {
    SAR_TRY(ckpt_check(n, C, t, x, codes, scales));
    if (n == 0) return SAR_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LnShape s = ln_shape(C, t, kLnCkpt, ln_alignment({x}), ln_alignment({codes}));
    if (C % kCkptBlock != 0 && s.E > 0) {
        LnArgs a = ln_args(n, C);
        a.y = x;
        a.codes = const_cast<int8_t *>(codes);
        a.scales = const_cast<uint8_t *>(scales);
        return (t == SAR_F32 ? ln_checkpoint_f32 : ln_checkpoint_bf16)(s, a, true, st);
    }
    const int nb = (int)ckpt_blocks(C), e = ckpt_width(C, t, x, codes);
    const long long blocks = n * nb;
    auto go = [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        using T = typename K::type;
        SAR_LAUNCH("ckpt8_unpack", st, launch_if(n * C <= kOverlapElems, ckpt8_unpack_kernel<T, K::g, K::v>, ckpt_grid(blocks, K::g * K::v * ckpt_ahead<1, K::g, K::v>), 256, 0, st,
                                                 blocks, C, row_divide(nb), codes, scales, static_cast<T *>(x)));
        return sar_after_launch();
    };
    return t == SAR_F32 ? ckpt_dispatch<float>(e, go) : ckpt_dispatch<__nv_bfloat16>(e, go);
}

}  // extern "C"
