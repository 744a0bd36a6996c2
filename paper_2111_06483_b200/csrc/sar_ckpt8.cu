// Checkpoints of node arrays in 8 bits: x[n, C] -> codes and block scales, and back (include/sar.h has the format and the
// contracts).  Each is one pass over its arrays; nothing is computed that memory would wait for.
#include "sar_ckpt8.cuh"
#include "sar_dispatch.cuh"

namespace sar {

// EPT columns a thread (8, 4 or 1), so 32 / EPT consecutive threads a block of 32 columns: a thread's share is one or two
// 16-byte vectors (8 bytes for 4 bf16) and EPT codes.  Rows whose columns are no multiple of 32 end in a shorter block, whose
// last threads have no columns; with whole blocks the rows do not matter and the blocks are counted through.
template <typename T, int EPT>
struct CkptVec;
template <int EPT>
struct CkptVec<float, EPT> {
    __device__ __forceinline__ static void load(const float *p, float (&x)[EPT]) {
        if constexpr (EPT >= 4) {
#pragma unroll
            for (int q = 0; q < EPT / 4; ++q) {
                const float4 v = __ldg(reinterpret_cast<const float4 *>(p) + q);
                x[4 * q] = v.x, x[4 * q + 1] = v.y, x[4 * q + 2] = v.z, x[4 * q + 3] = v.w;
            }
        } else {
            x[0] = __ldg(p);
        }
    }
    __device__ __forceinline__ static void store(float *p, const float (&x)[EPT]) {
        if constexpr (EPT >= 4) {
#pragma unroll
            for (int q = 0; q < EPT / 4; ++q) reinterpret_cast<float4 *>(p)[q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
        } else {
            *p = x[0];
        }
    }
};
template <int EPT>
struct CkptVec<__nv_bfloat16, EPT> {
    using E = Elem<__nv_bfloat16>;
    __device__ __forceinline__ static void load(const __nv_bfloat16 *p, float (&x)[EPT]) {
        if constexpr (EPT == 8) {
            E::unpack(__ldg(reinterpret_cast<const uint4 *>(p)), x);
        } else if constexpr (EPT == 4) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
            x[0] = __uint_as_float(v.x << 16), x[1] = __uint_as_float(v.x & 0xffff0000u);
            x[2] = __uint_as_float(v.y << 16), x[3] = __uint_as_float(v.y & 0xffff0000u);
        } else {
            x[0] = E::load1(p);
        }
    }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float (&x)[EPT]) {
        if constexpr (EPT == 8) *reinterpret_cast<uint4 *>(p) = E::pack(x);
        else if constexpr (EPT == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(E::pack2(x[0], x[1]), E::pack2(x[2], x[3]));
        else E::store1(p, x[0]);
    }
};
template <int EPT>
__device__ __forceinline__ void store_codes(int8_t *p, const float (&x)[EPT], float inverse, unsigned s) {
    if constexpr (EPT == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(ckpt_code4(x, inverse, s), ckpt_code4(x + 4, inverse, s));
    else if constexpr (EPT == 4) *reinterpret_cast<unsigned *>(p) = ckpt_code4(x, inverse, s);
    else *p = (int8_t)(s == 255u ? 0u : ckpt_code(x[0], inverse));
}
template <int EPT>
__device__ __forceinline__ void load_codes(const int8_t *p, float scale, float (&x)[EPT]) {
    if constexpr (EPT == 8) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
        const unsigned w[2] = {v.x, v.y};
        ckpt_decode_n<8>(w, scale, x);
    } else if constexpr (EPT == 4) {
        const unsigned w[1] = {__ldg(reinterpret_cast<const unsigned *>(p))};
        ckpt_decode_n<4>(w, scale, x);
    } else {
        x[0] = (float)__ldg(reinterpret_cast<const signed char *>(p)) * scale;
    }
}

// where a thread's columns lie: block b of the array, `at` the flat index of the thread's first column
struct CkptPlace {
    long long at;
    bool some;   // the thread has columns in this block
};
template <int EPT>
__device__ __forceinline__ CkptPlace ckpt_place(long long b, int sub, int C, int nb, bool whole) {
    if (whole) return {b * kCkptBlock + sub * EPT, true};
    long long row;
    int blk;
    if (b < (1ll << 31)) {   // a 32-bit division is a third of a 64-bit one
        row = (unsigned)b / (unsigned)nb;
        blk = (int)((unsigned)b - (unsigned)row * (unsigned)nb);
    } else {
        row = b / nb;
        blk = (int)(b - row * nb);
    }
    const int col = blk * kCkptBlock + sub * EPT;
    return {row * C + col, col < C};   // EPT divides C: a thread has all its columns or none
}

template <typename T, int EPT>
__global__ void __launch_bounds__(256) ckpt8_pack_kernel(long long blocks, int C, int nb, const T *__restrict__ x, int8_t *__restrict__ codes,
                                                         uint8_t *__restrict__ scales) {
    after_predecessor();
    constexpr int LPB = kCkptBlock / EPT;
    const long long stride = (long long)gridDim.x * (256 / LPB);
    const int sub = threadIdx.x % LPB;
    const bool whole = C == nb * kCkptBlock;
    // a warp's blocks all lie before the end or the warp takes this step as a whole: the shuffles need every lane
    for (long long b0 = (long long)blockIdx.x * (256 / LPB) + (threadIdx.x & ~31) / LPB; b0 < blocks; b0 += stride) {
        const long long b = b0 + (threadIdx.x & 31) / LPB;
        CkptPlace p = ckpt_place<EPT>(b, sub, C, nb, whole);
        p.some = p.some && b < blocks;
        float v[EPT];
#pragma unroll
        for (int i = 0; i < EPT; ++i) v[i] = 0.f;
        if (p.some) CkptVec<T, EPT>::load(x + p.at, v);
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < EPT; ++i) top = max(top, ckpt_magnitude(v[i]));
#pragma unroll
        for (int d = 1; d < LPB; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const unsigned s = ckpt_scale_byte(top);
        if (p.some) store_codes<EPT>(codes + p.at, v, ckpt_inverse(s), s);
        if (sub == 0 && b < blocks) scales[b] = (uint8_t)s;
    }
}

template <typename T, int EPT>
__global__ void __launch_bounds__(256) ckpt8_unpack_kernel(long long blocks, int C, int nb, const int8_t *__restrict__ codes,
                                                           const uint8_t *__restrict__ scales, T *__restrict__ x) {
    after_predecessor();
    constexpr int LPB = kCkptBlock / EPT;
    const long long stride = (long long)gridDim.x * (256 / LPB);
    const int sub = threadIdx.x % LPB;
    const bool whole = C == nb * kCkptBlock;
    for (long long b = (long long)blockIdx.x * (256 / LPB) + threadIdx.x / LPB; b < blocks; b += stride) {
        const CkptPlace p = ckpt_place<EPT>(b, sub, C, nb, whole);
        if (!p.some) continue;
        float v[EPT];
        load_codes<EPT>(codes + p.at, ckpt_scale(__ldg(scales + b)), v);
        CkptVec<T, EPT>::store(x + p.at, v);
    }
}

// columns per thread for these sizes and addresses
static int ckpt_ept(int32_t C, sar_dtype t, const void *x, const void *codes) {
    const size_t es = sar_elem_size(t);
    for (int ept : {8, 4})
        if (C % ept == 0 && sar_aligned(x, ept * es < 16 ? ept * es : 16) && sar_aligned(codes, ept)) return ept;
    return 1;
}

template <typename T, typename Fn>
static sar_status ckpt_launch(int ept, Fn &&f) {
    if (ept == 8) return f(Cfg<T, 8, 0, 0>{});
    if (ept == 4) return f(Cfg<T, 4, 0, 0>{});
    return f(Cfg<T, 1, 0, 0>{});
}

static sar_status ckpt_check(int64_t n, int32_t C, sar_dtype t, const void *x, const void *codes, const void *scales) {
    if (n < 0 || C < 1 || (t != SAR_F32 && t != SAR_BF16)) return SAR_ERR_INVALID_ARG;
    if (C > (1 << 20)) return SAR_ERR_UNSUPPORTED;
    if (n > 0 && (!x || !codes || !scales)) return SAR_ERR_INVALID_ARG;
    return check_elem_align({x}, sar_elem_size(t));
}

static unsigned ckpt_grid(long long blocks, int ept) {
    const long long per = 256 / (kCkptBlock / ept), want = (blocks + per - 1) / per;
    return (unsigned)(want < 148 * 64 ? want : 148 * 64);
}

}  // namespace sar

using namespace sar;

extern "C" {

sar_status sar_ckpt8_pack(int64_t n, int32_t C, sar_dtype t, const void *x, int8_t *codes, uint8_t *scales, void *stream) {
    SAR_TRY(ckpt_check(n, C, t, x, codes, scales));
    if (n == 0) return SAR_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int nb = (int)ckpt_blocks(C), ept = ckpt_ept(C, t, x, codes);
    const long long blocks = n * nb;
    auto go = [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        using T = typename K::type;
        SAR_LAUNCH("ckpt8_pack", st, launch_if(n * C <= kOverlapElems, ckpt8_pack_kernel<T, K::g>, ckpt_grid(blocks, ept), 256, 0, st, blocks, C, nb,
                                               static_cast<const T *>(x), codes, scales));
        return sar_after_launch();
    };
    return t == SAR_F32 ? ckpt_launch<float>(ept, go) : ckpt_launch<__nv_bfloat16>(ept, go);
}

sar_status sar_ckpt8_unpack(int64_t n, int32_t C, sar_dtype t, const int8_t *codes, const uint8_t *scales, void *x, void *stream) {
    SAR_TRY(ckpt_check(n, C, t, x, codes, scales));
    if (n == 0) return SAR_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int nb = (int)ckpt_blocks(C), ept = ckpt_ept(C, t, x, codes);
    const long long blocks = n * nb;
    auto go = [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        using T = typename K::type;
        SAR_LAUNCH("ckpt8_unpack", st, launch_if(n * C <= kOverlapElems, ckpt8_unpack_kernel<T, K::g>, ckpt_grid(blocks, ept), 256, 0, st, blocks, C, nb,
                                                 codes, scales, static_cast<T *>(x)));
        return sar_after_launch();
    };
    return t == SAR_F32 ? ckpt_launch<float>(ept, go) : ckpt_launch<__nv_bfloat16>(ept, go);
}

}  // extern "C"
