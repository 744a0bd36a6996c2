// Activation checkpoints in 8 bits (internal): how a block of 32 columns is held, shared by the kernels that write checkpoints
// and those that read them.  The format is in include/sar.h.
//
// The scale of a block is a power of two.  So x / scale is exact, the code is the one rounding of the format, and every kernel
// that packs the same values gives the same bytes; and code * scale has at most 7 significant bits, so it is exact in bf16 and
// the tensor cores take it as it is.  What a free scale (max / 127) would gain is at most one bit: with E = floor(log2(max))
// the step is 2^(E-6), max / 127 to max / 63.5.
#pragma once

#include "sar_common.cuh"
#include "sar_device.cuh"

namespace sar {

// E consecutive columns of a row of type T in one access, as pairs of float32
template <typename T, int E>
struct ColVec;
template <>
struct ColVec<float, 4> {
    using type = float4;
    __device__ __forceinline__ static void get(const float4 &r, float2 (&x)[2]) { x[0] = make_float2(r.x, r.y), x[1] = make_float2(r.z, r.w); }
    __device__ __forceinline__ static float4 put(const float2 (&x)[2]) { return make_float4(x[0].x, x[0].y, x[1].x, x[1].y); }
};
template <>
struct ColVec<__nv_bfloat16, 8> {
    using type = uint4;
    __device__ __forceinline__ static void get(const uint4 &r, float2 (&x)[4]) { Pairs<__nv_bfloat16>::get(r, x); }
    __device__ __forceinline__ static uint4 put(const float2 (&x)[4]) {
        using B = Elem<__nv_bfloat16>;
        return make_uint4(B::pack2(x[0].x, x[0].y), B::pack2(x[1].x, x[1].y), B::pack2(x[2].x, x[2].y), B::pack2(x[3].x, x[3].y));
    }
};
template <>
struct ColVec<__nv_bfloat16, 4> {
    using type = uint2;
    __device__ __forceinline__ static void get(const uint2 &r, float2 (&x)[2]) {
        x[0] = make_float2(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u));
        x[1] = make_float2(__uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
    }
    __device__ __forceinline__ static uint2 put(const float2 (&x)[2]) {
        using B = Elem<__nv_bfloat16>;
        return make_uint2(B::pack2(x[0].x, x[0].y), B::pack2(x[1].x, x[1].y));
    }
};
template <>   // one column: the second of the pair is zero throughout
struct ColVec<float, 1> {
    using type = float;
    __device__ __forceinline__ static void get(float r, float2 (&x)[1]) { x[0] = make_float2(r, 0.f); }
    __device__ __forceinline__ static float put(const float2 (&x)[1]) { return x[0].x; }
};
template <>
struct ColVec<__nv_bfloat16, 1> {
    using type = unsigned short;
    __device__ __forceinline__ static void get(unsigned short r, float2 (&x)[1]) { x[0] = make_float2(__uint_as_float((unsigned)r << 16), 0.f); }
    __device__ __forceinline__ static unsigned short put(const float2 (&x)[1]) { return __bfloat16_as_ushort(__float2bfloat16_rn(x[0].x)); }
};

constexpr int kCkptBlock = SAR_CKPT8_BLOCK;   // columns that share a scale

// the largest magnitude so far and of two more values; NaN where any of them is (a plain maximum would drop it)
__device__ __forceinline__ float ckpt_top(float top, float a, float b) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(top), "f"(a), "f"(b));
    return r;
}

// the scale byte of a block whose largest magnitude is `top`: 0 all zero, 255 anything infinite or NaN, else
// max(E - 6, -126) + 127, which is 1 to 248
__device__ __forceinline__ unsigned ckpt_scale_byte(float top) {
    const unsigned e = __float_as_uint(top) >> 23;   // top has no sign
    return top == 0.f ? 0u : e == 255u ? 255u : e > 7u ? e - 6u : 1u;
}
// 2^(127 - s) of the byte for `top`; some power of two where that is 0 (zeros have code 0 with any) or 255 (codes are masked)
__device__ __forceinline__ float ckpt_inverse(float top) { return __uint_as_float((260u - max(__float_as_uint(top) >> 23, 7u)) << 23); }
__device__ __forceinline__ bool ckpt_bad(float top) { return __float_as_uint(top) >= 0x7f800000u; }   // infinite or NaN: byte 255
// 2^(s - 127): 0 for the byte 0, NaN for 255
__device__ __forceinline__ float ckpt_scale(unsigned s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23); }

// Codes in the low bytes of floats.  Added to 1.5 * 2^23 the quotient x / scale, which is exact, is rounded to the nearest whole number,
// ties to even, and its two's complement is the sum's low byte.  Only a block whose largest quotient reaches 127.5 can round to
// 128: one in 200, so a warp votes on that (`cut`) and clamps there.
constexpr float kCkptMagic = 12582912.f;
__device__ __forceinline__ bool ckpt_cut(float top, float inverse) { return !(top * inverse < 127.5f); }   // for a warp's vote
__device__ __forceinline__ float ckpt_code(float x, float inverse, bool cut) {
    const float v = fmaf(x, inverse, kCkptMagic);
    return cut ? fminf(fmaxf(v, kCkptMagic - 127.f), kCkptMagic + 127.f) : v;
}
// four codes, each with the inverse scale of its own block
__device__ __forceinline__ unsigned ckpt_codes4(float2 a, float2 b, float2 inv_a, float2 inv_b, bool cut) {
    const float2 m = make_float2(kCkptMagic, kCkptMagic);
    a = __ffma2_rn(a, inv_a, m);
    b = __ffma2_rn(b, inv_b, m);
    if (cut) {
        const float lo = kCkptMagic - 127.f, hi = kCkptMagic + 127.f;
        a.x = fminf(fmaxf(a.x, lo), hi), a.y = fminf(fmaxf(a.y, lo), hi), b.x = fminf(fmaxf(b.x, lo), hi), b.y = fminf(fmaxf(b.y, lo), hi);
    }
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
// four codes of one block
__device__ __forceinline__ unsigned ckpt_code4(float2 a, float2 b, float inverse, bool bad, bool cut) {
    const float2 i = make_float2(inverse, inverse);
    const unsigned w = ckpt_codes4(a, b, i, i, cut);
    return bad ? 0u : w;
}
__device__ __forceinline__ int8_t ckpt_code1(float x, float inverse, bool bad, bool cut) {
    return (int8_t)(bad ? 0u : __float_as_uint(ckpt_code(x, inverse, cut)));
}
// code i of a word of four as a float: 2^23 + 128 + code is put together from its bytes, and the subtraction is exact
__device__ __forceinline__ float ckpt_decode(unsigned flipped /* the word ^ 0x80808080 */, int i) {
    return __uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7540u | i)) - 8388736.f;
}
// codes i and i + 1 of a word times the scale
__device__ __forceinline__ float2 ckpt_decode2(unsigned flipped, int i, float2 scale) {
    const float2 raw = make_float2(__uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7540u | i)), __uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7540u | (i + 1))));
    return __fmul2_rn(__fadd2_rn(raw, make_float2(-8388736.f, -8388736.f)), scale);
}
// 8 codes -> 8 values in bf16, which holds them exactly
__device__ __forceinline__ void ckpt_decode_bf16(const unsigned (&w)[2], float scale, uint32_t (&b)[4]) {
    const float2 s = make_float2(scale, scale);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 v = ckpt_decode2(w[q / 2] ^ 0x80808080u, 2 * q & 3, s);
        b[q] = Elem<__nv_bfloat16>::pack2(v.x, v.y);
    }
}

static inline int64_t ckpt_blocks(int32_t C) { return ((int64_t)C + kCkptBlock - 1) / kCkptBlock; }

}  // namespace sar
