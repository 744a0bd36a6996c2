// Kernels of the layer normalisation (internal; sar_ln.cu has the formulas and the entry points).
#pragma once

#include "sar_ckpt8.cuh"
#include "sar_device.cuh"
#include "sar_dispatch.cuh"
#include "sar_rowkernels.cuh"

namespace sar {

constexpr int kSms = 148;
constexpr int kLnBlocks = kSms * 8;   // largest grid (grids depend on the sizes alone: a fixed summation order)
constexpr int kLnRowCols = 1024;      // longest row that a warp holds in registers

struct LnArgs {
    long long n;
    int C;
    float inv_c, eps;
    const void *x, *gy;
    void *y;                      // forward: y; backward: gx
    const float *gamma, *beta;    // [C] or null
    const float *mean_in, *rstd_in;
    float *mean, *rstd;           // [n] or null
    int8_t *codes;                // checkpoint: [n, C] and [n, nb]
    uint8_t *scales;
    int nb;
    float *partial;               // [blocks][2][C] or null (no weight gradients asked for)
};

// A row across the G lanes of a group: slot v of lane gl holds E columns from (v G + gl) E on, E being 16 bytes (8 bf16, 4
// float32), 8 bytes (4 bf16) or one column, whatever C and the addresses allow.  Few lanes with many columns each, 16 where C
// allows it, rather than many lanes with few: a warp then has up to 8 rows in hand and joins their sums in 2 to 4 steps
// instead of 5.  (A million rows of 256 bf16, forward, 16 lanes of 16 columns against 32 of 8: see the table in sar_ln.cu.)
template <int G>
__device__ __forceinline__ float ln_sum(float x) {
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d, G);
    return x;
}
__device__ __forceinline__ float2 ln_splat(float x) { return make_float2(x, x); }

template <typename T, int E, int G, int V>
struct LnRow {
    static constexpr int P = (E + 1) / 2;   // pairs per slot
    using Raw = ColVec<T, E>;
    using raw_t = typename Raw::type;
    struct Packed {   // a slot of a checkpoint
        unsigned w[(E + 3) / 4];
        unsigned s;
    };
    int gl, C;
    bool ok[V];
    __device__ __forceinline__ LnRow(const LnArgs &a, int gl_) : gl(gl_), C(a.C) {
#pragma unroll
        for (int v = 0; v < V; ++v) ok[v] = col(v) < C;   // E divides C: a slot has all its columns or none
    }
    __device__ __forceinline__ int col(int v) const { return (v * G + gl) * E; }
    __device__ __forceinline__ long long at(long long row, int v) const { return row * C + col(v); }
    // plain loads: the result may be written over the array that was read (by the same lanes, after they have read it)
    __device__ __forceinline__ void ask(const void *base, long long row, bool live, raw_t (&r)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            r[v] = raw_t{};
            if (live && ok[v]) r[v] = *reinterpret_cast<const raw_t *>(static_cast<const T *>(base) + at(row, v));
        }
    }
    __device__ __forceinline__ void put(void *base, long long row, const float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (ok[v]) *reinterpret_cast<raw_t *>(static_cast<T *>(base) + at(row, v)) = Raw::put(x[v]);
    }
    __device__ __forceinline__ void cols(const float *p, float fill, float2 (&c)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                c[v][q].x = (p && ok[v]) ? __ldg(p + col(v) + 2 * q) : fill;
                c[v][q].y = E == 1 ? 0.f : (p && ok[v]) ? __ldg(p + col(v) + 2 * q + 1) : fill;
            }
    }
    // The checkpoint: 32 columns are the slots of LPB consecutive lanes, SPB slots each (the whole group where it is narrower).
    static constexpr int SPB = G * E >= 32 ? 1 : 32 / (G * E), LPB = 32 / E < G ? 32 / E : G;
    __device__ __forceinline__ void put_codes(const LnArgs &a, long long row, bool live, const float2 (&x)[V][P]) const {
#pragma unroll
        for (int v0 = 0; v0 < V; v0 += SPB) {
            float top = 0.f;
#pragma unroll
            for (int v = v0; v < v0 + SPB && v < V; ++v)
#pragma unroll
                for (int q = 0; q < P; ++q)
                    if (ok[v]) top = ckpt_top(top, x[v][q].x, E == 1 ? 0.f : x[v][q].y);
#pragma unroll
            for (int d = 1; d < LPB; d <<= 1) top = ckpt_top(top, __shfl_xor_sync(0xffffffffu, top, d, G), 0.f);
            const unsigned s = ckpt_scale_byte(top);
            const float inv = ckpt_inverse(s);
            const bool cut = ckpt_cut(top, inv);
            if (!live) continue;
#pragma unroll
            for (int v = v0; v < v0 + SPB && v < V; ++v) {
                if (!ok[v]) continue;
                int8_t *p = a.codes + at(row, v);
                if constexpr (E == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(ckpt_code4(x[v][0], x[v][1], inv, s, cut), ckpt_code4(x[v][2], x[v][3], inv, s, cut));
                else if constexpr (E == 4) *reinterpret_cast<unsigned *>(p) = ckpt_code4(x[v][0], x[v][1], inv, s, cut);
                else *p = ckpt_code1(x[v][0].x, inv, s, cut);
                if (v == v0 && col(v) % kCkptBlock == 0) a.scales[row * a.nb + col(v) / kCkptBlock] = (uint8_t)s;
            }
        }
    }
    __device__ __forceinline__ void ask(const LnArgs &a, long long row, bool live, Packed (&r)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            r[v] = Packed{};
            if (!live || !ok[v]) continue;
            const int8_t *p = a.codes + at(row, v);
            if constexpr (E == 8) {
                const uint2 c = __ldg(reinterpret_cast<const uint2 *>(p));
                r[v].w[0] = c.x, r[v].w[1] = c.y;
            } else if constexpr (E == 4) {
                r[v].w[0] = __ldg(reinterpret_cast<const unsigned *>(p));
            } else {
                r[v].w[0] = (unsigned char)__ldg(reinterpret_cast<const signed char *>(p));
            }
            r[v].s = __ldg(a.scales + row * a.nb + col(v) / kCkptBlock);
        }
    }
    __device__ __forceinline__ void decode(const Packed (&r)[V], float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float2 s = ln_splat(ckpt_scale(r[v].s));
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const unsigned w = r[v].w[q / 2] ^ 0x80808080u;
                x[v][q] = E == 1 ? make_float2(ckpt_decode(w, 0) * s.x, 0.f) : ckpt_decode2(w, 2 * q & 3, s);
            }
        }
    }
};

// Blocks that an SM is to hold at least, which bounds the registers, for N columns a lane.  A million rows of 256 columns, us:
// bf16 forward 106 registers 190, 80 (three blocks) 171; backward 138 344, 128 (two) 252, from the checkpoint 140 429, 128 245;
// float32 forward with the checkpoint 84 472, 78 (three) 397; backward from it 102 483, 80 (three) 392.
constexpr int ln_blocks(int N, int E, bool bwd, bool ck) {
    return N > 16 ? 1 : E == 8 ? (bwd || ck ? 2 : 3) : E == 4 ? (N > 8 ? 1 : bwd && !ck ? 2 : 3) : N > 8 ? 1 : bwd && N > 4 ? 2 : 3;
}

// Rows are walked one ahead: a group asks for its next row before it works on the one it has (two sets of registers in turn),
// so that loads are in flight all the time.
template <typename T, int E, int G, int V, bool CK>
__global__ void __launch_bounds__(kThreads, ln_blocks(E * V, E, false, CK)) ln_fwd_kernel(const LnArgs a) {
    after_predecessor();
    using Row = LnRow<T, E, G, V>;
    constexpr int P = Row::P;
    const LaneId<G> id;
    const Row r(a, id.gl);
    float2 ga[V][P], be[V][P];
    r.cols(a.gamma, 1.f, ga);
    r.cols(a.beta, 0.f, be);
    const long long stride = (long long)gridDim.x * kWarpsPerBlock * (32 / G);
    long long base = ((long long)blockIdx.x * kWarpsPerBlock + id.warp) * (32 / G);   // the warp's first row: the shuffles need all its lanes
    const auto ask = [&](long long base, typename Row::raw_t(&raw)[V]) { r.ask(a.x, base + id.gid, base + id.gid < a.n, raw); };
    const auto work = [&](long long base, const typename Row::raw_t(&raw)[V]) {
        const long long row = base + id.gid;
        const bool live = row < a.n;
        float2 x[V][P], sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Row::Raw::get(raw[v], x[v]);
#pragma unroll
            for (int q = 0; q < P; ++q) sum = __fadd2_rn(sum, x[v][q]);   // a slot without columns holds zeros
        }
        const float mean = ln_sum<G>(sum.x + sum.y) * a.inv_c;
        const float2 shift = make_float2(-mean, E == 1 ? 0.f : -mean);
        float2 dev = make_float2(0.f, 0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!r.ok[v]) continue;
#pragma unroll
            for (int q = 0; q < P; ++q) {
                x[v][q] = __fadd2_rn(x[v][q], shift);
                dev = __ffma2_rn(x[v][q], x[v][q], dev);
            }
        }
        const float rstd = __frsqrt_rn(fmaf(ln_sum<G>(dev.x + dev.y), a.inv_c, a.eps));
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q) x[v][q] = __fmul2_rn(x[v][q], ln_splat(rstd));
        if constexpr (CK) r.put_codes(a, row, live, x);
        if (!live) return;
        if (id.gl == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q) x[v][q] = __ffma2_rn(x[v][q], ga[v][q], be[v][q]);
        r.put(a.y, row, x);
    };
    typename Row::raw_t one[V], two[V];
    if (base < a.n) ask(base, one);
    for (; base < a.n; base += 2 * stride) {
        ask(base + stride, two);
        work(base, one);
        if (base + stride >= a.n) break;
        ask(base + 2 * stride, one);
        work(base + stride, two);
    }
}

template <typename T, int E, int G, int V, bool CK>
__global__ void __launch_bounds__(kThreads, ln_blocks(E * V, E, true, CK)) ln_bwd_kernel(const LnArgs a) {
    after_predecessor();
    using Row = LnRow<T, E, G, V>;
    constexpr int P = Row::P;
    extern __shared__ float smem[];   // [2][C]
    const LaneId<G> id;
    const Row r(a, id.gl);
    float2 ga[V][P], s0[V][P], s1[V][P];
    r.cols(a.gamma, 1.f, ga);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < P; ++q) s0[v][q] = s1[v][q] = make_float2(0.f, 0.f);
    const long long stride = (long long)gridDim.x * kWarpsPerBlock * (32 / G);
    long long base = ((long long)blockIdx.x * kWarpsPerBlock + id.warp) * (32 / G);
    struct Asked {
        typename Row::raw_t x[CK ? 1 : V], g[V];
        typename Row::Packed c[CK ? V : 1];
        float mu, rs;
    };
    const auto ask = [&](long long base, Asked &q) {
        const long long row = base + id.gid;
        const bool live = row < a.n;
        r.ask(a.gy, row, live, q.g);
        if constexpr (CK) r.ask(a, row, live, q.c);
        else r.ask(a.x, row, live, q.x);
        q.mu = !CK && live ? __ldg(a.mean_in + row) : 0.f;
        q.rs = live ? __ldg(a.rstd_in + row) : 0.f;
    };
    const auto work = [&](long long base, const Asked &in) {
        const long long row = base + id.gid;
        float2 x[V][P], g[V][P], along2 = make_float2(0.f, 0.f), level2 = along2;
        const float2 rs = ln_splat(in.rs);
        if constexpr (CK) r.decode(in.c, x);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (!CK) {
                const float2 shift = make_float2(-in.mu, E == 1 ? 0.f : -in.mu);
                Row::Raw::get(in.x[v], x[v]);
#pragma unroll
                for (int q = 0; q < P; ++q) x[v][q] = __fmul2_rn(__fadd2_rn(x[v][q], shift), rs);   // xhat; where there is no column, g is zero
            }
            Row::Raw::get(in.g[v], g[v]);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                s0[v][q] = __fadd2_rn(s0[v][q], g[v][q]);
                if (CK || r.ok[v]) s1[v][q] = __ffma2_rn(g[v][q], x[v][q], s1[v][q]);
                g[v][q] = __fmul2_rn(g[v][q], ga[v][q]);
                level2 = __fadd2_rn(level2, g[v][q]);
                if (CK || r.ok[v]) along2 = __ffma2_rn(g[v][q], x[v][q], along2);   // not 0 * xhat: a row of infinite mean would spoil it
            }
        }
        const float level = ln_sum<G>(level2.x + level2.y) * a.inv_c;
        const float along = ln_sum<G>(along2.x + along2.y) * a.inv_c;
        if (row >= a.n) return;
        const float2 minus_along = ln_splat(-along), minus_level = ln_splat(-level);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q) g[v][q] = __fmul2_rn(__fadd2_rn(g[v][q], __ffma2_rn(x[v][q], minus_along, minus_level)), rs);
        r.put(a.y, row, g);
    };
    Asked one, two;
    if (base < a.n) ask(base, one);
    for (; base < a.n; base += 2 * stride) {
        ask(base + stride, two);
        work(base, one);
        if (base + stride >= a.n) break;
        ask(base + 2 * stride, one);
        work(base + stride, two);
    }
    if (!a.partial) return;
    // the groups of a warp first, then the warps one after the other
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < P; ++q) {
#pragma unroll
            for (int d = 16; d >= G; d >>= 1) {
                s0[v][q].x += __shfl_xor_sync(0xffffffffu, s0[v][q].x, d);
                s0[v][q].y += __shfl_xor_sync(0xffffffffu, s0[v][q].y, d);
                s1[v][q].x += __shfl_xor_sync(0xffffffffu, s1[v][q].x, d);
                s1[v][q].y += __shfl_xor_sync(0xffffffffu, s1[v][q].y, d);
            }
        }
    for (int w = 0; w < kWarpsPerBlock; ++w) {
        if (id.warp == w && id.gid == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r.ok[v]) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int c = r.col(v) + e;
                        smem[c] = (w ? smem[c] : 0.f) + (e & 1 ? s1[v][e / 2].y : s1[v][e / 2].x);
                        smem[a.C + c] = (w ? smem[a.C + c] : 0.f) + (e & 1 ? s0[v][e / 2].y : s0[v][e / 2].x);
                    }
                }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * a.C; c += kThreads) a.partial[(size_t)blockIdx.x * 2 * a.C + c] = smem[c];
}

// ---- rows longer than the registers of a warp: a block takes a row and reads it again for every pass (from L1 or L2) ----------
template <typename T>
__device__ __forceinline__ float ln_load(const void *base, long long at) { return (float)static_cast<const T *>(base)[at]; }

__device__ __forceinline__ float ln_block_sum(float x, float *red) {   // red: kWarpsPerBlock floats; the same order in every block
    x = ln_sum<32>(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarpsPerBlock; ++w) s += red[w];
    return s;
}

template <typename T, bool CK>
__global__ void __launch_bounds__(kThreads) ln_fwd_long_kernel(const LnArgs a) {
    after_predecessor();
    __shared__ float red[kWarpsPerBlock];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const long long o = row * a.C;
        float sum = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) sum += ln_load<T>(a.x, o + c);
        const float mean = ln_block_sum(sum, red) * a.inv_c;
        float dev = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float d = ln_load<T>(a.x, o + c) - mean;
            dev = fmaf(d, d, dev);
        }
        const float rstd = __frsqrt_rn(fmaf(ln_block_sum(dev, red), a.inv_c, a.eps));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int b = warp; b < a.nb; b += kWarpsPerBlock) {   // 32 columns a warp, the block of a checkpoint
            const int c = b * kCkptBlock + lane;
            const float xh = c < a.C ? (ln_load<T>(a.x, o + c) - mean) * rstd : 0.f;
            if constexpr (CK) {
                float top = ckpt_top(xh, 0.f, 0.f);
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) top = ckpt_top(top, __shfl_xor_sync(0xffffffffu, top, d), 0.f);
                const unsigned s = ckpt_scale_byte(top);
                const float inv = ckpt_inverse(s);
                const bool cut = ckpt_cut(top, inv);
                if (c < a.C) a.codes[o + c] = ckpt_code1(xh, inv, s, cut);
                if (lane == 0) a.scales[row * a.nb + b] = (uint8_t)s;
            }
            if (c < a.C) Elem<T>::store1(static_cast<T *>(a.y) + o + c, fmaf(xh, a.gamma ? __ldg(a.gamma + c) : 1.f, a.beta ? __ldg(a.beta + c) : 0.f));
        }
    }
}

template <typename T, bool CK>
__device__ __forceinline__ float ln_long_xhat(const LnArgs &a, long long row, int c, float mean, float rstd) {
    if constexpr (CK) return (float)a.codes[row * a.C + c] * ckpt_scale(a.scales[row * a.nb + c / kCkptBlock]);
    else return (ln_load<T>(a.x, row * a.C + c) - mean) * rstd;
}

template <typename T, bool CK>
__global__ void __launch_bounds__(kThreads) ln_bwd_long_kernel(const LnArgs a) {
    after_predecessor();
    __shared__ float red[kWarpsPerBlock];
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const float mean = CK ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
        float along = 0.f, level = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float g = ln_load<T>(a.gy, row * a.C + c) * (a.gamma ? __ldg(a.gamma + c) : 1.f);
            level += g;
            along = fmaf(g, ln_long_xhat<T, CK>(a, row, c, mean, rstd), along);
        }
        level = ln_block_sum(level, red) * a.inv_c;
        along = ln_block_sum(along, red) * a.inv_c;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float g = ln_load<T>(a.gy, row * a.C + c) * (a.gamma ? __ldg(a.gamma + c) : 1.f);
            const float xh = ln_long_xhat<T, CK>(a, row, c, mean, rstd);
            Elem<T>::store1(static_cast<T *>(a.y) + row * a.C + c, rstd * (g - fmaf(xh, along, level)));
        }
    }
}

// the sums over the rows for long rows: thread (slice, column) walks every slices-th row
template <typename T, bool CK>
__global__ void __launch_bounds__(kThreads) ln_long_sums_kernel(const LnArgs a, int slices) {
    after_predecessor();
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (id >= (long long)slices * a.C) return;
    const int slice = (int)(id / a.C), c = (int)(id - (long long)slice * a.C);
    float s0 = 0.f, s1 = 0.f;
    for (long long row = slice; row < a.n; row += slices) {
        const float g = ln_load<T>(a.gy, row * a.C + c);
        s0 += g;
        s1 = fmaf(g, ln_long_xhat<T, CK>(a, row, c, CK ? 0.f : __ldg(a.mean_in + row), __ldg(a.rstd_in + row)), s1);
    }
    a.partial[(size_t)slice * 2 * a.C + c] = s1;
    a.partial[(size_t)slice * 2 * a.C + a.C + c] = s0;
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
// How rows of C columns are spread over lanes: E columns a slot, V slots in G lanes; E = 0: longer than a warp's registers.
struct LnShape {
    int E, G, V;
};
template <typename T, int E, int G, int V>
struct LnCfg {
    using type = T;
    static constexpr int e = E, g = G, v = V;
};
// Every (G, V) of a width E in ascending G V E: the first that covers C is taken.  16 columns a lane of bf16 and 8 of float32 or
// single ones where that covers the row, more only where 32 lanes do not.
#define SAR_LN_8(X) X(8, 4, 1) X(8, 4, 2) X(8, 4, 3) X(8, 8, 2) X(8, 8, 3) X(8, 16, 2) X(8, 16, 3) X(8, 32, 2) X(8, 32, 3) X(8, 32, 4)
#define SAR_LN_4(X) X(4, 4, 1) X(4, 4, 2) X(4, 8, 2) X(4, 8, 3) X(4, 16, 2) X(4, 16, 3) X(4, 32, 2) X(4, 32, 3) X(4, 32, 4) X(4, 32, 6) X(4, 32, 8)
#define SAR_LN_1(X) X(1, 4, 1) X(1, 4, 4) X(1, 4, 8) X(1, 8, 6) X(1, 8, 8) X(1, 16, 6) X(1, 16, 8) X(1, 32, 6) X(1, 32, 8) X(1, 32, 12) X(1, 32, 16) X(1, 32, 24) X(1, 32, 32)
// ... and of single columns in the backward pass, which carries two sums for each of them
#define SAR_LN_1B(X) X(1, 4, 1) X(1, 4, 4) X(1, 8, 4) X(1, 16, 3) X(1, 16, 4) X(1, 32, 3) X(1, 32, 4) X(1, 32, 6) X(1, 32, 8) X(1, 32, 12) X(1, 32, 16) X(1, 32, 24) X(1, 32, 32)

// blocks of a kernel that run at once: each walks its rows (a constant of the kernel and the device; 48 KB of shared memory and less)
template <typename K>
static unsigned ln_resident(K kernel, size_t smem) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, smem) != cudaSuccess) (void)cudaGetLastError();
    return (unsigned)(kSms * (per_sm < 1 ? 1 : per_sm > kLnBlocks / kSms ? kLnBlocks / kSms : per_sm));
}

template <typename T, bool BWD, typename Fn>
static inline sar_status ln_dispatch(const LnShape &s, Fn &&f) {
#define SAR_LN_CASE(EE, GG, VV) \
    if (s.E == EE && s.G == GG && s.V == VV) return f(LnCfg<T, EE, GG, VV>{});
    if constexpr (sizeof(T) == 2) {
        SAR_LN_8(SAR_LN_CASE)
    }
    SAR_LN_4(SAR_LN_CASE)
    if constexpr (BWD) {
        SAR_LN_1B(SAR_LN_CASE)
    } else {
        SAR_LN_1(SAR_LN_CASE)
    }
#undef SAR_LN_CASE
    return SAR_ERR_UNSUPPORTED;
}

template <typename T, bool CK>
static sar_status ln_forward_of(const LnShape &s, const LnArgs &a, cudaStream_t st) {
    const bool overlap = a.n * a.C <= kOverlapElems;
    const char *name = CK ? "ln_fwd_ckpt8" : "ln_fwd";
    if (s.E == 0) {
        const unsigned blocks = (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks);
        SAR_LAUNCH(name, st, launch_if(overlap, ln_fwd_long_kernel<T, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    }
    return ln_dispatch<T, false>(s, [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        static const unsigned most = ln_resident(ln_fwd_kernel<T, K::e, K::g, K::v, CK>, 0);
        const unsigned want = blocks_for(a.n, K::g), blocks = want < most ? want : most;
        SAR_LAUNCH(name, st, launch_if(overlap, ln_fwd_kernel<T, K::e, K::g, K::v, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    });
}

// the row pass and the records of the weights' sums (a.partial); *records: how many
template <typename T, bool CK>
static sar_status ln_backward_of(const LnShape &s, const LnArgs &a, unsigned *records, cudaStream_t st) {
    const bool overlap = a.n * a.C <= kOverlapElems;
    const char *name = CK ? "ln_bwd_ckpt8" : "ln_bwd";
    if (s.E == 0) {
        // the sums first: gx may be written over gy or x
        const int slices = (int)((a.n + 63) / 64 < 148 ? (a.n + 63) / 64 : 148);
        if (a.partial) {
            SAR_LAUNCH("ln_bwd_sums", st, launch_if(overlap, ln_long_sums_kernel<T, CK>, (unsigned)(((long long)slices * a.C + kThreads - 1) / kThreads), kThreads, 0, st, a, slices));
            SAR_TRY(sar_after_launch());
        }
        *records = (unsigned)slices;
        const unsigned blocks = (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks);
        SAR_LAUNCH(name, st, launch_if(overlap, ln_bwd_long_kernel<T, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    }
    return ln_dispatch<T, true>(s, [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        // a few rows per lane group before a block pays for its record
        const unsigned want = blocks_for((a.n + 3) / 4, K::g);
        static const unsigned most = ln_resident(ln_bwd_kernel<T, K::e, K::g, K::v, CK>, 2 * kLnRowCols * sizeof(float));
        const unsigned blocks = want < 1 ? 1 : want < most ? want : most;
        *records = blocks;
        SAR_LAUNCH(name, st, launch_if(overlap, ln_bwd_kernel<T, K::e, K::g, K::v, CK>, blocks, kThreads, a.partial ? (size_t)2 * a.C * 4 : 0, st, a));
        return sar_after_launch();
    });
}

// one translation unit per pass and storage type
sar_status ln_forward_f32(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st);
sar_status ln_forward_bf16(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st);
sar_status ln_backward_f32(const LnShape &s, const LnArgs &a, bool ckpt, unsigned *records, cudaStream_t st);
sar_status ln_backward_bf16(const LnShape &s, const LnArgs &a, bool ckpt, unsigned *records, cudaStream_t st);

}  // namespace sar
