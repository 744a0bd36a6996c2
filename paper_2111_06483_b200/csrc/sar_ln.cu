// Layer normalisation of node rows and its backward pass (contracts in include/sar.h):
//   xhat = (x - mean) rstd,  y = gamma xhat + beta,  mean and 1/rstd = sqrt(var + eps) taken over a row's C columns;
//   g = gamma gy,  gx = rstd (g - <g, 1>/C - xhat <g, xhat>/C),  dgamma = sum over the rows of gy xhat,  dbeta = sum of gy.
// Each pass reads and writes its arrays once and is bound by memory.  A group of G lanes holds a row in registers between its
// sums and its result, so the variance is the mean of squared deviations (no cancellation) without a second read; the sums
// over the rows are carried in registers from row to row, then one record per block, which a second launch adds up in a fixed
// order (no atomics).  With a checkpoint the normalised rows leave the forward pass as 8-bit codes as well, and the backward
// pass reads those in place of x and mean.
#include "sar_ckpt8.cuh"
#include "sar_dispatch.cuh"
#include "sar_reduce.cuh"
#include "sar_rowkernels.cuh"

namespace sar {

constexpr int kLnBlocks = 148 * 8;    // largest grid of the backward pass (it depends on the sizes alone: a fixed summation order)
constexpr int kLnScalarCols = 1024;   // longest row that the register kernels hold one column per lane and slot

struct LnArgs {
    long long n;
    int C;
    int n_vec;                    // 16-byte vectors per row (vector kernels)
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

// A row across the G lanes of a group: slot v of lane gl holds E columns from (v G + gl) E on.  VEC: E = a 16-byte vector;
// otherwise E = 1, for rows that are no whole number of vectors or not aligned to them.
template <typename T, bool VEC>
constexpr int ln_width = VEC ? Elem<T>::EPV : 1;

template <typename T, bool VEC>
struct LnRaw {
    using type = uint4;
    __device__ __forceinline__ static uint4 zero() { return make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ static void unpack(const uint4 &r, float (&x)[Elem<T>::EPV]) { Elem<T>::unpack(r, x); }
};
template <typename T>
struct LnRaw<T, false> {
    using type = T;
    __device__ __forceinline__ static T zero() { return T(0.f); }
    __device__ __forceinline__ static void unpack(const T &r, float (&x)[1]) { x[0] = (float)r; }
};

template <int G>
__device__ __forceinline__ float ln_sum(float x) {
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d, G);
    return x;
}

template <typename T, int G, int V, bool VEC>
struct LnRow {
    static constexpr int E = ln_width<T, VEC>;
    using Raw = LnRaw<T, VEC>;
    using raw_t = typename Raw::type;
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
            r[v] = Raw::zero();
            if (live && ok[v]) r[v] = *reinterpret_cast<const raw_t *>(static_cast<const T *>(base) + at(row, v));
        }
    }
    __device__ __forceinline__ void put(void *base, long long row, const float (&x)[V][E]) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (ok[v]) {
                T *p = static_cast<T *>(base) + at(row, v);
                if constexpr (VEC) *reinterpret_cast<uint4 *>(p) = Elem<T>::pack(x[v]);
                else Elem<T>::store1(p, x[v][0]);
            }
    }
    __device__ __forceinline__ void cols(const float *p, float fill, float (&c)[V][E]) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) c[v][e] = (p && ok[v]) ? __ldg(p + col(v) + e) : fill;
    }
    // the checkpoint: 32 columns are the slots v of 32 / E consecutive lanes (of the whole group where it is narrower)
    static constexpr int LPB = 32 / E < G ? 32 / E : G;
    __device__ __forceinline__ void put_codes(const LnArgs &a, long long row, bool live, const float (&x)[V][E]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) top = max(top, ok[v] ? ckpt_magnitude(x[v][e]) : 0u);
#pragma unroll
            for (int d = 1; d < LPB; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d, G));
            const unsigned s = ckpt_scale_byte(top);
            if (!live || !ok[v]) continue;
            const float inv = ckpt_inverse(s);
            int8_t *p = a.codes + at(row, v);
            if constexpr (E == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(ckpt_code4(x[v], inv, s), ckpt_code4(x[v] + 4, inv, s));
            else if constexpr (E == 4) *reinterpret_cast<unsigned *>(p) = ckpt_code4(x[v], inv, s);
            else *p = (int8_t)(s == 255u ? 0u : ckpt_code(x[v][0], inv));
            if (col(v) % kCkptBlock == 0) a.scales[row * a.nb + col(v) / kCkptBlock] = (uint8_t)s;
        }
    }
    struct Packed {
        unsigned w[(E + 3) / 4];
        unsigned s;
    };
    __device__ __forceinline__ void ask_codes(const LnArgs &a, long long row, bool live, Packed (&r)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int i = 0; i < (E + 3) / 4; ++i) r[v].w[i] = 0;
            r[v].s = 0;
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
    __device__ __forceinline__ void decode(const Packed (&r)[V], float (&x)[V][E]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) ckpt_decode_n<E>(r[v].w, ckpt_scale(r[v].s), x[v]);
    }
};

// rows that a group asks for before it uses the first
constexpr int ln_ahead(int regs) { return regs <= 8 ? 4 : regs <= 16 ? 2 : 1; }

template <typename T, int G, int V, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads) ln_fwd_kernel(const LnArgs a) {
    after_predecessor();
    using Row = LnRow<T, G, V, VEC>;
    constexpr int E = Row::E, U = ln_ahead(V * E);
    const LaneId<G> id;
    const Row r(a, id.gl);
    float ga[V][E], be[V][E];
    r.cols(a.gamma, 1.f, ga);
    r.cols(a.beta, 0.f, be);
    const long long stride = (long long)gridDim.x * kWarpsPerBlock * (32 / G);
    const long long first = ((long long)blockIdx.x * kWarpsPerBlock + id.warp) * (32 / G);   // the warp's first row: the shuffles need all its lanes
    for (long long base = first; base < a.n; base += U * stride) {
        typename Row::raw_t raw[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) r.ask(a.x, base + u * stride + id.gid, base + u * stride + id.gid < a.n, raw[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long row = base + u * stride + id.gid;
            if (base + u * stride >= a.n) break;   // the same for all lanes
            const bool live = row < a.n;
            float x[V][E];
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Row::Raw::unpack(raw[u][v], x[v]);
#pragma unroll
                for (int e = 0; e < E; ++e) sum += x[v][e];   // a slot without columns holds zeros
            }
            const float mean = ln_sum<G>(sum) * a.inv_c;
            float dev = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x[v][e] -= mean;
                    if (r.ok[v]) dev = fmaf(x[v][e], x[v][e], dev);
                }
            const float rstd = __frsqrt_rn(fmaf(ln_sum<G>(dev), a.inv_c, a.eps));
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) x[v][e] *= rstd;
            if constexpr (CK) r.put_codes(a, row, live, x);
            if (!live) continue;
            if (id.gl == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) x[v][e] = fmaf(x[v][e], ga[v][e], be[v][e]);
            r.put(a.y, row, x);
        }
    }
}

template <typename T, int G, int V, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads) ln_bwd_kernel(const LnArgs a) {
    after_predecessor();
    using Row = LnRow<T, G, V, VEC>;
    constexpr int E = Row::E, U = ln_ahead(2 * V * E);
    extern __shared__ float smem[];   // [2][C]
    const LaneId<G> id;
    const Row r(a, id.gl);
    float ga[V][E], s0[V][E], s1[V][E];
    r.cols(a.gamma, 1.f, ga);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) s0[v][e] = s1[v][e] = 0.f;
    const long long stride = (long long)gridDim.x * kWarpsPerBlock * (32 / G);
    const long long first = ((long long)blockIdx.x * kWarpsPerBlock + id.warp) * (32 / G);
    for (long long base = first; base < a.n; base += U * stride) {
        typename Row::raw_t xr[U][V], gr[U][V];
        typename Row::Packed cr[U][V];
        float mu[U], rs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long row = base + u * stride + id.gid;
            const bool live = row < a.n;
            r.ask(a.gy, row, live, gr[u]);
            if constexpr (CK) r.ask_codes(a, row, live, cr[u]);
            else r.ask(a.x, row, live, xr[u]);
            mu[u] = !CK && live ? __ldg(a.mean_in + row) : 0.f;
            rs[u] = live ? __ldg(a.rstd_in + row) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long row = base + u * stride + id.gid;
            if (base + u * stride >= a.n) break;
            const bool live = row < a.n;
            float x[V][E], g[V][E], along = 0.f, level = 0.f;
            if constexpr (CK) r.decode(cr[u], x);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (!CK) Row::Raw::unpack(xr[u][v], x[v]);
                Row::Raw::unpack(gr[u][v], g[v]);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (!CK) x[v][e] = r.ok[v] ? (x[v][e] - mu[u]) * rs[u] : 0.f;   // xhat
                    s0[v][e] += g[v][e];
                    s1[v][e] = fmaf(g[v][e], x[v][e], s1[v][e]);
                    g[v][e] *= ga[v][e];
                    level += g[v][e];
                    along = fmaf(g[v][e], x[v][e], along);
                }
            }
            level = ln_sum<G>(level) * a.inv_c;
            along = ln_sum<G>(along) * a.inv_c;
            if (!live) continue;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) g[v][e] = rs[u] * (g[v][e] - fmaf(x[v][e], along, level));
            r.put(a.y, row, g);
        }
    }
    if (!a.partial) return;
    // the groups of a warp first, then the warps one after the other
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
            for (int d = 16; d >= G; d >>= 1) {
                s0[v][e] += __shfl_xor_sync(0xffffffffu, s0[v][e], d);
                s1[v][e] += __shfl_xor_sync(0xffffffffu, s1[v][e], d);
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
                        smem[c] = (w ? smem[c] : 0.f) + s1[v][e];
                        smem[a.C + c] = (w ? smem[a.C + c] : 0.f) + s0[v][e];
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
                unsigned top = ckpt_magnitude(xh);
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
                const unsigned s = ckpt_scale_byte(top);
                if (c < a.C) a.codes[o + c] = (int8_t)(s == 255u ? 0u : ckpt_code(xh, ckpt_inverse(s)));
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

// ---- host ------------------------------------------------------------------------------------------------------------------
enum LnKind { kLnVector, kLnScalar, kLnLong };

// Which kernel, and its lanes and slots, for rows of C columns of type t whose arrays are aligned to 16 bytes or not.
struct LnShape {
    LnKind kind;
    int G, V;
};
static sar_status ln_shape(int32_t C, sar_dtype t, bool aligned, LnShape *s) {
    Shape m;
    SAR_TRY(make_shape(1, C, t, aligned, &m));
    if (m.fast) {
        *s = {kLnVector, m.G, m.V};
    } else if (C <= kLnScalarCols) {
        int G = sar_pow2_ceil(C);
        G = G > 32 ? 32 : G < 4 ? 4 : G;
        *s = {kLnScalar, G, sar_pow2_ceil((C + G - 1) / G)};
    } else {
        *s = {kLnLong, 32, 0};
    }
    return SAR_OK;
}

template <typename T, int G, int V, bool VEC>
struct LnCfg {
    using type = T;
    static constexpr int g = G, v = V;
    static constexpr bool vec = VEC;
};
template <typename T, typename Fn>
static sar_status ln_dispatch(const LnShape &s, Fn &&f) {
#define SAR_LN_CASE(KIND, VEC, GG, VV) \
    if (s.kind == KIND && s.G == GG && s.V == VV) return f(LnCfg<T, GG, VV, VEC>{});
    SAR_LN_CASE(kLnVector, true, 4, 1)
    SAR_LN_CASE(kLnVector, true, 8, 1)
    SAR_LN_CASE(kLnVector, true, 16, 1)
    SAR_LN_CASE(kLnVector, true, 32, 1)
    SAR_LN_CASE(kLnVector, true, 32, 2)
    SAR_LN_CASE(kLnVector, true, 32, 4)
    SAR_LN_CASE(kLnVector, true, 32, 8)
    SAR_LN_CASE(kLnScalar, false, 4, 1)
    SAR_LN_CASE(kLnScalar, false, 8, 1)
    SAR_LN_CASE(kLnScalar, false, 16, 1)
    SAR_LN_CASE(kLnScalar, false, 32, 1)
    SAR_LN_CASE(kLnScalar, false, 32, 2)
    SAR_LN_CASE(kLnScalar, false, 32, 4)
    SAR_LN_CASE(kLnScalar, false, 32, 8)
    SAR_LN_CASE(kLnScalar, false, 32, 16)
    SAR_LN_CASE(kLnScalar, false, 32, 32)
#undef SAR_LN_CASE
    return SAR_ERR_UNSUPPORTED;
}

static LnArgs ln_args(int64_t n, int32_t C, sar_dtype t) {
    LnArgs a{};
    a.n = n;
    a.C = C;
    a.n_vec = (int)((size_t)C * sar_elem_size(t) / 16);
    a.inv_c = 1.f / (float)C;
    a.nb = (int)ckpt_blocks(C);
    return a;
}

template <typename T, bool CK>
static sar_status ln_forward(const LnShape &s, const LnArgs &a, cudaStream_t st) {
    const bool overlap = a.n * a.C <= kOverlapElems;
    const char *name = CK ? "ln_fwd_ckpt8" : "ln_fwd";
    if (s.kind == kLnLong) {
        const unsigned blocks = (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks);
        SAR_LAUNCH(name, st, launch_if(overlap, ln_fwd_long_kernel<T, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    }
    return ln_dispatch<T>(s, [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        unsigned blocks = blocks_for(a.n, K::g);
        if (blocks > (unsigned)kLnBlocks * 4) blocks = kLnBlocks * 4;
        SAR_LAUNCH(name, st, launch_if(overlap, ln_fwd_kernel<T, K::g, K::v, K::vec, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    });
}

template <typename T, bool CK>
static sar_status ln_backward(const LnShape &s, LnArgs a, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    const bool sums = dgamma || dbeta, overlap = a.n * a.C <= kOverlapElems;
    if (sums) {
        if (!workspace || !sar_aligned(workspace, 16) || workspace_bytes < (size_t)kLnBlocks * 2 * a.C * 4) return SAR_ERR_WORKSPACE;
        a.partial = static_cast<float *>(workspace);
    }
    const char *name = CK ? "ln_bwd_ckpt8" : "ln_bwd";
    auto reduce = [&](unsigned records) -> sar_status {
        return sums ? reduce_partials("ln_reduce", (int)records, 2 * a.C, a.C, a.partial, 1.0, dgamma, dbeta, st) : SAR_OK;
    };
    if (s.kind == kLnLong) {
        // the sums first: gx may be written over gy or x
        long long slices = (a.n + 63) / 64;
        if (slices > 148) slices = 148;
        if (sums) {
            SAR_LAUNCH("ln_bwd_sums", st, launch_if(overlap, ln_long_sums_kernel<T, CK>, (unsigned)((slices * a.C + kThreads - 1) / kThreads), kThreads, 0, st, a, (int)slices));
            SAR_TRY(sar_after_launch());
            SAR_TRY(reduce((unsigned)slices));
        }
        const unsigned blocks = (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks);
        SAR_LAUNCH(name, st, launch_if(overlap, ln_bwd_long_kernel<T, CK>, blocks, kThreads, 0, st, a));
        return sar_after_launch();
    }
    return ln_dispatch<T>(s, [&](auto cfg) -> sar_status {
        using K = decltype(cfg);
        // a few rows per lane group before a block pays for its record
        const unsigned want = blocks_for((a.n + 3) / 4, K::g);
        const unsigned blocks = want < 1 ? 1 : want < (unsigned)kLnBlocks ? want : (unsigned)kLnBlocks;
        const size_t smem = sums ? (size_t)2 * a.C * 4 : 0;
        SAR_LAUNCH(name, st, launch_if(overlap, ln_bwd_kernel<T, K::g, K::v, K::vec, CK>, blocks, kThreads, smem, st, a));
        SAR_TRY(sar_after_launch());
        return reduce(blocks);
    });
}

static sar_status ln_zero(int32_t C, float *dgamma, float *dbeta, cudaStream_t st) {
    for (float *p : {dgamma, dbeta})
        if (p) SAR_CUDA_TRY(cudaMemsetAsync(p, 0, (size_t)C * 4, st));
    return SAR_OK;
}

// codes are moved as many bytes at a time as a vector has elements
static bool ln_codes_aligned(const int8_t *codes, sar_dtype t) { return sar_aligned(codes, t == SAR_F32 ? 4 : 8); }

}  // namespace sar

using namespace sar;

extern "C" {

size_t sar_ln_workspace_bytes(int32_t C) {
    if (C < 1) return 0;
    return (size_t)kLnBlocks * 2 * C * 4 + 256;
}

static sar_status ln_fwd_entry(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                               float *mean, float *rstd, int8_t *codes, uint8_t *scales, bool ckpt, void *stream) {
    if (n < 0 || C < 1 || !(eps >= 0.f) || (n > 0 && (!x || !y || (ckpt && (!rstd || !codes || !scales))))) return SAR_ERR_INVALID_ARG;
    LnShape s;
    SAR_TRY(ln_shape(C, t, all16({x, y}) && (!ckpt || ln_codes_aligned(codes, t)), &s));
    SAR_TRY(check_elem_align({mean, rstd, gamma, beta}, 4));
    SAR_TRY(check_elem_align({x, y}, sar_elem_size(t)));
    if (n == 0) return SAR_OK;
    LnArgs a = ln_args(n, C, t);
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.eps = eps;
    a.mean = mean;
    a.rstd = rstd;
    a.codes = codes;
    a.scales = scales;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (t == SAR_F32) return ckpt ? ln_forward<float, true>(s, a, st) : ln_forward<float, false>(s, a, st);
    return ckpt ? ln_forward<__nv_bfloat16, true>(s, a, st) : ln_forward<__nv_bfloat16, false>(s, a, st);
}

sar_status sar_ln_fwd(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                      float *mean, float *rstd, void *stream) {
    return ln_fwd_entry(n, C, t, x, gamma, beta, eps, y, mean, rstd, nullptr, nullptr, false, stream);
}

sar_status sar_ln_fwd_ckpt8(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                            float *rstd, int8_t *codes, uint8_t *scales, void *stream) {
    return ln_fwd_entry(n, C, t, x, gamma, beta, eps, y, nullptr, rstd, codes, scales, true, stream);
}

static sar_status ln_bwd_entry(int64_t n, int32_t C, sar_dtype t, const void *x, const float *mean, const int8_t *codes, const uint8_t *scales,
                               bool ckpt, const float *rstd, const float *gamma, const void *gy, void *gx, float *dgamma, float *dbeta,
                               void *workspace, size_t workspace_bytes, void *stream) {
    if (n < 0 || C < 1 || (n > 0 && (!rstd || !gy || !gx || (ckpt ? !codes || !scales : !x || !mean)))) return SAR_ERR_INVALID_ARG;
    LnShape s;
    SAR_TRY(ln_shape(C, t, all16({x, gy, gx}) && (!ckpt || ln_codes_aligned(codes, t)), &s));
    SAR_TRY(check_elem_align({mean, rstd, gamma, dgamma, dbeta}, 4));
    SAR_TRY(check_elem_align({x, gy, gx}, sar_elem_size(t)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n == 0) return ln_zero(C, dgamma, dbeta, st);
    LnArgs a = ln_args(n, C, t);
    a.x = x;
    a.gy = gy;
    a.y = gx;
    a.gamma = gamma;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.codes = const_cast<int8_t *>(codes);
    a.scales = const_cast<uint8_t *>(scales);
    if (t == SAR_F32)
        return ckpt ? ln_backward<float, true>(s, a, dgamma, dbeta, workspace, workspace_bytes, st)
                    : ln_backward<float, false>(s, a, dgamma, dbeta, workspace, workspace_bytes, st);
    return ckpt ? ln_backward<__nv_bfloat16, true>(s, a, dgamma, dbeta, workspace, workspace_bytes, st)
                : ln_backward<__nv_bfloat16, false>(s, a, dgamma, dbeta, workspace, workspace_bytes, st);
}

sar_status sar_ln_bwd(int64_t n, int32_t C, sar_dtype t, const void *x, const float *mean, const float *rstd, const float *gamma,
                      const void *gy, void *gx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, C, t, x, mean, nullptr, nullptr, false, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

sar_status sar_ln_bwd_ckpt8(int64_t n, int32_t C, sar_dtype t, const int8_t *codes, const uint8_t *scales, const float *rstd,
                            const float *gamma, const void *gy, void *gx, float *dgamma, float *dbeta, void *workspace,
                            size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, C, t, nullptr, nullptr, codes, scales, true, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

}  // extern "C"
