// Kernels of the layer normalisation (internal; sar_ln.cu has the formulas and the entry points).
#pragma once

#include "sar_ckpt8.cuh"
#include "sar_device.cuh"
#include "sar_dispatch.cuh"
#include "sar_rowkernels.cuh"

#include <type_traits>

namespace sar {

constexpr int kSms = 148;
constexpr int kLnBlocks = kSms * 8;   // largest grid (grids depend on the sizes alone: a fixed summation order)
// the sums of a block's weight gradients in shared memory: as many copies as fit, a copy for each warp at most
constexpr size_t kLnSmem = 32 * 1024;
__host__ __device__ constexpr int ln_copies(int C) {
    int k = kWarpsPerBlock;
    while (k > 1 && (size_t)k * 2 * C * 4 > kLnSmem) k /= 2;
    return k;
}

struct LnArgs {
    long long n;
    int C;
    float c, inv_c, eps;          // C, 1 / C
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
// ... of the backward kernels that know groups.  A type of its own: with two members more in LnArgs the other kernels came out with
// other registers (31,000 rows of 2,047 bf16 backward 218 -> 313 us, a million of 256 from the checkpoint 243 -> 265).
struct LnGroupedArgs : LnArgs {
    const int64_t *offsets;       // [groups + 1]: the rows that take part
    int groups;
};

// The rows of some group, from the first offset to the largest (offsets read as the products by group read them), for every thread of
// the block.
__device__ __forceinline__ long long *ln_range() {
    __shared__ long long range[2];
    return range;
}
__device__ __forceinline__ void ln_find_range(const LnGroupedArgs &a) {
    if (threadIdx.x < 32) {
        const auto at = [&](int g) { return min(max((long long)__ldg(reinterpret_cast<const long long *>(a.offsets) + g), 0ll), a.n); };
        long long end = 0;
        for (int g = threadIdx.x; g <= a.groups; g += 32) end = max(end, at(g));
        for (int d = 16; d > 0; d >>= 1) end = max(end, __shfl_xor_sync(0xffffffffu, end, d));
        if (threadIdx.x == 0) ln_range()[0] = at(0), ln_range()[1] = end;
    }
    __syncthreads();
}
__device__ __forceinline__ bool ln_in_range(long long row) { return row >= ln_range()[0] && row < ln_range()[1]; }

// Where a thread stands: lane gl of group gid of its warp, whose first row is the block's row `first`.  Groups of 64 lanes and more
// are several warps.
template <int G>
struct LnLane {
    static constexpr int kRows = kThreads / G;   // rows that a block has in hand
    static constexpr bool kWarps = G > 32;
    int gl, gid, first;
    __device__ __forceinline__ LnLane() {
        gl = threadIdx.x & (G - 1);
        gid = kWarps ? 0 : (threadIdx.x & 31) / G;
        first = kRows == 1 ? 0 : kWarps ? threadIdx.x / G : (threadIdx.x >> 5) * (32 / G);
    }
};
template <int G>
static inline unsigned ln_grid(long long rows) { return (unsigned)((rows + LnLane<G>::kRows - 1) / LnLane<G>::kRows); }

// Sums over a group's lanes.  Several warps' go by way of red[which], never the same for two sums in a row, so that a sum costs one
// barrier.
struct LnRed {
    alignas(16) float2 red[3][kWarpsPerBlock];
};
template <int G>
__device__ __forceinline__ void ln_group_sync() {
    if constexpr (G == kThreads) __syncthreads();
    else asm volatile("bar.sync %0, %1;\n" ::"r"(1u + threadIdx.x / G), "n"(G) : "memory");
}
template <int G>
__device__ __forceinline__ float2 ln_sum2(float2 x, LnRed &r, int which) {
    constexpr int W = G < 32 ? G : 32;
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) x.x += __shfl_xor_sync(0xffffffffu, x.x, d, W);
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) x.y += __shfl_xor_sync(0xffffffffu, x.y, d, W);
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) r.red[which][threadIdx.x >> 5] = x;
        ln_group_sync<G>();
        const float4 *const all = reinterpret_cast<const float4 *>(r.red[which] + threadIdx.x / G * (G / 32));
        x = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < G / 64; ++w) {
            const float4 two = all[w];
            x = __fadd2_rn(x, __fadd2_rn(make_float2(two.x, two.y), make_float2(two.z, two.w)));
        }
    }
    return x;
}
template <int G>
__device__ __forceinline__ float ln_sum(float x, LnRed &r, int which) {
    constexpr int W = G < 32 ? G : 32;
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d, W);
    if constexpr (G > 32) {
        float *const red = reinterpret_cast<float *>(r.red[which]);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
        ln_group_sync<G>();
        const float *const mine = red + threadIdx.x / G * (G / 32);
        x = 0.f;
        if constexpr (G == 64) {
            const float2 two = *reinterpret_cast<const float2 *>(mine);
            x = two.x + two.y;
        }
#pragma unroll
        for (int w = 0; w < G / 128; ++w) {
            const float4 four = reinterpret_cast<const float4 *>(mine)[w];
            x += four.x + four.y + (four.z + four.w);
        }
    }
    return x;
}
__device__ __forceinline__ float2 ln_splat(float x) { return make_float2(x, x); }

// A row across the G lanes of a group, each with V slots of E columns: 16 bytes (8 bf16, 4 float32), or one column where the
// arrays are not aligned to that.  Few lanes with many columns each, 16 of bf16 and 8 of float32 where that covers the row,
// rather than many lanes with few: a warp then has up to 8 rows in hand and joins their sums in 2 to 4 steps instead of 5
// (a million rows of 256 bf16, forward: 32 lanes of 8 columns 208 us, 16 of 16 171).  Wide rows take 64 lanes and more, up to the
// block, so that they too stay in registers and are read once (us, as the choice was made: 250,000 rows of 1,024 bf16, a warp against 64 lanes, forward with
// the checkpoint 273 / 252, backward from it 292 / 252; float32, forward 326 / 309 with 128 lanes, with the checkpoint 449 / 357;
// 120,000 rows of 2,048 bf16, a block that reads its row again for every pass against 128 lanes, forward 564 / 171, backward
// 945 / 260, with the checkpoint 1091 / 239, from it 1261 / 278; since the mean is divided, forward with the checkpoint 224 and 215).
//
// LnRow: E divides C (or is 1).  Slot v of lane gl holds the columns from (v G + gl) E on, all or none of them.
template <typename T_, int E_, int G_, int V_>
struct LnRow {
    using T = T_;
    static constexpr int E = E_, G = G_, V = V_, P = (E + 1) / 2;   // pairs per slot
    static constexpr bool kShifted = false;
    using Raw = ColVec<T, E>;
    using raw_t = typename Raw::type;
    struct Packed {   // a slot of a checkpoint
        unsigned w[(E + 3) / 4];
        unsigned s;
    };
    int gl, C;
    bool ok[V];
    __device__ __forceinline__ LnRow(const LnArgs &a, int gl_, long long) : gl(gl_), C(a.C) {
#pragma unroll
        for (int v = 0; v < V; ++v) ok[v] = col(v) < C;
    }
    __device__ __forceinline__ bool has(int v, int e) const { return ok[v]; }
    // what a slot holds where it has no column: zeros
    __device__ __forceinline__ void clean(int v, float2 (&x)[P]) const {
        if constexpr (E == 1) x[0].y = 0.f;
        if (!ok[v]) {
#pragma unroll
            for (int q = 0; q < P; ++q) x[q] = make_float2(0.f, 0.f);
        }
    }
    __device__ __forceinline__ void get(const raw_t (&r)[V], float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) Raw::get(r[v], x[v]);
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
        constexpr int B = (V + SPB - 1) / SPB;   // blocks that the lane has a part of
        float top[B];
        bool cut = false;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            top[b] = 0.f;
#pragma unroll
            for (int v = b * SPB; v < (b + 1) * SPB && v < V; ++v)
#pragma unroll
                for (int q = 0; q < P; ++q) top[b] = ckpt_top(top[b], x[v][q].x, x[v][q].y);   // what is no column is zero
#pragma unroll
            for (int d = 1; d < LPB; d <<= 1) top[b] = ckpt_top(top[b], __shfl_xor_sync(0xffffffffu, top[b], d, G < 32 ? G : 32), 0.f);
            cut = cut || ckpt_cut(top[b], ckpt_inverse(top[b]));
        }
        cut = __any_sync(0xffffffffu, cut);
        if (!live) return;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const float inv = ckpt_inverse(top[b]);
            const bool bad = ckpt_bad(top[b]);
#pragma unroll
            for (int v = b * SPB; v < (b + 1) * SPB && v < V; ++v) {
                if (!ok[v]) continue;
                int8_t *p = a.codes + at(row, v);
                if constexpr (E == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(ckpt_code4(x[v][0], x[v][1], inv, bad, cut), ckpt_code4(x[v][2], x[v][3], inv, bad, cut));
                else if constexpr (E == 4) *reinterpret_cast<unsigned *>(p) = ckpt_code4(x[v][0], x[v][1], inv, bad, cut);
                else *p = ckpt_code1(x[v][0].x, inv, bad, cut);
                if (v == b * SPB && col(v) % kCkptBlock == 0) a.scales[row * a.nb + col(v) / kCkptBlock] = (uint8_t)ckpt_scale_byte(top[b]);
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

// LnShiftedRow: any C, arrays aligned to 16 bytes.  A row then starts anywhere within a vector, m columns behind its start; rows E
// apart start at the same place, and a group's rows are a multiple of 8 apart.  So slot v of lane gl holds, for all the group's
// rows, the columns from (v G + gl) E - m on, which are whole vectors of the array; those at the row's ends hold columns of
// the rows beside it as well, which count as zeros and are written column by column.
template <typename T_, int E_, int G_, int V_>
struct LnShiftedRow {
    using T = T_;
    static constexpr int E = E_, G = G_, V = V_, P = E / 2;
    static constexpr bool kShifted = true;
    static constexpr int L = kCkptBlock / E;   // lanes whose slots make a checkpoint's block, but for the m columns before it
    static_assert(G % L == 0, "a block's lanes are one group's");
    static constexpr unsigned kAll = (1u << E) - 1u;
    using Raw = ColVec<T, E>;
    using raw_t = typename Raw::type;
    struct Packed {
        unsigned w[E / 4];
        unsigned s, before;   // the scale bytes of the slot's block and, for its first m columns, of the block before
    };
    int gl, C, m;
    long long total;          // the array's values
    unsigned mask[V];         // the slot's columns that are the row's
    bool head;                // the slots begin m columns before a block
    __device__ __forceinline__ LnShiftedRow(const LnArgs &a, int gl_, long long first_row) : gl(gl_), C(a.C), total(a.n * a.C) {
        m = (int)(first_row * C % E);
        head = m > 0 && gl % L == 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mask[v] = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) mask[v] |= (unsigned)(col(v) + e >= 0 && col(v) + e < C) << e;
        }
    }
    __device__ __forceinline__ int col(int v) const { return (v * G + gl) * E - m; }
    __device__ __forceinline__ long long at(long long row, int v) const { return row * C + col(v); }
    __device__ __forceinline__ bool has(int v, int e) const { return mask[v] >> e & 1u; }
    // the vector reaches past the array's end
    __device__ __forceinline__ bool beyond(long long row, int v) const { return at(row, v) + E > total; }
    __device__ __forceinline__ void clean(int v, float2 (&x)[P]) const {
        if (mask[v] == kAll) return;
#pragma unroll
        for (int q = 0; q < P; ++q) x[q] = make_float2(has(v, 2 * q) ? x[q].x : 0.f, has(v, 2 * q + 1) ? x[q].y : 0.f);
    }
    __device__ __forceinline__ void get(const raw_t (&r)[V], float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Raw::get(r[v], x[v]);
            clean(v, x[v]);
        }
    }
    __device__ __forceinline__ void ask(const void *base, long long row, bool live, raw_t (&r)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            r[v] = raw_t{};
            if (!live || mask[v] == 0u) continue;
            const T *p = static_cast<const T *>(base) + at(row, v);
            if (!beyond(row, v)) {
                r[v] = *reinterpret_cast<const raw_t *>(p);
            } else {
                float2 x[P];
#pragma unroll
                for (int q = 0; q < P; ++q) x[q] = make_float2(has(v, 2 * q) ? (float)p[2 * q] : 0.f, has(v, 2 * q + 1) ? (float)p[2 * q + 1] : 0.f);
                r[v] = Raw::put(x);
            }
        }
    }
    __device__ __forceinline__ void put(void *base, long long row, const float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (mask[v] == 0u) continue;
            T *p = static_cast<T *>(base) + at(row, v);
            if (mask[v] == kAll) {
                *reinterpret_cast<raw_t *>(p) = Raw::put(x[v]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (has(v, e)) Elem<T>::store1(p + e, e & 1 ? x[v][e / 2].y : x[v][e / 2].x);
            }
        }
    }
    __device__ __forceinline__ void cols(const float *p, float fill, float2 (&c)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q)
                c[v][q] = make_float2(p && has(v, 2 * q) ? __ldg(p + col(v) + 2 * q) : fill, p && has(v, 2 * q + 1) ? __ldg(p + col(v) + 2 * q + 1) : fill);
    }
    // what the group's lane before the first of this lane's block holds in slot v: the block before
    template <typename X>
    __device__ __forceinline__ X before(const X (&x)[V], int v) const {
        const int first = gl & ~(L - 1);
        const X here = __shfl_sync(0xffffffffu, x[v], (first - L) & (G - 1), G), back = __shfl_sync(0xffffffffu, x[v > 0 ? v - 1 : 0], G - 1, G);
        return first > 0 ? here : v > 0 ? back : X(0);
    }
    __device__ __forceinline__ void put_codes(const LnArgs &a, long long row, bool live, const float2 (&x)[V][P]) const {
        float top[V], front[V], inv[V];   // front: of the m columns that belong to the block before
#pragma unroll
        for (int v = 0; v < V; ++v) {
            top[v] = front[v] = 0.f;
            if (head) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float y = e & 1 ? x[v][e / 2].y : x[v][e / 2].x;
                    front[v] = ckpt_top(front[v], e < m ? y : 0.f, 0.f);
                    top[v] = ckpt_top(top[v], e < m ? 0.f : y, 0.f);
                }
            } else {
#pragma unroll
                for (int q = 0; q < P; ++q) top[v] = ckpt_top(top[v], x[v][q].x, x[v][q].y);
            }
#pragma unroll
            for (int d = 1; d < L; d <<= 1) top[v] = ckpt_top(top[v], __shfl_xor_sync(0xffffffffu, top[v], d, G), 0.f);
        }
        bool cut = false, bad = false;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int first = gl & ~(L - 1);
            const float next = __shfl_sync(0xffffffffu, front[v], (first + L) & (G - 1), G), after = __shfl_sync(0xffffffffu, front[v + 1 < V ? v + 1 : v], 0, G);
            top[v] = ckpt_top(top[v], first + L < G ? next : v + 1 < V ? after : 0.f, 0.f);
            inv[v] = ckpt_inverse(top[v]);
            cut = cut || ckpt_cut(top[v], inv[v]);
            bad = bad || ckpt_bad(top[v]);
        }
        cut = __any_sync(0xffffffffu, cut);
        bad = __any_sync(0xffffffffu, bad);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float inv_before = before(inv, v);
            const float top_before = before(top, v);
            if (!live || mask[v] == 0u) continue;
            unsigned w[E / 4];
#pragma unroll
            for (int q = 0; q < P; q += 2) {
                float2 y[2] = {x[v][q], x[v][q + 1]}, i[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool fx = head && 2 * (q + h) < m, fy = head && 2 * (q + h) + 1 < m;
                    i[h] = make_float2(fx ? inv_before : inv[v], fy ? inv_before : inv[v]);
                    if (bad) y[h] = make_float2(ckpt_bad(fx ? top_before : top[v]) ? 0.f : y[h].x, ckpt_bad(fy ? top_before : top[v]) ? 0.f : y[h].y);
                }
                w[q / 2] = ckpt_codes4(y[0], y[1], i[0], i[1], cut);
            }
            int8_t *p = a.codes + at(row, v);
            if (mask[v] == kAll) {
                if constexpr (E == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<unsigned *>(p) = w[0];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (has(v, e)) p[e] = (int8_t)(w[e / 4] >> (e % 4 * 8));
            }
            const int block = (v * G + gl) / L;
            if (gl % L == 0 && block < a.nb) a.scales[row * a.nb + block] = (uint8_t)ckpt_scale_byte(top[v]);
        }
    }
    __device__ __forceinline__ void ask(const LnArgs &a, long long row, bool live, Packed (&r)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            r[v] = Packed{};
            if (!live || mask[v] == 0u) continue;
            const int8_t *p = a.codes + at(row, v);
            if (!beyond(row, v)) {
                if constexpr (E == 8) {
                    const uint2 c = __ldg(reinterpret_cast<const uint2 *>(p));
                    r[v].w[0] = c.x, r[v].w[1] = c.y;
                } else {
                    r[v].w[0] = __ldg(reinterpret_cast<const unsigned *>(p));
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (has(v, e)) r[v].w[e / 4] |= (unsigned)(unsigned char)p[e] << (e % 4 * 8);
            }
            const int block = (v * G + gl) / L;
            if (block < a.nb) r[v].s = __ldg(a.scales + row * a.nb + block);
            if (head && block > 0) r[v].before = __ldg(a.scales + row * a.nb + block - 1);
        }
    }
    __device__ __forceinline__ void decode(const Packed (&r)[V], float2 (&x)[V][P]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float here = ckpt_scale(r[v].s), front = head ? ckpt_scale(r[v].before) : here;
#pragma unroll
            for (int q = 0; q < P; ++q)
                x[v][q] = ckpt_decode2(r[v].w[q / 2] ^ 0x80808080u, 2 * q & 3, make_float2(2 * q < m ? front : here, 2 * q + 1 < m ? front : here));
            clean(v, x[v]);
        }
    }
};

// Blocks that an SM is to hold at least, which bounds the registers, for N columns a lane.  64 million values in rows of 256, us, as the
// compiler likes and so: bf16 forward 106 registers 48, 80 (three blocks) 43; backward 138 86, 128 (two) 63, from the checkpoint 140
// 107, 128 61; float32 forward with the checkpoint 84 118, 78 (three) 99.  Groups of several warps wait for each other at every sum,
// so other blocks have to fill in: 60,000 rows of 4,096 bf16 forward two 207, three 176, four 185, backward one 408, two 255,
// three 442 (the sums leave the registers).  For these bounds whole vectors spill up to 60 bytes (across 256
// lanes up to 180), single columns up to 140, shifted rows 100 to 230 backward in slots of 8 and 250 to 350 forward in six of 4; other
// bounds have not been measured for the last two.
template <typename Row>
constexpr int ln_blocks(bool bwd, bool ck) {
    constexpr int N = Row::E * Row::V, E = Row::E;
    if (Row::G > 32) return bwd ? (N <= 4 ? 3 : N <= 8 ? (E == 4 ? 3 : 2) : N <= 16 ? 2 : 1) : N <= 8 ? 4 : N <= 16 && E != 4 ? 3 : 2;
    if (E == 1) return bwd && N > 4 ? 2 : 3;
    if (bwd) return N <= 8 && ck && E == 4 && !Row::kShifted ? 3 : N <= (Row::kShifted && E == 4 ? 12 : 16) ? 2 : 1;
    if (Row::kShifted) return N <= 24 ? 2 : 1;
    return E == 8 ? (N <= 16 && !ck ? 3 : 2) : N <= 8 ? 3 : 2;
}

// A sum and its product with 1 / C round, so the mean is off by some units in its last place, which against a small spread is no small
// error (a constant row of 12345.678 came out at 0.3).
// bf16: values within a factor of two of each other are whole multiples of 2^-7 of the least, so the sum of up to 65,536 of them is
// exact, and divided it gives the float32 next to the mean; values further apart have a spread that the sum's error is small against.
// float32: the mean of the deviations says how much the mean is off, without cancellation.  Rows whose mean is more than 8 deviations
// from zero take that sum and correct what they have: below that the mean's error is less than 2^-21 deviations for each
// addition that a term passes, and the sum would cost every row (1,360,000 rows of 47, with the checkpoint 159 us, with the sum in
// every row 170).
// The quotient is one of two forms with the same bits: a division, or the product corrected by its remainder (which is exact, so that the
// result before its rounding is within 2^-22 units of the quotient, and no quotient by C lies that close to the middle of two
// floats).  The compiler keeps more in registers around the division; what that does to the passes, us, corrected / divided:
// 60,000 rows of 5,000 308 / 255, with the checkpoint 481 / 390; 1,000,000 of 100 with it 160 / 140; but 120,000 of 2,048
// (128 lanes) 177 / 196, 31,000 of 2,047, column by column, 90 / 101, and 562,000 of 16 (one slot a lane) with the checkpoint 31.3 / 32.5.
template <typename T, bool DIVIDE>
__device__ __forceinline__ float ln_mean(float sum, const LnArgs &a) {
    if constexpr (sizeof(T) == 2 && DIVIDE) return __fdiv_rn(sum, a.c);
    const float mean = sum * a.inv_c;
    if constexpr (sizeof(T) == 4) return mean;
    const float left = fmaf(-mean, a.c, sum);
    return fabsf(left) < 1.f + fabsf(mean) ? fmaf(left, a.inv_c, mean) : mean;   // an infinite mean stays
}
__device__ __forceinline__ bool ln_far(float mean, float var, float eps) { return mean * mean > 64.f * (var + eps); }
__device__ __forceinline__ float ln_variance(float squares, float off) {   // from the means of the deviations and of their squares
    const float v = fmaf(-off, off, squares);
    return v < 0.f ? 0.f : v;   // NaN stays
}

// Rows are walked one ahead: a group asks for its next row before it works on the one it has (two sets of registers in turn),
// so that loads are in flight all the time.
template <typename Row, bool CK>
__global__ void __launch_bounds__(kThreads, ln_blocks<Row>(false, CK)) ln_fwd_kernel(const LnArgs a) {
    after_predecessor();
    using T = typename Row::T;
    constexpr int G = Row::G, V = Row::V, P = Row::P;
    __shared__ LnRed red;
    const LnLane<G> id;
    const long long stride = (long long)gridDim.x * id.kRows;
    long long base = (long long)blockIdx.x * id.kRows + id.first;   // the warp's first row: the shuffles need all its lanes
    const Row r(a, id.gl, base + id.gid);
    float2 ga[V][P], be[V][P];
    r.cols(a.gamma, 1.f, ga);
    r.cols(a.beta, 0.f, be);
    const auto ask = [&](long long base, typename Row::raw_t(&raw)[V]) { r.ask(a.x, base + id.gid, base + id.gid < a.n, raw); };
    const auto work = [&](long long base, const typename Row::raw_t(&raw)[V]) {
        const long long row = base + id.gid;
        const bool live = row < a.n;
        float2 x[V][P], sum = make_float2(0.f, 0.f);
        r.get(raw, x);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < P; ++q) sum = __fadd2_rn(sum, x[v][q]);   // what is no column is zero
        float mean = ln_mean<T, (Row::E > 1 && V > 1 && (CK || G != 128))>(ln_sum<G>(sum.x + sum.y, red, 0), a);
        float2 dev = make_float2(0.f, 0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int q = 0; q < P; ++q) x[v][q] = __fadd2_rn(x[v][q], ln_splat(-mean));
            r.clean(v, x[v]);
#pragma unroll
            for (int q = 0; q < P; ++q) dev = __ffma2_rn(x[v][q], x[v][q], dev);
        }
        const float var = ln_sum<G>(dev.x + dev.y, red, 1) * a.inv_c;
        float rstd = __frsqrt_rn(var + a.eps);   // before the vote, which would hold it up (69,288 rows of 136 float32, in the L2, 12 % longer)
        if (sizeof(T) == 4 && __any_sync(0xffffffffu, ln_far(mean, var, a.eps))) {   // the sums need all lanes; a group's lanes agree, and so do its warps
            float2 rest = make_float2(0.f, 0.f);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int q = 0; q < P; ++q) rest = __fadd2_rn(rest, x[v][q]);
            const float off = ln_sum<G>(rest.x + rest.y, red, 2) * a.inv_c;
            mean += off;
            rstd = __frsqrt_rn(ln_variance(var, off) + a.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int q = 0; q < P; ++q) x[v][q] = __fadd2_rn(x[v][q], ln_splat(-off));
                r.clean(v, x[v]);
            }
        }
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

template <typename Row, bool CK, typename Args>
__global__ void __launch_bounds__(kThreads, ln_blocks<Row>(true, CK)) ln_bwd_kernel(const Args a) {
    constexpr bool GROUPED = std::is_same<Args, LnGroupedArgs>::value;
    after_predecessor();
    constexpr int G = Row::G, V = Row::V, P = Row::P;
    // where the range is at hand, us, registers / shared memory: from the checkpoint a million rows of 256 bf16 251 / 282, of 100 165 / 160,
    // 674,000 of 95 176 / 159, 120,000 of 2,048 (128 lanes) 272 / 255; from the rows a million of 256 254 / 252
    constexpr bool kKeepRange = CK && G <= 32 && Row::E == 8;
    long long begin, end;
    if constexpr (GROUPED) {
        ln_find_range(a);
        if constexpr (kKeepRange) begin = ln_range()[0], end = ln_range()[1];
    }
    extern __shared__ float smem[];   // [copies][2][C]; groups of several warps: [2][C] where there is more than one
    __shared__ LnRed red;
    const LnLane<G> id;
    const long long stride = (long long)gridDim.x * id.kRows;
    long long base = (long long)blockIdx.x * id.kRows + id.first;
    const Row r(a, id.gl, base + id.gid);
    float2 ga[V][P], s0[V][P], s1[V][P];
    r.cols(a.gamma, 1.f, ga);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < P; ++q) s0[v][q] = s1[v][q] = make_float2(0.f, 0.f);
    struct Asked {
        typename Row::raw_t x[CK ? 1 : V], g[V];
        typename Row::Packed c[CK ? V : 1];
        float mu, rs;
    };
    const auto ask = [&](long long base, Asked &q) {
        const long long row = base + id.gid;
        bool live = row < a.n;
        if constexpr (GROUPED && kKeepRange) live = live && row >= begin && row < end;   // others are zeros, and so is their gx
        else if constexpr (GROUPED) live = live && ln_in_range(row);
        r.ask(a.gy, row, live, q.g);
        if constexpr (CK) r.ask(a, row, live, q.c);
        else r.ask(a.x, row, live, q.x);
        q.mu = !CK && live ? __ldg(a.mean_in + row) : 0.f;
        q.rs = live ? __ldg(a.rstd_in + row) : 0.f;
    };
    const auto work = [&](long long base, const Asked &in, int which) {
        const long long row = base + id.gid;
        float2 x[V][P], g[V][P], along2 = make_float2(0.f, 0.f), level2 = along2;
        const float2 rs = ln_splat(in.rs);
        if constexpr (CK) r.decode(in.c, x);
        else r.get(in.x, x);
        r.get(in.g, g);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (!CK) {
#pragma unroll
                for (int q = 0; q < P; ++q) x[v][q] = __fmul2_rn(__fadd2_rn(x[v][q], ln_splat(-in.mu)), rs);   // xhat
                r.clean(v, x[v]);
            }
#pragma unroll
            for (int q = 0; q < P; ++q) {
                s0[v][q] = __fadd2_rn(s0[v][q], g[v][q]);
                s1[v][q] = __ffma2_rn(g[v][q], x[v][q], s1[v][q]);
                g[v][q] = __fmul2_rn(g[v][q], ga[v][q]);
                level2 = __fadd2_rn(level2, g[v][q]);
                along2 = __ffma2_rn(g[v][q], x[v][q], along2);
            }
        }
        const float2 both = ln_sum2<G>(make_float2(level2.x + level2.y, along2.x + along2.y), red, which);
        const float level = both.x * a.inv_c, along = both.y * a.inv_c;
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
        work(base, one, 0);
        if (base + stride >= a.n) break;
        ask(base + 2 * stride, one);
        work(base + stride, two, 1);
    }
    if (!a.partial) return;
    if constexpr (id.kWarps) {   // a column is one thread's in each group: the groups' one after the other
        float *const p = a.partial + (size_t)blockIdx.x * 2 * a.C;
#pragma unroll
        for (int t = id.kRows - 1; t >= 0; --t) {
            if (id.first == t) {
                float *const to = t == 0 ? p : smem;
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < Row::E; ++e)
                        if (r.has(v, e)) {
                            const int c = r.col(v) + e;
                            float along = e & 1 ? s1[v][e / 2].y : s1[v][e / 2].x, level = e & 1 ? s0[v][e / 2].y : s0[v][e / 2].x;
                            if (t < id.kRows - 1) along += smem[c], level += smem[a.C + c];
                            to[c] = along;
                            to[a.C + c] = level;
                        }
            }
            if (t > 0) __syncthreads();
        }
        return;
    }
    // The groups of a warp, then the warps, which have a copy each where they fit (one after the other otherwise).  Rows that start at
    // different places of a vector have different columns in a lane: their groups add to shared memory in turn.
    if constexpr (!Row::kShifted) {
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
    }
    // The warp's number once more, from a source the compiler does not see through: kept from the start it can push a value that the
    // rows need out of the registers (from the checkpoint 1,360,000 rows of 47 bf16 200 us, so 184; 500,000 of 512 266, so 262; a million
    // of 256 float32 388, so 386; but 330,000 of 768 bf16 325, so 354; other widths and passes alike to 1 %).
    unsigned warp;
    asm volatile("shr.u32 %0, %1, 5;" : "=r"(warp) : "r"(threadIdx.x));
    const unsigned copies = ln_copies(a.C), turns = kWarpsPerBlock / copies;
    float *mine = smem + warp / turns * 2 * a.C;
    for (unsigned w = 0; w < turns; ++w) {
        if (warp % turns == w) {
            for (int t = 0; t < (Row::kShifted ? 32 / G : 1); ++t) {
                if (id.gid == t) {
                    const bool begin = w == 0 && t == 0;
#pragma unroll
                    for (int v = 0; v < V; ++v)
#pragma unroll
                        for (int e = 0; e < Row::E; ++e)
                            if (r.has(v, e)) {
                                float *p = mine + r.col(v) + e;
                                p[0] = (begin ? 0.f : p[0]) + (e & 1 ? s1[v][e / 2].y : s1[v][e / 2].x);
                                p[a.C] = (begin ? 0.f : p[a.C]) + (e & 1 ? s0[v][e / 2].y : s0[v][e / 2].x);
                            }
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * a.C; c += kThreads) {
        float acc = smem[c];
        for (unsigned k = 1; k < copies; ++k) acc += smem[k * 2 * a.C + c];
        a.partial[(size_t)blockIdx.x * 2 * a.C + c] = acc;
    }
}

// ---- checkpoints of rows whose last block is short ------------------------------------------------------------------
template <typename Row>
__global__ void __launch_bounds__(kThreads, 2) ln_pack_kernel(const LnArgs a) {
    after_predecessor();
    constexpr int G = Row::G, V = Row::V, P = Row::P;
    const LnLane<G> id;
    const long long stride = (long long)gridDim.x * id.kRows;
    long long base = (long long)blockIdx.x * id.kRows + id.first;
    const Row r(a, id.gl, base + id.gid);
    const auto ask = [&](long long base, typename Row::raw_t(&raw)[V]) { r.ask(a.x, base + id.gid, base + id.gid < a.n, raw); };
    const auto work = [&](long long base, const typename Row::raw_t(&raw)[V]) {
        float2 x[V][P];
        r.get(raw, x);
        r.put_codes(a, base + id.gid, base + id.gid < a.n, x);
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

template <typename Row>
__global__ void __launch_bounds__(kThreads, 2) ln_unpack_kernel(const LnArgs a) {
    after_predecessor();
    constexpr int G = Row::G, V = Row::V, P = Row::P;
    const LnLane<G> id;
    const long long stride = (long long)gridDim.x * id.kRows;
    long long row = (long long)blockIdx.x * id.kRows + id.first + id.gid;
    const Row r(a, id.gl, row);
    const auto work = [&](long long row, const typename Row::Packed(&raw)[V]) {
        float2 x[V][P];
        r.decode(raw, x);
        r.put(a.y, row, x);
    };
    typename Row::Packed one[V], two[V];
    r.ask(a, row, row < a.n, one);
    for (; row < a.n; row += 2 * stride) {
        r.ask(a, row + stride, row + stride < a.n, two);
        work(row, one);
        if (row + stride >= a.n) break;
        r.ask(a, row + 2 * stride, row + 2 * stride < a.n, one);
        work(row + stride, two);
    }
}

// ---- rows longer than the registers of a block: it takes a row and reads it again for every pass (from L1 or L2) ----------
template <typename T>
__device__ __forceinline__ float ln_load(const void *base, long long at) { return (float)static_cast<const T *>(base)[at]; }

__device__ __forceinline__ float ln_block_sum(float x, float *red) {   // red: kWarpsPerBlock floats; the same order in every block
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarpsPerBlock; ++w) s += red[w];
    return s;
}

template <typename T, bool CK>
__global__ void __launch_bounds__(kThreads, 8) ln_fwd_long_kernel(const LnArgs a) {
    after_predecessor();
    __shared__ float red[kWarpsPerBlock];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const long long o = row * a.C;
        float sum = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) sum += ln_load<T>(a.x, o + c);
        const float first = ln_mean<T, true>(ln_block_sum(sum, red), a);
        float dev = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float d = ln_load<T>(a.x, o + c) - first;
            dev = fmaf(d, d, dev);
        }
        float var = ln_block_sum(dev, red) * a.inv_c, off = 0.f;
        if (sizeof(T) == 4 && ln_far(first, var, a.eps)) {
            float rest = 0.f;
            for (int c = threadIdx.x; c < a.C; c += kThreads) rest += ln_load<T>(a.x, o + c) - first;
            off = ln_block_sum(rest, red) * a.inv_c;
            var = ln_variance(var, off);
        }
        const float rstd = __frsqrt_rn(var + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = first + off;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int b = warp; b < a.nb; b += kWarpsPerBlock) {   // 32 columns a warp, the block of a checkpoint
            const int c = b * kCkptBlock + lane;
            const float xh = c < a.C ? (ln_load<T>(a.x, o + c) - first - off) * rstd : 0.f;
            if constexpr (CK) {
                float top = ckpt_top(xh, 0.f, 0.f);
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) top = ckpt_top(top, __shfl_xor_sync(0xffffffffu, top, d), 0.f);
                const float inv = ckpt_inverse(top);
                const bool cut = __any_sync(0xffffffffu, ckpt_cut(top, inv));
                if (c < a.C) a.codes[o + c] = ckpt_code1(xh, inv, ckpt_bad(top), cut);
                if (lane == 0) a.scales[row * a.nb + b] = (uint8_t)ckpt_scale_byte(top);
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

template <typename T, bool CK, typename Args>
__global__ void __launch_bounds__(kThreads) ln_bwd_long_kernel(const Args a) {
    constexpr bool GROUPED = std::is_same<Args, LnGroupedArgs>::value;
    after_predecessor();
    __shared__ float red[kWarpsPerBlock];
    if constexpr (GROUPED) ln_find_range(a);
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        if constexpr (GROUPED) {
            if (!ln_in_range(row)) {
                for (int c = threadIdx.x; c < a.C; c += kThreads) Elem<T>::store1(static_cast<T *>(a.y) + row * a.C + c, 0.f);
                continue;
            }
        }
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
template <typename T, bool CK, typename Args>
__global__ void __launch_bounds__(kThreads) ln_long_sums_kernel(const Args a, int slices) {
    constexpr bool GROUPED = std::is_same<Args, LnGroupedArgs>::value;
    after_predecessor();
    if constexpr (GROUPED) ln_find_range(a);
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (id >= (long long)slices * a.C) return;
    const int slice = (int)(id / a.C), c = (int)(id - (long long)slice * a.C);
    float s0 = 0.f, s1 = 0.f;
    for (long long row = slice; row < a.n; row += slices) {
        if constexpr (GROUPED) {
            if (!ln_in_range(row)) continue;
        }
        const float g = ln_load<T>(a.gy, row * a.C + c);
        s0 += g;
        s1 = fmaf(g, ln_long_xhat<T, CK>(a, row, c, CK ? 0.f : __ldg(a.mean_in + row), __ldg(a.rstd_in + row)), s1);
    }
    a.partial[(size_t)slice * 2 * a.C + c] = s1;
    a.partial[(size_t)slice * 2 * a.C + a.C + c] = s0;
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
// How rows of C columns are spread over lanes: E columns a slot, V slots in G lanes, shifted or not; E = 0: longer than a block's
// registers.
struct LnShape {
    int E, G, V;
    bool shifted;
};
// Every (E, G, V) of a kind of row in ascending E G V: the first that covers the row is taken.
#define SAR_LN_8(X) X(8, 4, 1) X(8, 4, 2) X(8, 4, 3) X(8, 8, 2) X(8, 8, 3) X(8, 16, 2) X(8, 16, 3) X(8, 32, 2) X(8, 32, 3) X(8, 64, 2) X(8, 64, 3) X(8, 128, 2) X(8, 256, 2) X(8, 256, 4)
#define SAR_LN_4(X) X(4, 4, 1) X(4, 4, 2) X(4, 8, 2) X(4, 8, 3) X(4, 16, 2) X(4, 16, 3) X(4, 32, 2) X(4, 32, 3) X(4, 64, 2) X(4, 64, 3) X(4, 128, 2) X(4, 128, 3) X(4, 256, 2) X(4, 256, 4) X(4, 256, 8)
// ... bf16 that divides into fours but not eights, where the pass reads x: 16 columns a lane here, too.  A million rows of 100, us, 8 a
// lane against 16: forward 95 / 93, with the checkpoint 160 / 140, backward 165 / 119
#define SAR_LN_4H(X) X(4, 4, 1) X(4, 4, 2) X(4, 4, 4) X(4, 8, 3) X(4, 8, 4) X(4, 16, 3) X(4, 16, 4) X(4, 32, 3) X(4, 32, 4) X(4, 64, 3) X(4, 64, 4) X(4, 128, 4) X(4, 256, 4) X(4, 256, 8)
#define SAR_LN_8S(X) X(8, 16, 2) X(8, 32, 2) X(8, 32, 3) X(8, 32, 4)
#define SAR_LN_4S(X) X(4, 32, 2) X(4, 32, 3) X(4, 32, 4) X(4, 32, 6)
// ... and narrow shifted rows, for what reads checkpoints
#define SAR_LN_8N(X) X(8, 4, 1) X(8, 4, 2) X(8, 8, 2)
#define SAR_LN_4N(X) X(4, 8, 1) X(4, 8, 2) X(4, 16, 2)
#define SAR_LN_1(X) X(1, 4, 1) X(1, 4, 4) X(1, 4, 8) X(1, 8, 6) X(1, 8, 8) X(1, 16, 6) X(1, 16, 8) X(1, 32, 8) X(1, 256, 4) X(1, 256, 8)
// Columns from which rows that are no whole vectors are taken shifted.  64 million values, us, one column a lane and slot against
// shifted: 95 bf16 forward 95 / 167, with the checkpoint 173 / 322, backward 168 / 273; 191 bf16 115 / 97, 261 / 196, 175 / 163; 191
// float32 113 / 115, 253 / 271, 165 / 161; 333 bf16 410 / 142, 718 / 288, 616 / 239.  Packed: 47 bf16 105 / 138, float32 101 / 161; 95 bf16
// 119 / 138, float32 115 / 168; 191 bf16 197 / 140.  Backward from a checkpoint: 47 bf16 205 / 184, float32 209 / 194; 95 bf16 214 / 172.
// Unpacked: 95 bf16 92 / 81, float32 88 / 91.  Float32 up to 765 columns: 8 slots of 4 spill (84,000 rows of 761 in 6 slots forward 136 / 130,
// backward 216 / 152, from the checkpoint 265 / 168, packed 171 / 128; 64,000 of 1,001 in 8 slots 113 / 113, 184 / 275, 222 / 299, 152 / 227).
constexpr int kLnShiftedFrom = 128, kPackShiftedFrom = 128, kCkptShiftedFrom = 16;

template <typename R>
struct LnCfg {
    using row = R;
};
// Calls f(LnCfg<row>{}) with the shape's kind of row.
// kLnBwd8: from a checkpoint; kLnCkpt: the kernels that pack and unpack, whose shapes are asked for as kLnPack and kLnCkpt
enum LnPass { kLnFwd, kLnBwd, kLnBwd8, kLnCkpt, kLnPack };
template <typename T, LnPass PASS, typename Fn>
static inline sar_status ln_dispatch(const LnShape &s, Fn &&f) {
#define SAR_LN_CASE(EE, GG, VV) \
    if (!s.shifted && s.E == EE && s.G == GG && s.V == VV) return f(LnCfg<LnRow<T, EE, GG, VV>>{});
#define SAR_LN_SHIFTED(EE, GG, VV) \
    if (s.shifted && s.E == EE && s.G == GG && s.V == VV) return f(LnCfg<LnShiftedRow<T, EE, GG, VV>>{});
    if constexpr (sizeof(T) == 2) {
        SAR_LN_8S(SAR_LN_SHIFTED)
    } else {
        SAR_LN_4S(SAR_LN_SHIFTED)
    }
    if constexpr (PASS == kLnCkpt || PASS == kLnBwd8) {
        if constexpr (sizeof(T) == 2) {
            SAR_LN_8N(SAR_LN_SHIFTED)
        } else {
            SAR_LN_4N(SAR_LN_SHIFTED)
        }
    }
    if constexpr (sizeof(T) == 2) {
        SAR_LN_8(SAR_LN_CASE)
    }
    if constexpr (sizeof(T) == 2 && (PASS == kLnFwd || PASS == kLnBwd)) {
        SAR_LN_4H(SAR_LN_CASE)
    } else {
        SAR_LN_4(SAR_LN_CASE)
    }
    SAR_LN_1(SAR_LN_CASE)
#undef SAR_LN_CASE
#undef SAR_LN_SHIFTED
    return SAR_ERR_UNSUPPORTED;
}

// The shape for rows of C columns of type t in arrays aligned to `arrays` bytes and codes aligned to `codes`: as many columns at a
// time as divide C and are aligned; rows that allow one at a time are taken shifted where they are wide and the arrays aligned.
static inline LnShape ln_shape(int32_t C, sar_dtype t, LnPass pass, size_t arrays, size_t codes) {
    LnShape s{0, 32, 0, false};
    const int E = t == SAR_BF16 ? 8 : 4;
    const bool from_ckpt = pass == kLnCkpt || pass == kLnBwd8 || pass == kLnPack;
    const int shifted_from = pass == kLnPack ? kPackShiftedFrom : from_ckpt ? kCkptShiftedFrom : kLnShiftedFrom;
    const auto may = [&](int e) { return C % e == 0 && arrays >= e * sar_elem_size(t) && codes >= (size_t)e; };
    int need = C;
#define SAR_LN_FIT(EE, GG, VV) \
    if (s.E == 0 && EE * GG * VV >= need) s.E = EE, s.G = GG, s.V = VV;
    if (E == 8 && may(8)) {
        SAR_LN_8(SAR_LN_FIT)
    } else if (may(4)) {
        if (E == 8 && (pass == kLnFwd || pass == kLnBwd)) {
            SAR_LN_4H(SAR_LN_FIT)
        } else {
            SAR_LN_4(SAR_LN_FIT)
        }
    } else if (C >= shifted_from && arrays >= 16 && codes >= (size_t)E) {
        s.shifted = true;
        need = C + E - 1;   // wherever in a vector the row starts
        if (E == 8) {
            if (from_ckpt) {
                SAR_LN_8N(SAR_LN_FIT)
            }
            SAR_LN_8S(SAR_LN_FIT)
        } else {
            if (from_ckpt) {
                SAR_LN_4N(SAR_LN_FIT)
            }
            SAR_LN_4S(SAR_LN_FIT)
        }
    }
    if (s.E == 0) {
        s.shifted = false;
        need = C;
        SAR_LN_1(SAR_LN_FIT)
    }
#undef SAR_LN_FIT
    return s;
}

// the largest power of two up to 16 that divides all addresses
static inline size_t ln_alignment(std::initializer_list<const void *> ps) {
    size_t a = 16;
    for (const void *p : ps)
        while (a > 1 && p && !sar_aligned(p, a)) a /= 2;
    return a;
}

static inline LnArgs ln_args(int64_t n, int32_t C) {
    LnArgs a{};
    a.n = n;
    a.C = C;
    a.c = (float)C;
    a.inv_c = 1.f / a.c;
    a.nb = (int)ckpt_blocks(C);
    return a;
}

constexpr int kLnMostColumns = 1 << 20;
constexpr int kLnBlockColumns = 8192;   // that the registers of a block hold at most
// Records of the weights' sums that the backward pass writes at most for n rows.  Blocks take two rows at least; rows longer than a
// block's registers are cut into slices of 64 rows and more (ln_slices), so that 2^20 columns take 1.2 GB for many rows, not 10.
static inline int ln_slices(long long n) { return (int)((n - 1) / 64 + 1 < kSms ? (n - 1) / 64 + 1 : kSms); }
static inline int ln_records_most(long long n, int32_t C) {
    if (n < 1) return 0;
    if (C > kLnBlockColumns) return ln_slices(n);
    return (int)((n - 1) / 2 + 1 < kLnBlocks ? (n - 1) / 2 + 1 : kLnBlocks);
}

// blocks of a kernel that run at once: each walks its rows (a constant of the kernel and the device)
template <typename K>
static unsigned ln_resident(K kernel, size_t smem) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, smem) != cudaSuccess) (void)cudaGetLastError();
    return (unsigned)(kSms * (per_sm < 1 ? 1 : per_sm > kLnBlocks / kSms ? kLnBlocks / kSms : per_sm));
}
template <typename K, typename Args>
static sar_status ln_launch(const char *name, K kernel, unsigned want, unsigned most, size_t smem, const Args &a, cudaStream_t st) {
    SAR_LAUNCH(name, st, launch_if(a.n * a.C <= kOverlapElems, kernel, want < 1 ? 1 : want < most ? want : most, kThreads, smem, st, a));
    return sar_after_launch();
}

template <typename T, bool CK>
static sar_status ln_forward_of(const LnShape &s, const LnArgs &a, cudaStream_t st) {
    const char *name = CK ? "ln_fwd_ckpt8" : "ln_fwd";
    if (s.E == 0) return ln_launch(name, ln_fwd_long_kernel<T, CK>, (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks), kLnBlocks, 0, a, st);
    return ln_dispatch<T, kLnFwd>(s, [&](auto cfg) -> sar_status {
        using Row = typename decltype(cfg)::row;
        static const unsigned most = ln_resident(ln_fwd_kernel<Row, CK>, 0);
        return ln_launch(name, ln_fwd_kernel<Row, CK>, ln_grid<Row::G>(a.n), most, 0, a, st);
    });
}

// the row pass and the records of the weights' sums (a.partial); *records: how many
template <typename T, bool CK, typename Args>
static sar_status ln_backward_of(const LnShape &s, const Args &a, unsigned *records, cudaStream_t st) {
    const char *name = std::is_same<Args, LnGroupedArgs>::value ? (CK ? "ln_bwd_ckpt8_grouped" : "ln_bwd_grouped") : CK ? "ln_bwd_ckpt8" : "ln_bwd";
    if (s.E == 0) {
        // the sums first: gx may be written over gy or x
        const int slices = ln_slices(a.n);
        if (a.partial) {
            SAR_LAUNCH("ln_bwd_sums", st, launch_if(a.n * a.C <= kOverlapElems, ln_long_sums_kernel<T, CK, Args>, (unsigned)(((long long)slices * a.C + kThreads - 1) / kThreads), kThreads, 0, st, a, slices));
            SAR_TRY(sar_after_launch());
        }
        *records = (unsigned)slices;
        return ln_launch(name, ln_bwd_long_kernel<T, CK, Args>, (unsigned)(a.n < kLnBlocks ? a.n : kLnBlocks), kLnBlocks, 0, a, st);
    }
    return ln_dispatch<T, CK ? kLnBwd8 : kLnBwd>(s, [&](auto cfg) -> sar_status {
        using Row = typename decltype(cfg)::row;
        static const unsigned most = ln_resident(ln_bwd_kernel<Row, CK, Args>, Row::G == kThreads ? 0 : kLnSmem);
        const unsigned want = ln_grid<Row::G>((a.n + 1) / 2);   // two rows per lane group, which it asks for at once, before a block pays for its record
        *records = want < 1 ? 1 : want < most ? want : most;
        return ln_launch(name, ln_bwd_kernel<Row, CK, Args>, want, most, !a.partial || Row::G == kThreads ? 0 : (size_t)(Row::G > 32 ? 1 : ln_copies(a.C)) * 2 * a.C * 4, a, st);
    });
}

// one translation unit per pass and storage type
sar_status ln_forward_f32(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st);
sar_status ln_forward_bf16(const LnShape &s, const LnArgs &a, bool ckpt, cudaStream_t st);
sar_status ln_backward_f32(const LnShape &s, const LnArgs &a, bool ckpt, unsigned *records, cudaStream_t st);
sar_status ln_backward_bf16(const LnShape &s, const LnArgs &a, bool ckpt, unsigned *records, cudaStream_t st);
// ... over the rows of some group: kernels of their own, the others have no register to spare
sar_status ln_backward_grouped_f32(const LnShape &s, const LnGroupedArgs &a, bool ckpt, unsigned *records, cudaStream_t st);
sar_status ln_backward_grouped_bf16(const LnShape &s, const LnGroupedArgs &a, bool ckpt, unsigned *records, cudaStream_t st);
// checkpoints row by row: x -> codes and scales, and back to y
sar_status ln_checkpoint_f32(const LnShape &s, const LnArgs &a, bool unpack, cudaStream_t st);
sar_status ln_checkpoint_bf16(const LnShape &s, const LnArgs &a, bool unpack, cudaStream_t st);

}  // namespace sar
