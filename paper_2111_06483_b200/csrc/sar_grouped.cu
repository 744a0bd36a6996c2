// Products of node rows with a matrix for each group of rows (contracts in include/sar.h): rows offsets[g] .. offsets[g+1] of an
// array belong to group g (a node type), the groups' sizes are known on the device only.
//   z = h W[g],  dh = dz W[g]^T       grouped_rows_kernel: tiles of 128 rows, each within one group
//   dW[g] = h^T dz over g's rows      grouped_weight_kernel: the rows are cut into equal chunks; a chunk's part of every group
//                                     that it meets is a partial result, and a second launch adds them up
// bf16 operands, tensor-core products (tcgen05) with float32 sums in tensor memory, operands staged by tiled copies.
#include "sar_ckpt8.cuh"
#include "sar_device.cuh"
#include "sar_dispatch.cuh"
#include "sar_tc.cuh"

#include <atomic>
#include <utility>

namespace sar {

constexpr int kTileRows = 128;      // rows of a product's tile: all lanes of tensor memory
constexpr int kStep = 64;           // contraction per stage: 128 bytes of bf16
constexpr int kPanel = 64 * 128;    // 64 rows of 128 bytes
constexpr int kStepMost = 128;      // rows of a stage where they are the contraction
constexpr int kGroupsMax = SAR_MAX_GROUPS;
static std::atomic<long long> g_wait_limit{kWaitCycles};   // of the launches to come (sar_set_wait_limit)

sar_status tc_tensor_map(CUtensorMap *map, const void *base, int rank, const uint64_t *dims, const uint32_t *box) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = [] {   // the driver's function: the library links against the runtime alone
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) (void)cudaGetLastError();
        return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(f) : nullptr;
    }();
    if (!encode) return SAR_ERR_CUDA;
    cuuint64_t size[3], stride[2];
    cuuint32_t tile[3], one[3] = {1, 1, 1};
    uint64_t bytes = 2;
    for (int i = 0; i < rank; ++i) {
        size[i] = dims[i];
        tile[i] = box[i];
        bytes *= dims[i];
        if (i + 1 < rank) stride[i] = bytes;
    }
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(base), size, stride, tile, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SAR_OK : SAR_ERR_CUDA;
}

// First row of every group, and what precedes each group in tiles, by the block's first warp (the others see it after a barrier).  Offsets that lead backwards or out
// of the array are brought to the last one seen and to the array's ends: whatever they hold, every access stays in bounds.
struct GroupTable {
    int first[kGroupsMax + 1];   // first[g] .. first[g + 1]: g's rows
    int tiles[kGroupsMax + 1];   // tiles of 128 rows before group g
};
__device__ __forceinline__ void group_table(GroupTable &t, const int64_t *__restrict__ offsets, int G, int n) {
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int top = 0, tiles = 0;
        for (int g0 = 0; g0 <= G; g0 += 32) {
            const int g = g0 + lane;
            long long o = g > G ? 0 : offsets ? __ldg(reinterpret_cast<const long long *>(offsets) + g) : g ? n : 0;
            int lo = o < 0 ? 0 : o > n ? n : (int)o;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, lo, d);
                if (lane >= d) lo = max(lo, y);
            }
            lo = max(lo, top);
            const int before = __shfl_up_sync(0xffffffffu, lo, 1);
            // tiles of the group that ends here
            int k = g == 0 || g > G ? 0 : (lo - (lane ? before : top) + kTileRows - 1) / kTileRows;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, k, d);
                if (lane >= d) k += y;
            }
            k += tiles;
            if (g <= G) {
                t.first[g] = lo;
                t.tiles[g] = k;
            }
            top = __shfl_sync(0xffffffffu, lo, 31);
            tiles = __shfl_sync(0xffffffffu, k, 31);
        }
    }
}

// ---- rows: z = h W[g], dh = dz W[g]^T ----------------------------------------------------------------------------------------
//
// One block per SM.  A block keeps one slice of columns (all of them, up to 256) and walks a run of row tiles, so that
// the weights of a group, which are read again for every tile, are loaded once and stay in shared memory as long as the tiles
// belong to the group; each row is read once per slice and written once.  Warp 0 issues the copies, warp 1 the products into
// one of two accumulators, warps 2 to 5 round the other one to bf16 and store it.  A tile that ends inside a group's last rows
// reads the next group's along with them (a row's result depends on no other row) and stores its own rows alone.
struct RowsArgs {
    CUtensorMap a, w, d;
    const int64_t *offsets;
    __nv_bfloat16 *out;
    int *flag;
    long long wait_limit;
    int n, G, K, N;
    int cols;        // columns per slice (a multiple of 64 up to 256)
    int slices;      // slices of columns
    int steps;       // of 64 along the contraction
    int stages;      // of the ring
    int slots;       // sets of weights in shared memory; 0: they pass through the ring with the rows
    int store_bufs;  // 2, or 1 where the ring needs the room
    int zero_rest;   // rows of no group are written as zeros
};
constexpr int kRowsThreads = 192;
constexpr int kStoreBuf = 32 * 128;   // a warp's 32 rows of 64 columns
constexpr int kSlotsMax = 4, kStagesMax = 8;
struct RowsShared {
    alignas(8) uint64_t full[kStagesMax], empty[kStagesMax], w_full[kSlotsMax], w_empty[kSlotsMax], acc_full[2], acc_empty[2], done;
    uint32_t tmem, filled, sets;   // stages and sets of weights that copies were issued into
    int failed;
    GroupTable table;
};

template <bool WT>
__global__ void __launch_bounds__(kRowsThreads, 1) grouped_rows_kernel(const __grid_constant__ RowsArgs p) {
    after_predecessor();
    extern __shared__ uint8_t dyn[];
    RowsShared &sh = *reinterpret_cast<RowsShared *>(dyn);
    const int panels = p.cols / 64, w_step = panels * kPanel;
    const uint32_t w_set = (uint32_t)p.steps * w_step;
    const uint32_t base = (smem_addr(dyn) + (uint32_t)sizeof(RowsShared) + 1023u) & ~1023u;
    const uint32_t stage_bytes = kTileRows * 128 + (p.slots ? 0 : w_step);
    const uint32_t ring = base + 4 * p.store_bufs * kStoreBuf, weights = ring + p.stages * stage_bytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Waits waits{&sh.failed, p.wait_limit};

    // the table, tensor memory, the barriers and the maps, each by a warp of its own
    group_table(sh.table, p.offsets, p.G, p.n);
    if (warp == 1) tmem_alloc(smem_addr(&sh.tmem));
    if (threadIdx.x == 64) {
        for (int i = 0; i < p.stages; ++i) bar_init(smem_addr(&sh.full[i]), 1), bar_init(smem_addr(&sh.empty[i]), 1);
        for (int i = 0; i < kSlotsMax; ++i) bar_init(smem_addr(&sh.w_full[i]), 1), bar_init(smem_addr(&sh.w_empty[i]), 1);
        for (int i = 0; i < 2; ++i) bar_init(smem_addr(&sh.acc_full[i]), 1), bar_init(smem_addr(&sh.acc_empty[i]), 4);
        bar_init(smem_addr(&sh.done), 1);
        sh.failed = 0;
        bar_init_fence();
    }
    if (threadIdx.x == 96) map_prefetch(&p.a), map_prefetch(&p.w), map_prefetch(&p.d);
    __syncwarp();
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = sh.tmem;

    // this block's slice and its run of tiles
    const int teams = gridDim.x / p.slices, team = blockIdx.x / p.slices;   // the grid is teams x slices
    const int n0 = (blockIdx.x % p.slices) * p.cols, cols = min(p.cols, p.N - n0);
    const int total = sh.table.tiles[p.G];
    const int t0 = (int)((long long)total * team / teams), t1 = (int)((long long)total * (team + 1) / teams);
    int g0 = 0;
    {
        int hi = p.G;   // the group of tile t0: tiles[g0] <= t0 < tiles[g0 + 1]
        while (hi - g0 > 1) {
            const int mid = (g0 + hi) / 2;
            (sh.table.tiles[mid] <= t0 ? g0 : hi) = mid;
        }
    }

    // all lanes of a warp walk its role's loop and wait; one of them issues
    if (warp == 0) {
        RingPlace st, ws;   // in the ring of stages, among the sets of weights
        uint32_t use = 0, set = 0;   // stages and sets filled so far
        int g = g0, held = -1;
        bool ok = true;
        for (int t = t0; ok && t < t1; ++t) {
            while (t >= sh.table.tiles[g + 1]) ++g;
            if (p.slots && g != held) {
                const uint32_t slot = ws.at, bar = smem_addr(&sh.w_full[slot]);
                ok = warp_wait(smem_addr(&sh.w_empty[slot]), ws.round ^ 1, waits);
                if (!ok) break;
                if (one_lane()) {
                    bar_expect(bar, w_set);
                    for (int k = 0; k < p.steps; ++k) {
                        const uint32_t at = weights + slot * w_set + k * w_step;
                        if (WT) tile_load_3d(at, &p.w, k * kStep, n0, g, bar);
                        else
                            for (int c = 0; c < panels; ++c) tile_load_3d(at + c * kPanel, &p.w, n0 + c * 64, k * kStep, g, bar);
                    }
                }
                __syncwarp();
                held = g;
                ++set;
                ws.next(p.slots);
            }
            const int row = sh.table.first[g] + (t - sh.table.tiles[g]) * kTileRows;
            for (int k = 0; k < p.steps; ++k, ++use, st.next(p.stages)) {
                const uint32_t s = st.at, bar = smem_addr(&sh.full[s]), at = ring + s * stage_bytes;
                ok = warp_wait(smem_addr(&sh.empty[s]), st.round ^ 1, waits);
                if (!ok) break;
                if (one_lane()) {
                    bar_expect(bar, stage_bytes);
                    tile_load_2d(at, &p.a, k * kStep, row, bar);
                    if (!p.slots) {
                        const uint32_t b = at + kTileRows * 128;
                        if (WT) tile_load_3d(b, &p.w, k * kStep, n0, g, bar);
                        else
                            for (int c = 0; c < panels; ++c) tile_load_3d(b + c * kPanel, &p.w, n0 + c * 64, k * kStep, g, bar);
                    }
                }
                __syncwarp();
            }
        }
        if (lane == 0) sh.filled = use, sh.sets = set;
    } else if (warp == 1) {
        const uint32_t instr = tc_instr((cols + 15) & ~15, false, !WT);
        RingPlace st, ws, acc;
        uint32_t wset = 0;
        int g = g0, held = -1;
        bool ok = true;
        for (int t = t0; ok && t < t1; ++t, acc.next(2)) {
            while (t >= sh.table.tiles[g + 1]) ++g;
            if (p.slots && g != held) {
                if (held >= 0) {
                    if (one_lane()) tc_commit(smem_addr(&sh.w_empty[ws.at]));   // all products with the last set
                    __syncwarp();
                    ws.next(p.slots);
                }
                ok = warp_wait(smem_addr(&sh.w_full[ws.at]), ws.round, waits);
                if (!ok) break;
                wset = weights + ws.at * w_set;
                held = g;
            }
            ok = warp_wait(smem_addr(&sh.acc_empty[acc.at]), acc.round ^ 1, waits);
            if (!ok) break;
            tc_after_sync();
            const uint32_t d = tmem + acc.at * 256;
            for (int k = 0; k < p.steps; ++k, st.next(p.stages)) {
                const uint32_t at = ring + st.at * stage_bytes, b = p.slots ? wset + k * w_step : at + kTileRows * 128;
                ok = warp_wait(smem_addr(&sh.full[st.at]), st.round, waits);
                if (!ok) break;
                const int left = (min(kStep, p.K - k * kStep) + 15) / 16;   // copies fill what lies beyond K with zeros
                if (one_lane()) {
                    const uint64_t da = tc_operand(at, 16, 1024), db = tc_operand(b, WT ? 16 : kPanel, 1024);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < left) tc_mma(d, tc_advance(da, j * 32), tc_advance(db, j * (WT ? 32 : 2048)), instr, k > 0 || j > 0);
                    tc_commit(smem_addr(&sh.empty[st.at]));
                }
                __syncwarp();
            }
            if (ok && one_lane()) tc_commit(smem_addr(&sh.acc_full[acc.at]));
            __syncwarp();
        }
    } else {
        const int quad = warp & 3;   // the lanes of tensor memory that this warp may read
        const uint32_t stage = base + (warp - 2) * p.store_bufs * kStoreBuf;
        uint32_t stored = 0;
        RingPlace acc;
        int g = g0;
        for (int t = t0; t < t1; ++t, acc.next(2)) {
            const uint32_t buf = acc.at;
            while (t >= sh.table.tiles[g + 1]) ++g;
            if (!warp_wait(smem_addr(&sh.acc_full[buf]), acc.round, waits)) break;
            tc_after_sync();
            const int row = sh.table.first[g] + (t - sh.table.tiles[g]) * kTileRows + quad * 32;
            const int rows = min(32, sh.table.first[g + 1] - row);   // may be <= 0
            for (int c = 0; c < cols; c += 64, ++stored) {
                const uint32_t at = stage + (p.store_bufs == 2 ? (stored & 1) * kStoreBuf : 0);
                if (p.store_bufs == 2) store_wait_read<1>();   // lane 0's last copy out of this buffer
                else store_wait_read<0>();
                __syncwarp();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[32];
                    tmem_ask(tmem + buf * 256 + c + h * 32 + ((uint32_t)(quad * 32) << 16), x);
                    tmem_wait_load(x);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x[q * 8 + e]);
                        const uint4 r = Elem<__nv_bfloat16>::pack(v);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + lane * 128 + (((h * 4 + q) ^ (lane & 7)) << 4)), "r"(r.x),
                                     "r"(r.y), "r"(r.z), "r"(r.w)
                                     : "memory");
                    }
                }
                if (rows == 32) {
                    async_proxy_fence();
                    __syncwarp();
                    if (lane == 0) tile_store_2d(&p.d, n0 + c, row, at);
                } else {   // the group ends here: its rows alone
                    __syncwarp();
                    const int chunk = lane & 7;
                    if (n0 + c + chunk * 8 < p.N)
                        for (int r = lane >> 3; r < rows; r += 4) {
                            uint4 v;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at + r * 128 + ((chunk ^ (r & 7)) << 4)));
                            *reinterpret_cast<uint4 *>(p.out + (long long)(row + r) * p.N + n0 + c + chunk * 8) = v;
                        }
                    __syncwarp();
                }
                if (lane == 0) store_commit();
            }
            tc_before_sync();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&sh.acc_empty[buf]));
        }
        if (p.zero_rest) {
            const int head = sh.table.first[0], tail = sh.table.first[p.G], rest = head + p.n - tail;
            for (int i = team * 4 + warp - 2; i < rest; i += teams * 4) {
                const int r = i < head ? i : tail + i - head;
                for (int c = lane * 8; c < cols; c += 256) *reinterpret_cast<uint4 *>(p.out + (long long)r * p.N + n0 + c) = make_uint4(0, 0, 0, 0);
            }
        }
        if (lane == 0) store_wait_all();
    }
    __syncwarp();
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (sh.failed) {
        if (threadIdx.x == 0) drain_copies(sh.full, p.stages, sh.filled), drain_copies(sh.w_full, p.slots, sh.sets);
        if (warp == 1) drain_products(&sh.done);
        // What is missing must not pass as a result: NaN in all of the block's tiles (the copies out have ended, the roles wait for them).
        const int across = cols / 8;
        for (int t = t0, g = g0; t < t1; ++t) {
            while (t >= sh.table.tiles[g + 1]) ++g;
            const int row = sh.table.first[g] + (t - sh.table.tiles[g]) * kTileRows, rows = min(kTileRows, sh.table.first[g + 1] - row);
            for (int i = threadIdx.x; i < rows * across; i += kRowsThreads)
                *reinterpret_cast<uint4 *>(p.out + (long long)(row + i / across) * p.N + n0 + i % across * 8) = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
        }
    }
    if (warp == 1) tmem_free(tmem);
    if (threadIdx.x == 0 && sh.failed && p.flag) *p.flag = 1;
}

// ---- weights: dW[g] = h^T dz ---------------------------------------------------------------------------------------------------
//
// The contraction runs along the rows, so both operands are read as they lie (contraction along a tile's rows).  A block owns a
// tile of 128 x (up to) 256 of dW and a chunk of rows; the blocks of a chunk's tiles run side by side and share its rows in L2.
//
// The tensor cores add to a float32 sum by cutting off what does not fit: every step of 16 rows takes up to one unit of the last
// place towards zero, and 16,384 rows in one sum are 2e-5 to 3e-5 off (256 rows 2e-7, 1,024 rows 1e-6, 65,536 rows 8e-5 and
// more).  So a sum runs over kRunRows rows at most; then eight warps add it, rounding to nearest, to sums that lie beside it
// in tensor memory (128 x 256 sums would take half of the register file).
//
// With a checkpoint eight more warps make the first operand: codes times scale, exact in bf16, written where a copy would have put
// them.  Its rows stand for gamma v + beta, and  (gamma v + beta)^T dz = gamma (v^T dz) + beta (column sums of dz):  gamma and
// beta enter in float32 after the product instead of rounding every value, and the column sums are taken from the tiles of dz
// that are in shared memory anyway.
constexpr int kRunRows = 512;
struct WeightArgs {
    CUtensorMap h, dz;
    const int64_t *offsets;
    const int8_t *codes;
    const uint8_t *scales;
    float *part;     // [chunks + G][d_in][d_out]: chunk c's part of group g in record c + g (along the way both only grow)
    float *sums;     // [chunks + G][2 m_tiles][d_out]: sums of dz's columns, a share of the rows each, or null
    int *flag;
    long long wait_limit;
    int n, G, d_in, d_out, nb;
    int cols;        // of a tile (a multiple of 64 up to 256)
    int m_tiles, n_tiles;
    int chunk_rows;  // a multiple of 64
    int stages;
    int step;        // rows per stage: 64 or 128
    int h_panels;    // of a stage: 2, or 1 where h has no more
};
constexpr int kAdders = 8, kMakers = 8;   // warps; the adders' work is laid out for 8
constexpr int kWeightThreads = 64 + kAdders * 32, kWeightThreads8 = kWeightThreads + kMakers * 32;
constexpr uint32_t kTurnBuf = 32 * 64;    // an adder's 32 rows of 16 sums on their way out
struct WeightShared {
    alignas(8) uint64_t full[kStagesMax], empty[kStagesMax], made[kStagesMax], acc_full[2], acc_empty[2], done;
    uint32_t tmem, filled;   // stages that copies were issued into
    int failed;
    GroupTable table;
};

// NaN in the block's part of its records, and so in the sums over them.  A function of its own, called rarely: within the kernel it
// keeps values over the roles' loops, which the 96 registers of the checkpoint's threads have no room for.
__device__ __noinline__ void weight_gave_up(const WeightArgs &p, const GroupTable &table) {
    const int tiles = p.m_tiles * p.n_tiles, chunk = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int m0 = tile / p.n_tiles * 128, n0 = tile % p.n_tiles * p.cols, across = min(p.cols, p.d_out - n0) / 4;
    const long long chunk0 = (long long)chunk * p.chunk_rows, chunk1 = chunk0 + p.chunk_rows;
    for (int g = 0; g < p.G; ++g) {
        if (table.first[g] >= chunk1 || table.first[g + 1] <= chunk0 || table.first[g] == table.first[g + 1]) continue;
        for (int i = threadIdx.x; i < min(128, p.d_in - m0) * across; i += blockDim.x)
            *reinterpret_cast<uint4 *>(p.part + ((long long)(chunk + g) * p.d_in + m0 + i / across) * p.d_out + n0 + i % across * 4) =
                make_uint4(0x7fffffffu, 0x7fffffffu, 0x7fffffffu, 0x7fffffffu);
    }
}

template <bool CK>
__global__ void __launch_bounds__(CK ? kWeightThreads8 : kWeightThreads, 1) grouped_weight_kernel(const __grid_constant__ WeightArgs p) {
    after_predecessor();
    extern __shared__ uint8_t dyn[];
    WeightShared &sh = *reinterpret_cast<WeightShared *>(dyn);
    const uint32_t turns = (smem_addr(dyn) + (uint32_t)sizeof(WeightShared) + 1023u) & ~1023u, ring = turns + kAdders * kTurnBuf;
    const int panels = p.cols / 64;
    const uint32_t panel = p.step * 128, stage_bytes = (p.h_panels + panels) * panel, dz_at = p.h_panels * panel;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Waits waits{&sh.failed, p.wait_limit};

    group_table(sh.table, p.offsets, p.G, p.n);
    if (warp == 1) tmem_alloc(smem_addr(&sh.tmem));
    if (threadIdx.x == 64) {
        // a stage is free when its products are done, and the adders have taken their sums of it
        for (int i = 0; i < p.stages; ++i) bar_init(smem_addr(&sh.full[i]), 1), bar_init(smem_addr(&sh.empty[i]), p.sums ? 1 + kAdders : 1), bar_init(smem_addr(&sh.made[i]), kMakers);
        for (int i = 0; i < 2; ++i) bar_init(smem_addr(&sh.acc_full[i]), 1), bar_init(smem_addr(&sh.acc_empty[i]), kAdders);
        bar_init(smem_addr(&sh.done), 1);
        sh.failed = 0;
        bar_init_fence();
    }
    if (threadIdx.x == 96) {
        if (!CK) map_prefetch(&p.h);
        map_prefetch(&p.dz);
    }
    __syncwarp();
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = sh.tmem;

    const int tiles = p.m_tiles * p.n_tiles;
    const int chunk = blockIdx.x / tiles, tile = blockIdx.x % tiles, m_tile = tile / p.n_tiles;
    const int m0 = m_tile * 128, n0 = tile % p.n_tiles * p.cols, cols = min(p.cols, p.d_out - n0);
    const int h_panels = p.d_in - m0 > 64 ? 2 : 1;   // with columns
    // tensor memory: two accumulators and the sums where all three fit, one of up to 256 columns and the sums otherwise
    const uint32_t apart = (cols + 31) & ~31, bufs = 3 * apart <= kTmemCols ? 2 : 1, sum_cols = bufs == 2 ? 2 * apart : kTmemCols / 2;
    const int chunk0 = (int)min((long long)p.n, (long long)chunk * p.chunk_rows), chunk1 = (int)min((long long)p.n, (long long)chunk0 + p.chunk_rows);
    int g0 = 0;   // the first group that ends behind the chunk's start
    for (int hi = p.G; g0 < hi;) {
        const int mid = (g0 + hi) / 2;
        if (sh.table.first[mid + 1] > chunk0) hi = mid;
        else g0 = mid + 1;
    }
    // every role walks the same segments: group g's rows within the chunk
    const auto segment = [&](int g, int &lo, int &hi) {
        lo = max(chunk0, sh.table.first[g]);
        hi = min(chunk1, sh.table.first[g + 1]);
        return lo < hi;
    };
    const auto more = [&](int g) { return g < p.G && sh.table.first[g] < chunk1; };
    // rows from `rows` to the next multiple of 16 of a tile take part in the products, but are another group's: zeros in the
    // panels from .. to - 1 of the stage, by the threads me = 0 .. of - 1
    const auto clear = [&](uint32_t at, int rows, int from, int to, int me, int of) {
        const int rest = 16 - rows % 16;
        for (int i = me; i < rest * 8 * (to - from); i += of) {
            const uint32_t where = at + (from + i / (rest * 8)) * panel + (rows + i / 8 % rest) * 128 + (i % 8) * 16;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};\n" ::"r"(where), "r"(0) : "memory");
        }
    };

    if (warp == 0) {
        RingPlace st;
        uint32_t use = 0;
        bool ok = true;
        for (int g = g0; ok && more(g); ++g) {
            int lo, hi;
            if (!segment(g, lo, hi)) continue;
            for (int r = lo; r < hi; r += p.step, ++use, st.next(p.stages)) {
                const uint32_t s = st.at, bar = smem_addr(&sh.full[s]), at = ring + s * stage_bytes;
                ok = warp_wait(smem_addr(&sh.empty[s]), st.round ^ 1, waits);
                if (!ok) break;
                if (one_lane()) {
                    bar_expect(bar, ((CK ? 0 : h_panels) + panels) * panel);
                    if (!CK)
                        for (int c = 0; c < h_panels; ++c) tile_load_2d(at + c * panel, &p.h, m0 + c * 64, r, bar);
                    for (int c = 0; c < panels; ++c) tile_load_2d(at + dz_at + c * panel, &p.dz, n0 + c * 64, r, bar);
                }
                __syncwarp();
            }
        }
        if (lane == 0) sh.filled = use;
    } else if (warp == 1) {
        const uint32_t instr = tc_instr((cols + 15) & ~15, true, true);
        RingPlace st, acc;
        bool ok = true;
        for (int g = g0; ok && more(g); ++g) {
            int lo, hi;
            if (!segment(g, lo, hi)) continue;
            for (int r0 = lo; ok && r0 < hi; r0 += kRunRows, acc.next(bufs)) {
                const uint32_t buf = acc.at;
                ok = warp_wait(smem_addr(&sh.acc_empty[buf]), acc.round ^ 1, waits);
                if (!ok) break;
                tc_after_sync();
                const int r1 = min(hi, r0 + kRunRows);
                for (int r = r0; r < r1; r += p.step, st.next(p.stages)) {
                    const uint32_t s = st.at, at = ring + s * stage_bytes;
                    const int rows = min(p.step, hi - r);
                    ok = warp_wait(smem_addr(&sh.full[s]), st.round, waits);
                    if (CK) ok = ok && warp_wait(smem_addr(&sh.made[s]), st.round, waits);
                    if (!ok) break;
                    if (!CK && rows % 16) {
                        clear(at, rows, 0, h_panels, lane, 32);
                        clear(at, rows, p.h_panels, p.h_panels + panels, lane, 32);
                        async_proxy_fence();
                        __syncwarp();
                    }
                    if (one_lane()) {
                        const uint64_t da = tc_operand(at, panel, 1024), db = tc_operand(at + dz_at, panel, 1024);
#pragma unroll
                        for (int j = 0; j < kStep / 16; ++j)
                            if (j * 16 < rows) tc_mma(tmem + buf * apart, tc_advance(da, j * 2048), tc_advance(db, j * 2048), instr, r > r0 || j > 0);
                        if (rows > kStep) {
#pragma unroll
                            for (int j = kStep / 16; j < kStepMost / 16; ++j)
                                if (j * 16 < rows) tc_mma(tmem + buf * apart, tc_advance(da, j * 2048), tc_advance(db, j * 2048), instr, true);
                        }
                        tc_commit(smem_addr(&sh.empty[s]));
                    }
                    __syncwarp();
                }
                if (ok && one_lane()) tc_commit(smem_addr(&sh.acc_full[buf]));
                __syncwarp();
            }
        }
    } else if (warp < 2 + kAdders) {
        const uint32_t quad = warp & 3, part = (warp - 2) / 4, lanes = quad * 32 << 16;   // rows m0 + 32 quad + lane of dW, every other 32 columns
        const uint32_t turn_buf = turns + (warp - 2) * kTurnBuf;
        // The column sums of dz: panel quad, 8 columns of every fourth row of one half of a step, the steps shared by the blocks of a
        // chunk.  A thread's rows are 4 apart, so that their chunks lie at one of two places of the swizzle.
        const bool want_sums = CK && p.sums && (int)quad < panels;
        const int half = p.step / 2, row0 = part * half + (lane >> 3);
        const uint32_t sum_at = dz_at + quad * panel + row0 * 128, even = ((lane & 7) ^ (row0 & 7)) << 4, odd = ((lane & 7) ^ ((row0 + 4) & 7)) << 4;
        float2 cs[4];
        RingPlace st, acc;
        bool ok = true;
        for (int g = g0; ok && more(g); ++g) {
            int lo, hi;
            if (!segment(g, lo, hi)) continue;
            float *out = p.part + ((long long)(chunk + g) * p.d_in + m0 + quad * 32) * p.d_out + n0;   // the warp's first row
            int turn = 0;   // the step's number modulo the tiles that share the sums
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[e] = make_float2(0.f, 0.f);
            for (int r0 = lo; r0 < hi; r0 += kRunRows, acc.next(bufs)) {
                if (CK && p.sums) {
                    const int r1 = min(hi, r0 + kRunRows);
                    for (int r = r0; r < r1; r += p.step, st.next(p.stages)) {
                        // also where it is another block's turn: the arrival below belongs to this round of the stage
                        ok = warp_wait(smem_addr(&sh.full[st.at]), st.round, waits);
                        if (!ok) break;
                        if (want_sums && turn == m_tile) {
                            const uint32_t at = ring + st.at * stage_bytes + sum_at;
                            float2 cr[4];   // a step's sums first: long sums of single values lose digits
#pragma unroll
                            for (int e = 0; e < 4; ++e) cr[e] = make_float2(0.f, 0.f);
                            for (int i0 = 0; i0 < half / 4; i0 += 8) {   // 8 rows of a thread at a time
                                uint4 v[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    v[i] = make_uint4(0u, 0u, 0u, 0u);
                                    if (row0 + 4 * (i0 + i) < hi - r)
                                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n"
                                                     : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                                                     : "r"(at + (i0 + i) * 512 + (i & 1 ? odd : even)));
                                }
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    float2 x[4];
                                    Pairs<__nv_bfloat16>::get(v[i], x);
#pragma unroll
                                    for (int e = 0; e < 4; ++e) cr[e] = __fadd2_rn(cr[e], x[e]);
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) cs[e] = __fadd2_rn(cs[e], cr[e]);
                            __syncwarp();
                        }
                        if (lane == 0) bar_arrive(smem_addr(&sh.empty[st.at]));
                        if (++turn == p.m_tiles) turn = 0;
                    }
                    if (!ok) break;
                }
                const uint32_t buf = acc.at;
                ok = warp_wait(smem_addr(&sh.acc_full[buf]), acc.round, waits);
                if (!ok) break;
                tc_after_sync();
                const bool first = r0 == lo, last = r0 + kRunRows >= hi;
                for (int c = part * 32; c < cols; c += kAdders / 4 * 32) {
                    uint32_t x[32], y[32];
                    tmem_ask(tmem + buf * apart + c + lanes, x);
                    if (!first) tmem_ask(tmem + sum_cols + c + lanes, y);
                    tmem_wait_load(x);
                    if (!first) {
                        tmem_tie(y);
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) + __uint_as_float(y[e]));
                    }
                    if (!last) {
                        tmem_store(tmem + sum_cols + c + lanes, x);
                    } else {
                        // A thread has a row of 32 sums.  Written so, a store touches 32 lines (128 x 256 sums: 10,000 cycles); turned in
                        // shared memory, where chunk q of row l lies at q ^ (l >> 1 & 3), it writes 64 bytes of 8 rows.
#pragma unroll
                        for (int f = 0; f < 2; ++f) {
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(turn_buf + lane * 64 + ((q ^ (lane >> 1 & 3)) << 4)), "r"(x[f * 16 + q * 4]),
                                             "r"(x[f * 16 + q * 4 + 1]), "r"(x[f * 16 + q * 4 + 2]), "r"(x[f * 16 + q * 4 + 3])
                                             : "memory");
                            __syncwarp();
                            const int q = lane & 3, col = c + f * 16 + q * 4;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int r = i * 8 + (lane >> 2);
                                uint4 v;
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(turn_buf + r * 64 + ((q ^ (r >> 1 & 3)) << 4)) : "memory");
                                if (m0 + (int)quad * 32 + r < p.d_in && col < cols) *reinterpret_cast<uint4 *>(out + (long long)r * p.d_out + col) = v;
                            }
                            __syncwarp();
                        }
                    }
                }
                tmem_wait_store();
                tc_before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&sh.acc_empty[buf]));
            }
            if (ok && want_sums) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int d = 8; d < 32; d <<= 1) {
                        cs[e].x += __shfl_xor_sync(0xffffffffu, cs[e].x, d);
                        cs[e].y += __shfl_xor_sync(0xffffffffu, cs[e].y, d);
                    }
                const int col = quad * 64 + lane * 8;
                if (lane < 8 && col < cols) {
                    float4 *to = reinterpret_cast<float4 *>(p.sums + ((long long)(chunk + g) * 2 * p.m_tiles + m_tile * 2 + part) * p.d_out + n0 + col);
                    to[0] = make_float4(cs[0].x, cs[0].y, cs[1].x, cs[1].y);
                    to[1] = make_float4(cs[2].x, cs[2].y, cs[3].x, cs[3].y);
                }
            }
        }
    } else if constexpr (CK) {
        const int w = warp - 2 - kAdders, me = w * 32 + lane;
        // the part of h: 8 columns of four rows a step and thread, asked for kAhead steps before they are used
        constexpr int kAhead = 3, kRows = 4;
        const int across = p.h_panels * 8, hc = me & (across - 1), hr = me / across, apart = kMakers * 32 / across;   // apart * kRows = p.step
        uint2 code[kAhead][kRows];
        unsigned scale[kAhead][kRows];
        const bool h_cols = m0 + hc * 8 < p.d_in;
        const int8_t *codes;     // of the thread's first row kAhead steps on, or where the segment begins
        const uint8_t *scales;
        const int code_rows = apart * p.d_in, scale_rows = apart * p.nb;
        const auto begin = [&](int r) {
            codes = p.codes + (long long)(r + hr) * p.d_in + m0 + hc * 8;
            scales = p.scales + (long long)(r + hr) * p.nb + (m0 + hc * 8) / kCkptBlock;
        };
        const auto ask = [&](uint2 (&code)[kRows], unsigned (&scale)[kRows], int left) {   // `left` rows to the segment's end
            if (left >= p.step && h_cols) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    code[i] = __ldg(reinterpret_cast<const uint2 *>(codes + i * code_rows));
                    scale[i] = __ldg(scales + i * scale_rows);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    code[i] = make_uint2(0u, 0u);
                    scale[i] = 0;
                    if (h_cols && hr + apart * i < left) {
                        code[i] = __ldg(reinterpret_cast<const uint2 *>(codes + i * code_rows));
                        scale[i] = __ldg(scales + i * scale_rows);
                    }
                }
            }
            codes += (long long)p.step * p.d_in;
            scales += p.step * p.nb;
        };
        // where they go in a stage (apart is a multiple of 8: the rows of a thread have one place in the swizzle)
        const uint32_t h_at = (hc >> 3) * panel + hr * 128 + (((hc & 7) ^ (hr & 7)) << 4), h_apart = apart * 128;
        RingPlace st;
        bool ok = true;
        for (int g = g0; ok && more(g); ++g) {
            int lo, hi;
            if (!segment(g, lo, hi)) continue;
            begin(lo);
#pragma unroll
            for (int d = 0; d < kAhead; ++d) ask(code[d], scale[d], hi - lo - d * p.step);
            for (int r3 = lo; ok && r3 < hi; r3 += kAhead * p.step) {
#pragma unroll
                for (int d = 0; d < kAhead; ++d) {   // unrolled: the sets are registers
                    const int r = r3 + d * p.step;
                    if (r >= hi) break;
                    const uint32_t s = st.at, at = ring + s * stage_bytes;
                    const int rows = min(p.step, hi - r);
                    ok = warp_wait(smem_addr(&sh.empty[s]), st.round ^ 1, waits);
                    if (!ok) break;
                    if (h_cols) {
#pragma unroll
                        for (int i = 0; i < kRows; ++i) {
                            const unsigned word[2] = {code[d][i].x, code[d][i].y};
                            uint32_t b[4];
                            ckpt_decode_bf16(word, ckpt_scale(scale[d][i]), b);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + h_at + i * h_apart), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]) : "memory");
                        }
                    }
                    ask(code[d], scale[d], hi - r - kAhead * p.step);
                    if (rows % 16) {
                        ok = warp_wait(smem_addr(&sh.full[s]), st.round, waits);
                        if (!ok) break;
                        clear(at, rows, p.h_panels, p.h_panels + panels, me, kMakers * 32);   // h's rows are zeros already
                    }
                    async_proxy_fence();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_addr(&sh.made[s]));
                    st.next(p.stages);
                }
            }
        }
    }
    __syncwarp();
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (sh.failed) {
        if (threadIdx.x == 0) drain_copies(sh.full, p.stages, sh.filled);
        if (warp == 1) drain_products(&sh.done);
        weight_gave_up(p, sh.table);
    }
    if (warp == 1) tmem_free(tmem);
    if (threadIdx.x == 0 && sh.failed && p.flag) *p.flag = 1;
}

// The records of group g, for every thread of the block: from, from + 1, ... (the group's rows as group_table reads them: the largest
// offset so far).
struct Records {
    long long from;
    int count;
};
__device__ __forceinline__ Records group_records(const int64_t *__restrict__ offsets, int g, long long n, int chunk_rows) {
    long long lo = 0;
    if (offsets) {
        for (int j = threadIdx.x & 31; j <= g; j += 32) lo = max(lo, (long long)__ldg(reinterpret_cast<const long long *>(offsets) + j));
        for (int d = 16; d > 0; d >>= 1) lo = max(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    }
    lo = min(lo, n);
    const long long hi = offsets ? min(max(lo, (long long)__ldg(reinterpret_cast<const long long *>(offsets) + g + 1)), n) : n;
    const long long first = lo / chunk_rows;
    return {first + g, hi > lo ? (int)((hi - 1) / chunk_rows - first) + 1 : 0};
}

// The column sums of a group's dz: its records' shares in order.  One launch ahead of the next kernel where that has many outputs: it
// needs the sums in every row of dW, and added up there they would be read d_in times.
__global__ void __launch_bounds__(512) grouped_sums_reduce_kernel(const int64_t *__restrict__ offsets, long long n, int d_out, int chunk_rows, int shares,
                                                                  const float *__restrict__ sums, float *__restrict__ total) {
    after_predecessor();
    const int g = blockIdx.y;
    const Records r = group_records(offsets, g, n, chunk_rows);
    __shared__ float red[16][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float acc = 0.f;
    if (c < d_out) {
#pragma unroll 4
        for (int s = w; s < r.count * shares; s += 16) acc += sums[(r.from * shares + s) * d_out + c];
    }
    red[w][lane] = acc;
    __syncthreads();
    if (w != 0 || c >= d_out) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) acc += red[k][lane];
    total[(long long)g * d_out + c] = acc;
}

// dW[g] = the sum of group g's records, times gamma, plus beta times the sums of dz's columns.  4 outputs a thread; SHARES warps share
// the records of the same outputs where there are too few outputs to fill the device (the order is fixed either way).  turned: the
// records are dW's transpose, [d_in][d_out] here with the names swapped.
template <int SHARES>
__global__ void __launch_bounds__(SHARES == 32 ? 1024 : 256) grouped_weight_reduce_kernel(const int64_t *__restrict__ offsets, long long n, int d_in, int d_out, int chunk_rows,
                                                                    const float *__restrict__ part, const float *__restrict__ sums, int sum_shares,
                                                                    const float *__restrict__ gamma, const float *__restrict__ beta, bool turned, float *__restrict__ dw) {
    after_predecessor();
    constexpr int kAcross = SHARES == 1 ? 256 : 32;
    const int g = blockIdx.y;
    const Records r = group_records(offsets, g, n, chunk_rows);
    __shared__ float4 red[SHARES][kAcross], red_col[SHARES][kAcross];
    const int lane = threadIdx.x % kAcross, share = threadIdx.x / kAcross;
    const long long size = (long long)d_in * d_out, x = (blockIdx.x * (long long)kAcross + lane) * 4;
    const int row = (int)(x / d_out), c = (int)(x - (long long)row * d_out);
    const auto add = [](float4 &a, const float4 &b) { a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w; };
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f), col = acc;
    if (x < size) {
        const float *at = part + r.from * size + x;
#pragma unroll 8
        for (int s = share; s < r.count; s += SHARES) add(acc, *reinterpret_cast<const float4 *>(at + s * size));
        if (sums) {
            if constexpr (SHARES > 1) {   // few outputs: the records' column sums are added up here as well
#pragma unroll 4
                for (int s = share; s < r.count * sum_shares; s += SHARES) add(col, *reinterpret_cast<const float4 *>(sums + (r.from * sum_shares + s) * d_out + c));
            } else {
                col = *reinterpret_cast<const float4 *>(sums + (long long)g * d_out + c);   // of grouped_sums_reduce_kernel
            }
        }
    }
    if constexpr (SHARES > 1) {
        red[share][lane] = acc;
        red_col[share][lane] = col;
        __syncthreads();
        if (share != 0) return;
#pragma unroll
        for (int k = 1; k < SHARES; ++k) add(acc, red[k][lane]), add(col, red_col[k][lane]);
    }
    if (x >= size) return;
    if (gamma) {
        const float k = __ldg(gamma + row);
        acc.x *= k, acc.y *= k, acc.z *= k, acc.w *= k;
    }
    if (sums) {
        const float k = __ldg(beta + row);
        acc.x = fmaf(k, col.x, acc.x), acc.y = fmaf(k, col.y, acc.y), acc.z = fmaf(k, col.z, acc.z), acc.w = fmaf(k, col.w, acc.w);
    }
    if (turned) {
        float *to = dw + g * size + (long long)c * d_in + row;
        to[0] = acc.x, to[d_in] = acc.y, to[2ll * d_in] = acc.z, to[3ll * d_in] = acc.w;
    } else {
        *reinterpret_cast<float4 *>(dw + g * size + x) = acc;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------
constexpr int kSms = 148;
constexpr size_t kSharedMost = 227 * 1024;

static sar_status grouped_check(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, sar_dtype t, const int64_t *offsets, std::initializer_list<const void *> ps) {
    if (n < 0 || groups < 1 || d_in < 1 || d_out < 1 || (!offsets && groups > 1)) return SAR_ERR_INVALID_ARG;
    if (t != SAR_BF16) return t == SAR_F32 ? SAR_ERR_UNSUPPORTED : SAR_ERR_INVALID_ARG;
    if (n > INT32_MAX - 2048 || groups > kGroupsMax || d_in % 8 || d_out % 8 || d_in > (1 << 20) || d_out > (1 << 20)) return SAR_ERR_UNSUPPORTED;
    if (offsets && !sar_aligned(offsets, 8)) return SAR_ERR_ALIGNMENT;
    for (const void *p : ps)
        if (!p) return SAR_ERR_INVALID_ARG;
        else if (!sar_aligned(p, 16)) return SAR_ERR_ALIGNMENT;
    return SAR_OK;
}

static bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes) {
    const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
    return x < y + b_bytes && y < x + a_bytes;
}
// a result over the rows or the weights: other blocks may still have to read them
static sar_status grouped_apart(int64_t n, int64_t groups, int64_t d_in, int64_t d_out, const void *rows, int64_t d_rows, const void *w, const void *out, int64_t d_result) {
    return overlap(out, n * d_result * 2, rows, n * d_rows * 2) || overlap(out, n * d_result * 2, w, groups * d_in * d_out * 2) ? SAR_ERR_INVALID_ARG : SAR_OK;
}

static int round_up_int(int x, int a) { return (x + a - 1) / a * a; }

// out [n, N] = rows [n, K] times W[g] (WT: its transpose)
template <bool WT>
static sar_status grouped_rows(int64_t n, int32_t groups, int K, int N, const int64_t *offsets, const void *rows, const void *w, void *out, uint32_t flags,
                               int32_t *flag, cudaStream_t st, const char *name) {
    RowsArgs p{};
    p.offsets = offsets;
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.flag = flag;
    p.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    p.n = (int)n;
    p.G = groups;
    p.K = K;
    p.N = N;
    p.zero_rest = (flags & SAR_GROUPED_ZERO_REST) != 0;
    p.steps = (K + kStep - 1) / kStep;
    // Weights stay in shared memory where 128 KB hold 192 columns of them and more: every row tile then costs the loads of its rows
    // alone (300,000 rows, 264 x 264: 85 us, through the ring 120).  Longer contractions take both operands through the ring: narrower
    // slices that stay read the rows again (500,000 rows, 512 x 512: slices of 128 that stay 382 us, of 256 through the ring 236).
    const int widest = p.steps == 5 ? 192 : 256;
    const bool stay = p.steps <= 5;
    p.slices = (N + widest - 1) / widest;
    p.cols = round_up_int((N + p.slices - 1) / p.slices, 64);
    p.slices = (N + p.cols - 1) / p.cols;
    const size_t w_step = (size_t)(p.cols / 64) * kPanel, w_set = p.steps * w_step, row_stage = kTileRows * 128;
    p.store_bufs = stay && p.steps * p.cols < 4 * 256 ? 2 : 1;   // where the weights take 128 KB a second buffer costs a stage of four
    const size_t fixed = sizeof(RowsShared) + 1024 + 4 * p.store_bufs * kStoreBuf;
    size_t smem;
    if (stay) {
        const size_t room = kSharedMost - fixed;
        p.slots = (int)((room - 3 * row_stage) / w_set);
        p.slots = p.slots > kSlotsMax ? kSlotsMax : p.slots;
        p.stages = (int)((room - p.slots * w_set) / row_stage);
        p.stages = p.stages > kStagesMax ? kStagesMax : p.stages;
        smem = fixed + p.slots * w_set + p.stages * row_stage;
    } else {
        p.slots = 0;
        p.stages = (int)((kSharedMost - fixed) / (row_stage + w_step));
        p.stages = p.stages > kStagesMax ? kStagesMax : p.stages;
        smem = fixed + p.stages * (row_stage + w_step);
    }
    const uint64_t a_dims[2] = {(uint64_t)K, (uint64_t)n}, d_dims[2] = {(uint64_t)N, (uint64_t)n};
    const uint64_t w_dims[3] = {(uint64_t)(WT ? K : N), (uint64_t)(WT ? N : K), (uint64_t)groups};
    const uint32_t a_box[2] = {64, kTileRows}, d_box[2] = {64, 32}, w_box[3] = {64, (uint32_t)(WT ? p.cols : kStep), 1};
    SAR_TRY(tc_tensor_map(&p.a, rows, 2, a_dims, a_box));
    SAR_TRY(tc_tensor_map(&p.w, w, 3, w_dims, w_box));
    SAR_TRY(tc_tensor_map(&p.d, out, 2, d_dims, d_box));
    const long long most_tiles = (n + kTileRows - 1) / kTileRows + groups;   // what the groups' ragged ends can add
    long long teams = kSms / p.slices;
    teams = teams < 1 ? 1 : teams > most_tiles ? most_tiles : teams;
    auto kern = grouped_rows_kernel<WT>;
    SAR_TRY(ensure_smem(kern, smem));
    SAR_LAUNCH(name, st, launch_if(n * (K + N) <= kOverlapElems, kern, (unsigned)(teams * p.slices), kRowsThreads, smem, st, p));
    return sar_after_launch();
}

struct WeightPlan {
    int cols, m_tiles, n_tiles, chunks, chunk_rows, stages, step, h_panels;
    size_t smem, part_bytes, sum_bytes, total_bytes;   // the scratch: records, their column sums, the groups' column sums
};
static WeightPlan weight_plan(int64_t n, int groups, int d_in, int d_out, bool ckpt) {
    WeightPlan w;
    w.n_tiles = (d_out + 255) / 256;
    w.cols = round_up_int((d_out + w.n_tiles - 1) / w.n_tiles, 64);
    w.n_tiles = (d_out + w.cols - 1) / w.cols;
    w.m_tiles = (d_in + 127) / 128;
    const int tiles = w.m_tiles * w.n_tiles;
    long long chunks = kSms / tiles;
    if (chunks > (n + kStep - 1) / kStep) chunks = (n + kStep - 1) / kStep;   // short chunks cost a record each, but small calls wait for steps: 2,000 rows, 256 x 256, chunks of 64, 128, 256 rows and more 29, 35, 42 us
    if (chunks < 1) chunks = 1;
    const size_t records = (size_t)(chunks + groups);   // of the scratch: what follows can only take fewer, but not fewer for fewer rows
    long long rows = (n + chunks - 1) / chunks;
    rows = (rows + kStep - 1) / kStep * kStep;
    w.chunk_rows = (int)rows;
    w.chunks = (int)((n + rows - 1) / rows);
    // Twice as many rows a stage, so that a step is worth its waits, where three stages of that fit (2 million rows, 64 x 64: 99 -> 85 us,
    // from a checkpoint 144 -> 86).  The makers' shares of a stage are 64 rows of two panels of h or 128 of one.
    const size_t fixed = sizeof(WeightShared) + 1024 + kAdders * kTurnBuf;
    w.h_panels = d_in <= 64 && w.cols <= 192 ? 1 : 2;
    w.step = w.h_panels == 1 || (!ckpt && w.cols <= 128) ? kStepMost : kStep;
    const size_t stage = (size_t)(w.h_panels + w.cols / 64) * w.step * 128;
    w.stages = (int)((kSharedMost - fixed) / stage);
    w.stages = w.stages > kStagesMax ? kStagesMax : w.stages;
    w.smem = fixed + w.stages * stage;
    w.part_bytes = sar_round_up(records * d_in * d_out * 4, 256);
    w.sum_bytes = sar_round_up(records * 2 * w.m_tiles * d_out * 4, 256);
    w.total_bytes = sar_round_up((size_t)groups * d_out * 4, 256);
    return w;
}

// A tile is twice as wide as it is high, so dW^T = dz^T h can take fewer of them, and dz is read once a tile of h's columns.  It pays where
// that reading is dear, dz's rows ending in half a sector of 32 bytes, but dz is narrow, and where there are rows enough for what the
// records cost, which are written to dW across its rows.  us, as they lie and turned: 300,000 rows of one group 136 x 72 50 / 39,
// 168 x 24 45 / 38, 264 x 40 61 / 56, 456 x 72 88 / 72; of 64 groups 56 / 48, 45 / 45, 67 / 68, 103 / 97; a million of
// 64 groups 456 x 104 294 / 218.  Not so whole sectors (200 x 48 39 / 39, 200 x 112 of 200,000 rows 36 / 39), wide dz (200 x 120 51 / 51, with 64
// groups 60 / 69; 160 x 120 40 / 45), h in whole lines (256 x 72 45 / 47), few rows (20,000 of 4 groups 136 x 72 13 / 14,
// 456 x 72 17 / 25) and many groups (100,000 rows of 64 200 x 72 29 / 35; of 8, 12,500 each, between 25 / 23 and 29 / 33).  Rows of a
// checkpoint are always the first operand, which the makers write.
static bool weight_turned(int64_t n, int groups, int d_in, int d_out) {
    if (d_in % 64 == 0 || d_out % 16 == 0 || d_out > 104 || n < 50000 || n < 2048ll * groups) return false;
    const WeightPlan a = weight_plan(n, groups, d_in, d_out, false), b = weight_plan(n, groups, d_out, d_in, false);
    return b.m_tiles * b.n_tiles < a.m_tiles * a.n_tiles;
}

static sar_status grouped_weight(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, const int64_t *offsets, const void *h, const int8_t *codes,
                                 const uint8_t *scales, const float *gamma, const float *beta, const void *dz, float *dw, int32_t *flag,
                                 void *workspace, size_t workspace_bytes, cudaStream_t st) {
    const bool turned = h && weight_turned(n, groups, d_in, d_out);
    if (turned) std::swap(d_in, d_out), std::swap(h, dz);
    const WeightPlan w = weight_plan(n, groups, d_in, d_out, !h);
    if (!workspace || !sar_aligned(workspace, 16) || workspace_bytes < w.part_bytes + w.sum_bytes + w.total_bytes) return SAR_ERR_WORKSPACE;
    WeightArgs p{};
    p.offsets = offsets;
    p.codes = codes;
    p.scales = scales;
    p.part = static_cast<float *>(workspace);
    p.sums = beta ? reinterpret_cast<float *>(static_cast<char *>(workspace) + w.part_bytes) : nullptr;
    p.flag = flag;
    p.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    p.n = (int)n;
    p.G = groups;
    p.d_in = d_in;
    p.d_out = d_out;
    p.nb = (int)ckpt_blocks(d_in);
    p.cols = w.cols;
    p.m_tiles = w.m_tiles;
    p.n_tiles = w.n_tiles;
    p.chunk_rows = w.chunk_rows;
    p.stages = w.stages;
    p.step = w.step;
    p.h_panels = w.h_panels;
    const uint32_t box[2] = {64, (uint32_t)w.step};
    const uint64_t h_dims[2] = {(uint64_t)d_in, (uint64_t)n}, z_dims[2] = {(uint64_t)d_out, (uint64_t)n};
    if (h) SAR_TRY(tc_tensor_map(&p.h, h, 2, h_dims, box));
    SAR_TRY(tc_tensor_map(&p.dz, dz, 2, z_dims, box));
    const bool early = n * (d_in + d_out) <= kOverlapElems;
    const unsigned blocks = (unsigned)(w.chunks * w.m_tiles * w.n_tiles);
    if (h) {
        SAR_TRY(ensure_smem(grouped_weight_kernel<false>, w.smem));
        SAR_LAUNCH("linear_grouped_bwd_weight", st, launch_if(early, grouped_weight_kernel<false>, blocks, kWeightThreads, w.smem, st, p));
    } else {
        SAR_TRY(ensure_smem(grouped_weight_kernel<true>, w.smem));
        SAR_LAUNCH("linear_grouped_bwd_weight_ckpt8", st, launch_if(early, grouped_weight_kernel<true>, blocks, kWeightThreads8, w.smem, st, p));
    }
    SAR_TRY(sar_after_launch());
    const long long quads = (long long)d_in * d_out / 4;
    const bool many = quads * groups >= 32 * 1024;   // outputs enough to fill the device with a thread for four
    const float *sums = p.sums;
    if (sums && many) {
        float *total = reinterpret_cast<float *>(static_cast<char *>(workspace) + w.part_bytes + w.sum_bytes);
        SAR_LAUNCH("linear_grouped_sums_reduce", st,
                   launch(grouped_sums_reduce_kernel, dim3((unsigned)((d_out + 31) / 32), (unsigned)groups), 512, 0, st, offsets, (long long)n, (int)d_out, w.chunk_rows,
                          2 * w.m_tiles, sums, total));
        SAR_TRY(sar_after_launch());
        sums = total;
    }
    const bool few = quads * groups < 4 * 1024;
    auto reduce = many ? grouped_weight_reduce_kernel<1> : few ? grouped_weight_reduce_kernel<32> : grouped_weight_reduce_kernel<8>;
    const int across = many ? 256 : 32;
    SAR_LAUNCH("linear_grouped_bwd_weight_reduce", st,
               launch(reduce, dim3((unsigned)((quads + across - 1) / across), (unsigned)groups), few ? 1024 : 256, 0, st, offsets, (long long)n, (int)d_in, (int)d_out,
                      w.chunk_rows, p.part, sums, 2 * w.m_tiles, gamma, beta, turned, dw));
    return sar_after_launch();
}

}  // namespace sar

using namespace sar;

extern "C" {

int64_t sar_set_wait_limit(int64_t cycles) { return g_wait_limit.exchange(cycles < 0 ? kWaitCycles : cycles); }

sar_status sar_linear_grouped(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, sar_dtype t, const int64_t *offsets, const void *h,
                              const void *w, void *z, uint32_t flags, int32_t *flag, void *stream) {
    if (flags & ~(uint32_t)SAR_GROUPED_ZERO_REST) return SAR_ERR_INVALID_ARG;
    if (n == 0) return grouped_check(n, groups, d_in, d_out, t, offsets, {});
    SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {h, w, z}));
    SAR_TRY(grouped_apart(n, groups, d_in, d_out, h, d_in, w, z, d_out));
    return grouped_rows<false>(n, groups, d_in, d_out, offsets, h, w, z, flags, flag, static_cast<cudaStream_t>(stream), "linear_grouped");
}

sar_status sar_linear_grouped_bwd_input(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, sar_dtype t, const int64_t *offsets,
                                        const void *dz, const void *w, void *dh, uint32_t flags, int32_t *flag, void *stream) {
    if (flags & ~(uint32_t)SAR_GROUPED_ZERO_REST) return SAR_ERR_INVALID_ARG;
    if (n == 0) return grouped_check(n, groups, d_in, d_out, t, offsets, {});
    SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {dz, w, dh}));
    SAR_TRY(grouped_apart(n, groups, d_in, d_out, dz, d_out, w, dh, d_in));
    return grouped_rows<true>(n, groups, d_out, d_in, offsets, dz, w, dh, flags, flag, static_cast<cudaStream_t>(stream), "linear_grouped_bwd_input");
}

size_t sar_linear_grouped_workspace_bytes(int64_t n, int32_t groups, int32_t d_in, int32_t d_out) {
    if (n < 1 || n > INT32_MAX || groups < 1 || d_in < 1 || d_out < 1) return 0;
    size_t most = 0;   // of rows and of a checkpoint, as they lie and turned
    for (const WeightPlan &w : {weight_plan(n, groups, d_in, d_out, true), weight_plan(n, groups, d_out, d_in, false)})
        most = w.part_bytes + w.sum_bytes + w.total_bytes > most ? w.part_bytes + w.sum_bytes + w.total_bytes : most;
    return most + 256;
}

static sar_status grouped_zero(int32_t groups, int32_t d_in, int32_t d_out, float *dw, void *stream) {
    if (!dw) return SAR_ERR_INVALID_ARG;
    SAR_CUDA_TRY(cudaMemsetAsync(dw, 0, (size_t)groups * d_in * d_out * 4, static_cast<cudaStream_t>(stream)));
    return SAR_OK;
}

sar_status sar_linear_grouped_bwd_weight(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, sar_dtype t, const int64_t *offsets,
                                         const void *h, const void *dz, float *dw, int32_t *flag, void *workspace, size_t workspace_bytes,
                                         void *stream) {
    if (n == 0) {
        SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {}));
        return grouped_zero(groups, d_in, d_out, dw, stream);
    }
    SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {h, dz, dw}));
    return grouped_weight(n, groups, d_in, d_out, offsets, h, nullptr, nullptr, nullptr, nullptr, dz, dw, flag, workspace, workspace_bytes,
                          static_cast<cudaStream_t>(stream));
}

sar_status sar_linear_grouped_bwd_weight_ckpt8(int64_t n, int32_t groups, int32_t d_in, int32_t d_out, sar_dtype t, const int64_t *offsets,
                                               const int8_t *codes, const uint8_t *scales, const float *gamma, const float *beta,
                                               const void *dz, float *dw, int32_t *flag, void *workspace, size_t workspace_bytes,
                                               void *stream) {
    if (n == 0) {
        SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {}));
        return grouped_zero(groups, d_in, d_out, dw, stream);
    }
    SAR_TRY(grouped_check(n, groups, d_in, d_out, t, offsets, {dz, dw}));
    if (!codes || !scales) return SAR_ERR_INVALID_ARG;
    if (!sar_aligned(codes, 8)) return SAR_ERR_ALIGNMENT;
    SAR_TRY(check_elem_align({gamma, beta}, 4));
    return grouped_weight(n, groups, d_in, d_out, offsets, nullptr, codes, scales, gamma, beta, dz, dw, flag, workspace, workspace_bytes,
                          static_cast<cudaStream_t>(stream));
}

}  // extern "C"
