// The 5th-generation tensor cores and the asynchronous copies that feed them, as thin wrappers over their PTX (internal):
// barriers in shared memory with bounded waits, tiled copies, tensor memory, and the descriptors of 128-byte swizzled tiles.
#pragma once

#include <cuda.h>

#include "sar_common.cuh"

namespace sar {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_over(uint32_t bar, uint32_t parity) {   // one look; bar_try may put the thread to sleep for a while
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits until the phase of this parity is over.  A wait that lasts longer than the limit (seconds; a tile takes microseconds)
// gives up, and so do all waits of the block after it: *failed, in shared memory, is set, and the roles leave their loops.
// With a limit of 0 a wait gives up that is not over at the first look.
constexpr long long kWaitCycles = 4000000000ll;
struct Waits {
    volatile int *failed;
    long long limit;
};
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const Waits &w) {
    if (bar_over(bar, parity)) return true;   // without a look at the limit: 156,475 rows, 296 x 16, 25.1 us with one, 23.4 without
    if (w.limit == 0) {
        *w.failed = 1;
        return false;
    }
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (bar_try(bar, parity)) return true;
        if (*w.failed) return false;
        if (clock64() - t0 > w.limit) {
            *w.failed = 1;
            return false;
        }
    }
}
// the same without regard to *failed and the limit: for what a block that has given up still has in flight
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!bar_try(bar, parity) && clock64() - t0 < kWaitCycles) {
    }
}
// the same for all lanes of a warp together
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const Waits &w) { return __all_sync(0xffffffffu, bar_wait(bar, parity, w)); }
// One lane of a warp whose lanes are all here.  Copies and products take their operands from registers that a warp shares; behind a
// test of the lane's number the compiler has to allow for several lanes with operands of their own, and goes over them one by one.
__device__ __forceinline__ bool one_lane() {
    uint32_t yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(yes));
    return yes != 0;
}
// A role's place in a ring of `size` buffers, and the parity of its present round there.  Who fills a buffer waits for the other
// parity of the buffer's `empty` barrier (a fresh barrier lets the first round pass), who reads it for this one of `full`.
struct RingPlace {
    uint32_t at = 0, round = 0;
    __device__ __forceinline__ void next(uint32_t size) {
        if (++at == size) at = 0, round ^= 1;
    }
};
__device__ __forceinline__ void bar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory"); }
// writes of this thread to shared memory before asynchronous reads of it (copies out, tensor cores)
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }

// ---- tiled copies ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tile_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tile_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void map_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];\n" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tile_store_2d(const CUtensorMap *map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
template <int N>   // all but the last N groups have read their shared memory
__device__ __forceinline__ void store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(N) : "memory");
}
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }

// ---- tensor memory and products ----------------------------------------------------------------------------------------------
constexpr int kTmemCols = 512;   // all of an SM's: a block of these kernels has the SM to itself
__device__ __forceinline__ void tmem_alloc(uint32_t where) {   // a whole warp; the address is written to shared memory
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(where), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n");
}
__device__ __forceinline__ void tmem_free(uint32_t at) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(at), "r"(kTmemCols)); }
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
// D (+)= A B for one step of 16 along the contraction: bf16 operands in shared memory, float32 in tensor memory; one thread issues it
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(instr),
                 "r"((uint32_t)accumulate)
                 : "memory");
}
// the barrier gets an arrival when all products that this thread has issued are done
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
// What a block that has given up still has in flight ends before the block does: the copies into `filled` buffers of a ring of `size`
// (by any one thread), and the products of the thread that issued them (by its whole warp; `done`: a barrier of one arrival that
// nothing else uses).  A role that has come to its end may have left copies or products behind that others have given up
// waiting for, so this follows the last barrier of all roles.
__device__ __forceinline__ void drain_copies(const uint64_t *full, uint32_t size, uint32_t filled) {
    for (uint32_t s = 0; s < size && s < filled; ++s) bar_drain(smem_addr(&full[s]), ((filled - 1 - s) / size) & 1);
}
__device__ __forceinline__ void drain_products(uint64_t *done) {
    if (one_lane()) tc_commit(smem_addr(done));
    __syncwarp();
    bar_drain(smem_addr(done), 0);
    tc_after_sync();
}
// Columns of the warp's 32 lanes: thread l has columns at, at + 1, ... of lane l (the lanes that warp % 4 may reach).  The
// registers of a load may be used after tmem_wait_load, through which they pass, so that no use of them is moved before it.
__device__ __forceinline__ void tmem_ask(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_tie(uint32_t (&r)[32]) { asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])); }
__device__ __forceinline__ void tmem_wait_load(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
    tmem_tie(r);
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// Operands lie in shared memory as tiled copies leave them: rows of 128 bytes (64 bf16), the 16-byte chunk c of row r at chunk
// c ^ (r & 7) (128-byte swizzle), tiles on 1024-byte boundaries.  Two readings of such a tile:
//   contraction along the 128 bytes (K-major): groups of 8 rows follow at `group` bytes; a step of 16 is 32 bytes further on;
//   contraction along the rows (MN-major): groups of 8 rows follow at 1024 bytes, the next 64 columns at `panel` bytes; a step
//   of 16 is 16 rows, 2048 bytes, further on.
__device__ __forceinline__ uint64_t tc_operand(uint32_t at, uint32_t leading, uint32_t stride) {
    return (uint64_t)((at & 0x3ffffu) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// the same operand `bytes` further on (a multiple of 16; the address is the descriptor's lowest field)
__device__ __forceinline__ uint64_t tc_advance(uint64_t operand, uint32_t bytes) { return operand + (bytes >> 4); }
// float32 += bf16 x bf16, 128 rows, `cols` columns (a multiple of 16 up to 256)
__host__ __device__ constexpr uint32_t tc_instr(int cols, bool a_mn, bool b_mn) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (uint32_t)(cols >> 3) << 17 | (128u >> 4) << 24;
}

// ---- host: tensor maps -------------------------------------------------------------------------------------------------------
// bf16 array of `rank` dimensions, innermost first, dense; tiles of box[] elements (64 innermost) with the 128-byte swizzle
sar_status tc_tensor_map(CUtensorMap *map, const void *base, int rank, const uint64_t *dims, const uint32_t *box);

}  // namespace sar
