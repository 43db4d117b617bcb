// Tensor memory, tensor-core products, tiled copies and barriers of sm_100a, as the PTX instructions that they are.
//
// Every wait has an end: where a barrier is not passed within some cycles (Waits::limit) the block's `stop` word is set, every other wait of
// the block sees it, and the block winds up.  What it has in flight it waits for even then (bw_wait_end), before its memory is another's.
#pragma once

#include <cuda.h>
#include <stdint.h>

__device__ __forceinline__ uint32_t bw_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers ------------------------------------------------------------------------------
__device__ __forceinline__ void bw_bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bw_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// An arrival of a whole warp: what its lanes have done is done.
__device__ __forceinline__ void bw_arrive_warp(uint32_t bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bw_arrive(bar);
    __syncwarp();                                                 // (together again: what follows may be for whole warps only)
}
__device__ __forceinline__ void bw_arrive_expect(uint32_t bar, uint32_t bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }

__device__ __forceinline__ bool bw_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}

// In shared memory, of a block: whether a wait was given up, and the cycles that one may take.
struct Waits {
    int stop;
    long long limit;
};

// What is in flight comes to its end, or two hundred million cycles (a tenth of a second) pass: the block has given up already.
__device__ __noinline__ void bw_wait_end(uint32_t bar, uint32_t parity) {
    const long long begin = clock64();
    while (!bw_try(bar, parity) && clock64() - begin <= 200000000ll) {}
}
// False: given up, here or elsewhere in the block.  For a whole warp: all of its lanes go on or none does.  They come together first: lanes that wait may keep the others
// of their warp from running, so none of them may still have something to do that the barrier waits for.
__device__ __noinline__ bool bw_wait_slow_warp(uint32_t bar, uint32_t parity, volatile Waits* w) {
    const long long begin = clock64(), limit = w->limit;
    while (!__all_sync(~0u, bw_try(bar, parity))) {
        if (__any_sync(~0u, w->stop || clock64() - begin > limit)) { w->stop = 1; return false; }
    }
    return true;
}
__device__ __forceinline__ bool bw_wait_warp(uint32_t bar, uint32_t parity, volatile Waits* w) {
    __syncwarp();
    if (__all_sync(~0u, bw_try(bar, parity))) return true;
    return bw_wait_slow_warp(bar, parity, w);
}

__device__ __forceinline__ void bw_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }   // plain writes before what the tensor cores and copies do

// ---- tiled copies --------------------------------------------------------------------------
__device__ __forceinline__ void bw_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void bw_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void bw_prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// ---- tensor memory -------------------------------------------------------------------------
__device__ __forceinline__ void bw_tmem_alloc(uint32_t where, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void bw_tmem_free(uint32_t at, uint32_t columns) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory"); }
__device__ __forceinline__ void bw_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void bw_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// What was loaded is there: nothing that uses it is moved before the wait.
__device__ __forceinline__ void bw_wait_ld32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), 
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), 
                   "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 ::"memory");
}
__device__ __forceinline__ void bw_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the lane of each thread of a warp (the lanes of tensor memory that belong to the warp).
__device__ __forceinline__ void bw_ld32(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void bw_ld16(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at));
}
__device__ __forceinline__ void bw_wait_ld16(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ void bw_st16(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at) : "memory");
}
__device__ __forceinline__ void bw_ld8(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at));
}
__device__ __forceinline__ void bw_wait_ld8(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])::"memory");
}
__device__ __forceinline__ void bw_st8(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t bw_ld1(uint32_t at) {
    uint32_t x;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(x) : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(x)::"memory");
    return x;
}
__device__ __forceinline__ void bw_st32(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
                   "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
                   "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at) : "memory");
}

// ---- products ------------------------------------------------------------------------------
// Operands in shared memory lie in rows of 128 bytes (64 elements), eight rows a swizzle atom of 1,024 bytes: 16-byte piece c of row r
// at r * 128 + ((c ^ r % 8) * 16).  K-major: rows are those of the operand, its depth runs along a row.  Depth-major ("across"): rows
// run along the depth, and the next 64 of the other dimension lie `next` bytes on.
__device__ __forceinline__ uint64_t bw_desc(uint32_t addr) {                       // K-major
    return (uint64_t)(addr >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ uint64_t bw_desc_across(uint32_t addr, uint32_t next) {
    return (uint64_t)(addr >> 4) | (uint64_t)(next >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 16-bit operands (bf16 or fp16, both alike), 32-bit sums, M rows and N columns; `minus_a`: of the first operand negated.
__device__ __forceinline__ constexpr uint32_t bw_idesc(bool bf16, int M, int N, bool b_across, bool minus_a) {
    return 1u << 4 | (minus_a ? 1u << 13 : 0u) | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_across ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
// Called by a whole warp that stays together (so that operands are computed once for it); `leader`: one of its lanes, which issues.
__device__ __forceinline__ void bw_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add, bool leader) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)leader) : "memory");
}
// A from tensor memory: two elements a column.
__device__ __forceinline__ void bw_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add, bool leader) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)leader) : "memory");
}
// The barrier is arrived at when all products that the leader has issued are done.
__device__ __forceinline__ void bw_commit(uint32_t bar, bool leader) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"((uint32_t)leader) : "memory");
}
__device__ __forceinline__ bool bw_elect() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is;
}
