// kvs_tcgen05.cuh -- the fifth-generation tensor cores (tcgen05.mma with accumulators in
// tensor memory) and tiled TMA loads, as inline PTX.
//
// Operand tiles in shared memory are rows of 64 16-bit elements (128 bytes) in the 128-byte
// swizzle: the 16-byte vector c of row r lies at r * 128 + ((c ^ (r & 7)) << 4) from a
// 1024-byte aligned base.  Wider rows are further such tiles behind.
#pragma once

#include <cstdint>
#include <cuda.h>

#include "kvs_async.cuh"
#include "kvs_ops.cuh"

namespace kvs {
namespace {

// ---- tensor memory -----------------------------------------------------------
// A whole warp allocates (columns: a power of two from 32 to 512); the address lands in shared memory.
__device__ __forceinline__ void tmem_alloc(uint32_t smem_out, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_out), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Generic writes to shared memory before this are seen by the tensor cores and TMA after it.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

#define KVS_R8(r, k) "=r"(r[k]), "=r"(r[k + 1]), "=r"(r[k + 2]), "=r"(r[k + 3]), "=r"(r[k + 4]), "=r"(r[k + 5]), "=r"(r[k + 6]), "=r"(r[k + 7])
#define KVS_I8(r, k) "r"(r[k]), "r"(r[k + 1]), "r"(r[k + 2]), "r"(r[k + 3]), "r"(r[k + 4]), "r"(r[k + 5]), "r"(r[k + 6]), "r"(r[k + 7])
#define KVS_U8(r, k) "+r"(r[k]), "+r"(r[k + 1]), "+r"(r[k + 2]), "+r"(r[k + 3]), "+r"(r[k + 4]), "+r"(r[k + 5]), "+r"(r[k + 6]), "+r"(r[k + 7])

// 32 columns of the thread's lane (a warp reads lanes 32 (warp % 4) ...); valid after tmem_wait_ld.
__device__ __forceinline__ void tmem_ld32(uint32_t* r, uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : KVS_R8(r, 0), KVS_R8(r, 8), KVS_R8(r, 16), KVS_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        :: KVS_I8(r, 0), KVS_I8(r, 8), KVS_I8(r, 16), KVS_I8(r, 24), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t* r, uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : KVS_R8(r, 0), KVS_R8(r, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 :: KVS_I8(r, 0), KVS_I8(r, 8), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Keeps the compiler from using r[0..32) before the wait that this stands behind.
__device__ __forceinline__ void tmem_loaded32(uint32_t* r) {
    asm volatile("" : KVS_U8(r, 0), KVS_U8(r, 8), KVS_U8(r, 16), KVS_U8(r, 24) :: "memory");
}
__device__ __forceinline__ void tmem_loaded16(uint32_t* r) { asm volatile("" : KVS_U8(r, 0), KVS_U8(r, 8) :: "memory"); }

__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// ---- matrix products ---------------------------------------------------------
// Shared-memory operand.  K-major (rows are M or N, contiguous in K): stride = bytes between
// groups of eight rows.  MN-major (rows are K, contiguous in M or N): stride = bytes between
// groups of eight K rows, lead = bytes between groups of 64 columns.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 |
           1ull << 46 | 2ull << 61;
}
// 16-bit operands, 32-bit accumulators, M = 128.  kNegA: the products' sign is turned.
constexpr uint32_t kNegA = 1u << 13;
__host__ __device__ constexpr uint32_t tc_idesc(bool half, int n, bool b_mn_major) {
    return 1u << 4 | (half ? 0u : 1u) << 7 | (half ? 0u : 1u) << 10 | (b_mn_major ? 1u : 0u) << 16 | (uint32_t)(n / 8) << 17 | 8u << 24;
}
// The operand `bytes` further on.
__device__ __forceinline__ uint64_t tc_ahead(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }
// The warp's number, as a value that the compiler knows to be the same in all lanes: what
// follows from it may then live in uniform registers, where tcgen05.mma takes its operands.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0); }
// One lane of a converged warp, the same at every call.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// d (+)= a b over 16 elements of K, both operands in shared memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// ... with a in tensor memory: lane = row, two elements to a column.
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// One arrival on `bar` when all products that this thread issued are done.
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}

// ---- tiled loads of the paged planes -----------------------------------------
// A box of [rows of a block][64 elements of one head]; the plane's map is [NB][B][H][D].  A
// coordinate beyond the plane (a head dim's end, a block that there is not) reads as zeros.
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int32_t d, int32_t h, int32_t t, int32_t b, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        :: "r"(dst), "l"(map), "r"(bar), "r"(d), "r"(h), "r"(t), "r"(b) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int32_t d, int32_t h, int32_t n, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        :: "r"(dst), "l"(map), "r"(bar), "r"(d), "r"(h), "r"(n) : "memory");
}

// 128 cached tokens from t0 of one KV head, as a tile at dst; tokens beyond the cache's last
// block are left as they are.  By boxes: WARPS warps, of which this is w, take a share of them
// each -- issuing one takes a warp about 120 cycles -- and arrive on `bar` with its bytes.  A
// lane's box is known ahead of the tile (box_of), so that its table entry is there when it is.
struct Box {
    int32_t block, row, at;                                      // block (num_blocks: reads as zeros), first token in it, token of the tile
};
template <int DP, int WARPS>
__device__ __forceinline__ Box box_of(const StepView& st, const int32_t* table, int32_t t0, int32_t T, int w, int lane) {
    constexpr int HALVES = DP / 64;
    const int32_t size = min(st.block_size, 128), i = (lane / HALVES) * WARPS + w;      // this lane's box of the tile
    Box x{-1, 0, i * size};
    const int32_t tok = t0 + x.at;
    if (x.at < 128 && tok < T) {
        const uint32_t blk = block_of(st, tok);
        x.block = __ldg(table + blk);
        x.row = tok - blk * st.block_size;
        if ((uint32_t)x.block >= (uint32_t)st.num_blocks) {
            record_error(st.err, KVS_ERR_BOUNDS);
            x.block = st.num_blocks;
        }
    }
    return x;
}
template <int DP>
__device__ __forceinline__ void tile_boxes(uint32_t dst, const CUtensorMap* map, const StepView& st, int32_t h, const Box& x, uint32_t bar, int lane) {
    constexpr int HALVES = DP / 64;
    const int count = __popc(__ballot_sync(0xffffffffu, x.block >= 0));
    if (lane == 0) mbar_expect_tx(bar, (uint32_t)count * min(st.block_size, 128) * 128);
    __syncwarp();
    if (x.block >= 0) {
        const int c = lane % HALVES;
        tma_load_4d(dst + c * 128 * 128 + x.at * 128, map, 64 * c, h, x.row, x.block, bar);
    }
    __syncwarp();
}
// By rows: THREADS threads, of which this is t, with cp.async; tokens outside [lo, hi) become zeros.
template <int DP, int THREADS = 128>
__device__ __forceinline__ void tile_rows(uint32_t dst, const char* plane, const StepView& st, const int32_t* table, int32_t h, int32_t t0, int32_t lo, int32_t hi,
                                          int t) {
    constexpr int CH = DP / 8;                                   // 16-byte vectors of a row
#pragma unroll 4
    for (int v = t; v < 128 * CH; v += THREADS) {
        const int k = v / CH, c = v % CH;
        const int32_t tok = t0 + k;
        const int64_t row = tok >= lo && tok < hi ? row_of(st, table, tok) : -1;
        const bool there = row >= 0 && 8 * c < st.head_dim;
        cp_async16(dst + (c >> 3) * 128 * 128 + k * 128 + (((c & 7) ^ (k & 7)) << 4),
                   plane + (there ? 2 * (row + (int64_t)h * st.head_dim + 8 * c) : 0), there);
    }
}

// Barrier of `threads` threads under a number of its own (1 to 15).
__device__ __forceinline__ void bar_some(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// (a0, a1) * (b, b) + (c, c), and sums, two binary32 numbers at a time.
__device__ __forceinline__ void fma2(float& x, float& y, float b, float c) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %2};\n\tmov.b64 r, {%3, %3};\n\t"
        "fma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(x), "+f"(y) : "f"(b), "f"(c));
}
// The same, and whether any of them says so.
__device__ __forceinline__ bool bar_or(int id, int threads, bool p) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbar.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(id), "r"(threads), "r"((uint32_t)p) : "memory");
    return r != 0;
}

// (x, y) * (b, b) + (c, d)
__device__ __forceinline__ void fma2(float& x, float& y, float b, float c, float d) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %2};\n\tmov.b64 r, {%3, %4};\n\t"
        "fma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(x), "+f"(y) : "f"(b), "f"(c), "f"(d));
}
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\t"
        "add.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}

}  // namespace
}  // namespace kvs
