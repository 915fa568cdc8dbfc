// kvs_ops.cuh -- device arithmetic shared by the model operators' kernels.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kvs_job.cuh"
#include "kvs_ops.h"

namespace kvs {
namespace {

__device__ __forceinline__ void record_error(int32_t* err, int32_t code) { atomicCAS(err, 0, code); }

// One request's rows and lengths.  Anything outside the step's bounds leaves it without
// rows and without cached tokens, and is recorded.
struct Request {
    int32_t q0, n, T;      // first row, new tokens, cached tokens
};

// fetch_request starts the loads, check_request needs them.
struct RawRequest {
    int32_t T, q0, end;
};
__device__ __forceinline__ RawRequest fetch_request(const StepView& st, int32_t r) {
    RawRequest w;
    w.T = __ldg(st.kv_lens + r);
    w.q0 = st.q_starts ? __ldg(st.q_starts + r) : r;
    w.end = st.q_starts ? __ldg(st.q_starts + r + 1) : r + 1;
    return w;
}
__device__ __forceinline__ Request check_request(const StepView& st, const RawRequest& w) {
    Request q{w.q0, w.end - w.q0, w.T};
    if (w.q0 < 0 || w.end < w.q0 || w.end > st.total_q || w.end - w.q0 > st.max_q || w.T < 0 || w.T > st.max_kv) {
        record_error(st.err, KVS_ERR_BOUNDS);
        q.q0 = q.n = q.T = 0;
    }
    return q;
}
__device__ __forceinline__ Request load_request(const StepView& st, int32_t r) { return check_request(st, fetch_request(st, r)); }

__device__ __forceinline__ uint32_t block_of(const StepView& st, uint32_t t) {
    return (uint32_t)(((uint64_t)t * st.block_m) >> st.block_p);
}

// Token and query head (of the KV head's) of a packed row.
__device__ __forceinline__ int32_t token_of(const StepView& st, int32_t p, int32_t& g) {
    const int32_t t = (int32_t)(((uint64_t)(uint32_t)p * st.group_m) >> st.group_p);
    g = p - t * st.group;
    return t;
}

// Element offset of cached token t's row in a plane; negative (and recorded) where the
// table names a block that the cache does not have.
__device__ __forceinline__ int64_t row_of(const StepView& st, const int32_t* table, uint32_t t) {
    const uint32_t k = block_of(st, t);
    const int32_t b = __ldg(table + k);
    if ((uint32_t)b >= (uint32_t)st.num_blocks) {
        record_error(st.err, KVS_ERR_BOUNDS);
        return -1;
    }
    return ((int64_t)b * st.block_size + (t - k * st.block_size)) * st.kv_heads * st.head_dim;
}

// Cached tokens [lo, hi) that new tokens i0 .. i1 (inclusive) of the request see at most.
struct Span {
    int32_t lo, hi;
};
__device__ __forceinline__ Span seen_by(const Request& q, int32_t i0, int32_t i1, int32_t causal, int32_t window) {
    Span s;
    s.hi = causal ? min(q.T, q.T - q.n + i1 + 1) : q.T;
    s.lo = window > 0 ? max(0, q.T - q.n + i0 + 1 - window) : 0;
    if (s.hi < s.lo) s.hi = s.lo;
    return s;
}

template <bool HALF>
struct Num;
template <>
struct Num<false> {
    using T = __nv_bfloat16;
    using T2 = __nv_bfloat162;
    static __device__ __forceinline__ float to(T x) { return __bfloat162float(x); }
    static __device__ __forceinline__ T from(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ float2 to2(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<T2*>(&w)); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const T2 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};
template <>
struct Num<true> {
    using T = __half;
    using T2 = __half2;
    static __device__ __forceinline__ float to(T x) { return __half2float(x); }
    static __device__ __forceinline__ T from(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ float2 to2(uint32_t w) { return __half22float2(*reinterpret_cast<T2*>(&w)); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const T2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};

// Attention weights in half are multiples of 2^-24, and none is above 65504: log2 of what the
// heaviest of `tokens` is scaled to, so that a long cache's light ones are not lost beside it.
// What their rounding takes from a sum is then below 2^-15 of the largest value (half's own
// rounding is 2^-11), and above this lie 2^(16 - top) for weights that outgrow the reference.
__device__ __forceinline__ float half_top(int32_t tokens, int32_t least) { return (float)min(10, max(least, 22 - __clz(tokens))); }

// 2^x by the hardware's approximation (relative error about 2^-22); 0 at -infinity.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Of shared memory in the cluster's CTA `rank`, at this CTA's address.
__device__ __forceinline__ uint32_t cluster_at(uint32_t addr, int rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    return at;
}
__device__ __forceinline__ float2 cluster_ld2(uint32_t at) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
// All threads of all of the cluster's CTAs; what they wrote before is seen behind it.
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory"); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
    const int n = there ? 16 : 0;      // 0: the 16 bytes become zeros, src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

}  // namespace
}  // namespace kvs
