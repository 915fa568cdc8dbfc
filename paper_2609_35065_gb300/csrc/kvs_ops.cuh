// kvs_ops.cuh -- device arithmetic shared by the model operators' kernels.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kvs_job.cuh"
#include "kvs_ops.h"

namespace kvs {
namespace {

// A load of something that no kernel writes while this one runs.  LATE: a kernel that is launched programmatically
// (launch_behind) is there while the one before it still writes: its loads have to be coherent.
template <bool LATE, class T>
__device__ __forceinline__ T load_of(const T* p) {
    return LATE ? *p : __ldg(p);
}

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
template <bool LATE = false>
__device__ __forceinline__ RawRequest fetch_request(const StepView& st, int32_t r) {
    RawRequest w;
    w.T = load_of<LATE>(st.kv_lens + r);
    w.q0 = st.q_starts ? load_of<LATE>(st.q_starts + r) : r;
    w.end = st.q_starts ? load_of<LATE>(st.q_starts + r + 1) : r + 1;
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
template <bool LATE = false>
__device__ __forceinline__ Request load_request(const StepView& st, int32_t r) { return check_request(st, fetch_request<LATE>(st, r)); }

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
template <bool LATE = false>
__device__ __forceinline__ int64_t row_of(const StepView& st, const int32_t* table, uint32_t t) {
    const uint32_t k = block_of(st, t);
    const int32_t b = load_of<LATE>(table + k);
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

// A window with sinks leaves the first tokens and the last ones visible, and blocks between them may
// be gone.  The kernels go over such a cache as if it had no others: place u is token u below `cut`
// and token u + shift behind it.  Places hold whole units of tokens, a unit being what one load
// brings of a block, so a few tokens that nobody sees are among them: those of [sinks, lo - shift).
struct Held {
    int32_t cut, shift;
};
__device__ __forceinline__ Held held_of(int32_t lo, int32_t sinks, int32_t unit) {
    const int32_t first = unit > 1 ? lo / unit * unit : lo, some = min(sinks, lo);
    const int32_t cut = min(unit > 1 ? (some + unit - 1) / unit * unit : some, first);
    return Held{cut, first - cut};
}
__device__ __forceinline__ int32_t token_at(const Held& h, int32_t u) { return u < h.cut ? u : u + h.shift; }
// Where shift > 0, cut is at least `sinks`: so in places, too, a row sees [lo, hi) and [0, sinks) of it.
__device__ __forceinline__ Span in_places(const Held& h, Span s) {
    // a row that sees nothing has lo = 0 in a request that has no shift
    s.lo -= h.shift;
    s.hi -= h.shift;
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
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool there) {
    const int n = there ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

// The attributes of a launch: `cluster` CTAs in x to a cluster (at most 1: none), and whether it is made behind
// the stream's previous kernel, as by launch_behind.
unsigned launch_attributes(cudaLaunchAttribute (&at)[2], unsigned cluster, bool behind) {
    unsigned n = 0;
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = cluster;
        at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
        ++n;
    }
    if (behind) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    return n;
}

// Launches a kernel programmatically: its CTAs are in place as those of the stream's previous kernel end, which is
// 2 us of every call among others (a decode step of 16 sessions' weights 34.8 -> 31.9 us, attention of one session
// 8.3 -> 6.6).  Such a kernel begins with grid_wait() in every thread, before any load, store or trigger
// of its own, so that whatever it sets off starts behind all that was before it; its loads are load_of<true>.
template <class... P, class... A>
cudaError_t launch_behind(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, const A&... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[2];
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = launch_attributes(at, 1, true);
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace
}  // namespace kvs
