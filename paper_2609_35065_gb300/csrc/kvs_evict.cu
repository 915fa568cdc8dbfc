// kvs_evict.cu -- eviction by accumulated attention weight: which cached tokens each head
// keeps, and their copy into new blocks.
//
// Selection is a radix selection of the J-th largest key, eight bits a pass, on the weights'
// bits in an order that compares as unsigned numbers; the tokens above it, and the first of
// those equal to it, are then written out in their own order.
#include "kvs_ops.cuh"

namespace kvs {
namespace {

constexpr int kSelect = 1024;          // threads of a selecting CTA
constexpr int kCopy = 256;

// Unsigned keys in the weights' order; NaN below all, always-kept tokens above all.
__device__ __forceinline__ uint32_t key_of(float w, int32_t t, int32_t T, const EvictJob& j) {
    if (t < j.sinks || t >= T - j.recent) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.0f);                // -0 is 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of v over the CTA's earlier threads; `total` gets the CTA's.
__device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t& total, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    uint32_t s = warp_sums[lane];                                // 32 warps
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += y;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    const uint32_t before = warp ? __shfl_sync(0xffffffffu, s, warp - 1) : 0;
    __syncthreads();
    return before + x - v;
}

__global__ void __launch_bounds__(kSelect) kvs_evict_select_kernel(EvictJob j) {
    __shared__ uint32_t hist[256], warp_sums[32], found[2];
    const StepView& st = j.step;
    const int32_t h = blockIdx.x, r = blockIdx.y, l = blockIdx.z;
    int32_t T = __ldg(st.kv_lens + r);
    if (T < 0 || T > st.max_kv) {
        if (threadIdx.x == 0) record_error(st.err, KVS_ERR_BOUNDS);
        T = 0;
    }
    const int32_t J = min(T, j.budget);
    if (h == 0 && l == 0 && threadIdx.x == 0 && j.new_lens) j.new_lens[r] = J;
    const float* w = j.weights + l * j.layer_stride + r * j.request_stride + h * j.head_stride;
    const int64_t row = (((int64_t)l * st.requests + r) * st.kv_heads + h) * j.budget;
    int32_t* kept = j.kept + row;
    float* nw = j.new_weights ? j.new_weights + row : nullptr;

    uint32_t limit = 0, equal = 0;                               // keep keys above limit, and `equal` of those at it
    if (T > J) {
        uint32_t prefix = 0, mask = 0, need = J;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int32_t t = threadIdx.x; t < T; t += kSelect) {
                const uint32_t k = key_of(w[t], t, T, j);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t left = need;
                int b = 255;
                while (hist[b] < left) left -= hist[b--];        // the counts of all bins reach `need`
                found[0] = b;
                found[1] = left;
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= 255u << shift;
            need = found[1];
            __syncthreads();
        }
        limit = prefix;
        equal = need;
    }
    uint32_t above = 0, at = 0;                                  // of the tiles before
    for (int32_t t0 = 0; t0 < T; t0 += kSelect) {
        const int32_t t = t0 + threadIdx.x;
        float x = 0.0f;
        uint32_t k = 0;
        if (t < T) {
            x = w[t];
            k = key_of(x, t, T, j);
        }
        const bool in = t < T, all = T <= J;
        const bool gt = in && (all || k > limit), eq = in && !all && k == limit;
        uint32_t total;
        const uint32_t before = scan((gt ? 1u : 0u) | (eq ? 0x10000u : 0u), total, warp_sums);
        const uint32_t g = above + (before & 0xffffu), e = at + (before >> 16);
        if (gt || (eq && e < equal)) {
            const uint32_t p = g + min(e, equal);
            kept[p] = t;
            if (nw) nw[p] = x;
        }
        above += total & 0xffffu;
        at += total >> 16;
    }
    for (int32_t p = J + threadIdx.x; p < j.budget; p += kSelect) {
        kept[p] = -1;
        if (nw) nw[p] = 0.0f;
    }
}

constexpr int kMostPlanes = 448;       // plane addresses that a launch carries

struct Planes {
    uint64_t at[kMostPlanes];
};

// A lane per 16-byte vector of a kept row of one head, K and V together; four rows in flight.
__global__ void __launch_bounds__(kCopy) kvs_evict_copy_kernel(EvictJob j, const __grid_constant__ Planes planes, int32_t layer0) {
    const StepView& st = j.step;
    const int32_t l = blockIdx.z, r = blockIdx.y, vecs = st.head_dim / 8, H = st.kv_heads;
    int32_t T = __ldg(st.kv_lens + r);
    if (T < 0 || T > st.max_kv) T = 0;
    const int64_t items = (int64_t)min(T, j.budget) * H * vecs;
    const char* kp = reinterpret_cast<const char*>(planes.at[2 * l]);
    const char* vp = reinterpret_cast<const char*>(planes.at[2 * l + 1]);
    const int32_t* kept = j.kept + ((int64_t)(layer0 + l) * st.requests + r) * H * j.budget;
    const int32_t* src_table = st.tables + (int64_t)r * st.table_stride;
    const int32_t* dst_table = j.dst_tables + (int64_t)r * j.dst_stride;
    constexpr int U = 4;
    for (int64_t i0 = (int64_t)blockIdx.x * kCopy * U + threadIdx.x; i0 < items; i0 += (int64_t)gridDim.x * kCopy * U) {
        uint4 a[U], b[U];
        int64_t to[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * kCopy;
            to[u] = -1;
            if (i < items) {
                const int32_t c = (int32_t)(i % vecs), h = (int32_t)(i / vecs % H), p = (int32_t)(i / vecs / H);
                const int64_t from = row_of(st, src_table, __ldg(kept + (int64_t)h * j.budget + p));
                to[u] = row_of(st, dst_table, p);
                a[u] = b[u] = make_uint4(0, 0, 0, 0);
                if (from >= 0) {
                    a[u] = __ldg(reinterpret_cast<const uint4*>(kp + 2 * (from + h * st.head_dim + 8 * c)));
                    b[u] = __ldg(reinterpret_cast<const uint4*>(vp + 2 * (from + h * st.head_dim + 8 * c)));
                }
                if (to[u] >= 0) to[u] += h * st.head_dim + 8 * c;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (to[u] >= 0) {
                *reinterpret_cast<uint4*>(const_cast<char*>(kp) + 2 * to[u]) = a[u];
                *reinterpret_cast<uint4*>(const_cast<char*>(vp) + 2 * to[u]) = b[u];
            }
    }
}

}  // namespace

int launch_evict(const EvictJob& j, cudaStream_t s) {
    kvs_evict_select_kernel<<<dim3(j.step.kv_heads, j.step.requests, j.layers), kSelect, 0, s>>>(j);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return -(int)e;
    int n = 1;
    const int64_t rows = j.step.max_kv < j.budget ? j.step.max_kv : j.budget;
    const int64_t ctas = (rows * j.step.kv_heads * (j.step.head_dim / 8) + kCopy * 4 - 1) / (kCopy * 4);
    for (int l0 = 0; l0 < j.layers && ctas > 0; l0 += kMostPlanes / 2, ++n) {
        const int count = j.layers - l0 < kMostPlanes / 2 ? j.layers - l0 : kMostPlanes / 2;
        Planes p{};
        for (int k = 0; k < 2 * count; ++k) p.at[k] = (uint64_t)j.planes[2 * l0 + k];
        kvs_evict_copy_kernel<<<dim3((unsigned)ctas, j.step.requests, count), kCopy, 0, s>>>(j, p, l0);
        e = cudaGetLastError();
        if (e != cudaSuccess) return -(int)e;
    }
    return n;
}

}  // namespace kvs
