// kvs_evict.cu -- eviction by accumulated attention weight: which cached tokens each head
// keeps, and their copy into new blocks.
//
// Selection is a radix selection of the J-th largest key, in digits of 11, 11 and 10 bits, on
// the weights' bits in an order that compares as unsigned numbers; the tokens above it, and the
// first of those equal to it, are then written out in their own order.
#include "kvs_async.cuh"
#include "kvs_ops.cuh"

namespace kvs {
namespace {

constexpr int kSelect = 1024;          // threads of a selecting CTA
constexpr int kOwn = 8;                // consecutive tokens of a thread
constexpr int kBins = 2048;
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
    __syncthreads();                                             // the sums of the scan before are read
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    uint32_t s = warp_sums[lane];                                // 32 warps
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += y;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, s, warp ? warp - 1 : 0);
    return (warp ? before : 0) + x - v;
}

// One CTA per (head, request, layer).  A cache of up to 8192 tokens stays in registers, eight
// consecutive ones to a thread; a longer one is read again, from L2, by each pass.
__global__ void __launch_bounds__(kSelect) kvs_evict_select_kernel(EvictJob j) {
    __shared__ uint32_t hist[kBins], warp_sums[32], found[2];
    const StepView& st = j.step;
    const int32_t h = blockIdx.x, r = blockIdx.y, l = blockIdx.z;
    grid_trigger();                                              // the copy may come and wait
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

    const int32_t chunk = kSelect * kOwn, chunks = (T + chunk - 1) / chunk;
    float x[kOwn];
    auto load = [&](int32_t n) {
        const int32_t t0 = n * chunk + threadIdx.x * kOwn;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) x[e] = t0 + e < T ? w[t0 + e] : 0.0f;
    };
    if (chunks > 0) load(0);

    const bool all = T <= J;
    uint32_t limit = 0, equal = 0;                               // keep keys above limit, and `equal` of those at it
    if (!all) {
        uint32_t mask = 0, need = J;
#pragma unroll
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : kBins;
            hist[threadIdx.x] = hist[threadIdx.x + kSelect] = 0;
            __syncthreads();
            for (int32_t n = 0; n < chunks; ++n) {
                if (chunks > 1) load(n);
                const int32_t t0 = n * chunk + threadIdx.x * kOwn;
#pragma unroll
                for (int e = 0; e < kOwn; ++e) {
                    const uint32_t k = key_of(x[e], t0 + e, T, j);
                    if (t0 + e < T && (k & mask) == limit) atomicAdd(&hist[k >> shift & (bins - 1)], 1u);
                }
            }
            __syncthreads();
            // the bin, from the top, in which the count reaches what is needed: two bins to a thread
            const int b = kBins - 1 - 2 * (int)threadIdx.x;
            const uint32_t hi = hist[b], lo = hist[b - 1];
            uint32_t total;
            const uint32_t before = scan(hi + lo, total, warp_sums);
            if (before < need && need <= before + hi + lo) {
                const bool first = need <= before + hi;
                found[0] = first ? b : b - 1;
                found[1] = need - before - (first ? 0 : hi);
            }
            __syncthreads();
            limit |= found[0] << shift;
            mask |= (uint32_t)(bins - 1) << shift;
            need = found[1];
            __syncthreads();
        }
        equal = need;
    }
    uint32_t above = 0, at = 0;                                  // of the chunks before
    for (int32_t n = 0; n < chunks; ++n) {
        if (chunks > 1) load(n);
        const int32_t t0 = n * chunk + threadIdx.x * kOwn;
        uint32_t gt = 0, eq = 0;                                 // bit e: token t0 + e
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            if (t0 + e < T) {
                const uint32_t k = key_of(x[e], t0 + e, T, j);
                if (all || k > limit) gt |= 1u << e;
                else if (k == limit) eq |= 1u << e;
            }
        }
        uint32_t total;
        const uint32_t before = scan(__popc(gt) | __popc(eq) << 16, total, warp_sums);
        uint32_t g = above + (before & 0xffffu), q = at + (before >> 16);
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            const bool is_eq = eq >> e & 1;
            if ((gt >> e & 1) || (is_eq && q < equal)) {
                const uint32_t p = g + min(q, equal);
                kept[p] = t0 + e;
                if (nw) nw[p] = x[e];
            }
            g += gt >> e & 1;
            q += is_eq;
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

// A lane per 16-byte vector of a kept row of one head, K and V together; a CTA takes `tokens`
// kept tokens of all heads, whose rows in the new blocks are contiguous, and two vectors of
// each thread are in flight.  Bound by HBM: a kept row is read and written once.
__global__ void __launch_bounds__(kCopy) kvs_evict_copy_kernel(EvictJob j, const __grid_constant__ Planes planes, int32_t layer0, uint32_t tokens) {
    const StepView& st = j.step;
    const int32_t l = blockIdx.z, r = blockIdx.y;
    const uint32_t vecs = st.head_dim / 8, H = st.kv_heads, per_token = vecs * H;
    const char* kp = reinterpret_cast<const char*>(planes.at[2 * l]);
    const char* vp = reinterpret_cast<const char*>(planes.at[2 * l + 1]);
    const int32_t* kept = j.kept + ((int64_t)(layer0 + l) * st.requests + r) * H * j.budget;
    const int32_t* src_table = st.tables + (int64_t)r * st.table_stride;
    const int32_t* dst_table = j.dst_tables + (int64_t)r * j.dst_stride;
    int32_t T = __ldg(st.kv_lens + r);
    if (T < 0 || T > st.max_kv) T = 0;
    const int32_t J = min(T, j.budget), j0 = blockIdx.x * tokens;
    if (j0 >= J) return;
    const uint32_t items = min(tokens, (uint32_t)(J - j0)) * per_token;
    grid_wait();                                                 // the selection
    constexpr int U = 2;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += kCopy * U) {
        uint4 a[U], b[U];
        int64_t from[U], to[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * kCopy;
            from[u] = to[u] = -1;
            if (i < items) {
                const uint32_t row = i / vecs, c = i - row * vecs, p = row / H, h = row - p * H;
                from[u] = row_of(st, src_table, kept[(int64_t)h * j.budget + j0 + p]);
                to[u] = row_of(st, dst_table, j0 + p);
                const int64_t off = h * st.head_dim + 8 * c;
                if (from[u] >= 0) from[u] += off;
                if (to[u] >= 0) to[u] += off;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            a[u] = b[u] = make_uint4(0, 0, 0, 0);
            if (from[u] >= 0) {
                a[u] = *reinterpret_cast<const uint4*>(kp + 2 * from[u]);
                b[u] = *reinterpret_cast<const uint4*>(vp + 2 * from[u]);
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
    const StepView& st = j.step;
    kvs_evict_select_kernel<<<dim3(st.kv_heads, st.requests, j.layers), kSelect, 0, s>>>(j);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return -(int)e;
    int n = 1;
    const int64_t rows = st.max_kv < j.budget ? st.max_kv : j.budget;
    const uint32_t per_token = st.head_dim / 8 * st.kv_heads, full = kCopy * 2;
    const uint32_t tokens = per_token >= full ? 1 : full / per_token;
    for (int l0 = 0; l0 < j.layers && rows > 0; l0 += kMostPlanes / 2, ++n) {
        const int count = j.layers - l0 < kMostPlanes / 2 ? j.layers - l0 : kMostPlanes / 2;
        Planes p{};
        for (int k = 0; k < 2 * count; ++k) p.at[k] = (uint64_t)j.planes[2 * l0 + k];
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)((rows + tokens - 1) / tokens), st.requests, count);
        cfg.blockDim = dim3(kCopy);
        cfg.stream = s;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at;
        cfg.numAttrs = l0 == 0;                                  // behind the selection; the others behind a copy
        e = cudaLaunchKernelEx(&cfg, kvs_evict_copy_kernel, j, p, (int32_t)l0, tokens);
        if (e != cudaSuccess) return -(int)e;
    }
    return n;
}

}  // namespace kvs
