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

constexpr int kSelect = 256;           // threads of a selecting CTA
constexpr int kWarps = kSelect / 32;
constexpr int kBins = 2048;
constexpr int kCached = 16384;         // weights that a CTA keeps in shared memory
constexpr int kCopy = 256;

// Unsigned keys in the weights' order; NaN below all, always-kept tokens above all.
__device__ __forceinline__ uint32_t key_of(float w, int32_t t, int32_t T, const EvictJob& j) {
    if (t < j.sinks || t >= T - j.recent) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.0f);                // -0 is 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The weight of a key, where the key tells it: not of always-kept tokens, NaN and zeros.
__device__ __forceinline__ bool tells(uint32_t k) { return k != 0xffffffffu && k != 0 && k != 0x80000000u; }
__device__ __forceinline__ float weight_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Sum of v over the CTA's earlier threads (warp_sums: kWarps).
__device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before += w < warp ? warp_sums[w] : 0;
    return before + x - v;
}

// One CTA per (head, request, layer), whose warps own a stretch of consecutive tokens each:
// only the digits' counts and the warps' own are shared, so that a pass has few barriers.  Up
// to 16384 keys stay in shared memory; of a longer cache each pass makes them again, from L2.
// Bound by its chain of passes -- a digit's count and its bin some 3000 cycles, writing the
// kept ones 4000 to 8000 -- and by its instructions (about three a token); several CTAs to an SM
// overlap theirs.  512 heads of 8192 tokens: about 22 us of the call's 182.5 us.  512 threads to
// a CTA: 186 us.  A long cache has one CTA a head all the same: a call takes 525 us for 1 layer of
// 8 heads with 131072 tokens, of which 32768 stay (41 us of bytes), and 450 us for 32 layers with
// 32768 and 8192 (324).
template <bool CACHED>
__global__ void __launch_bounds__(kSelect) kvs_evict_select_kernel(EvictJob j) {
    extern __shared__ __align__(16) uint32_t cache[];
    __shared__ __align__(16) uint32_t hist[kBins];
    __shared__ uint32_t sums[2][kWarps], found[3];
    const StepView& st = j.step;
    const int32_t h = blockIdx.x, r = blockIdx.y, l = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
    for (int32_t p = J + threadIdx.x; p < j.budget; p += kSelect) {
        kept[p] = -1;
        if (nw) nw[p] = 0.0f;
    }
    if (T <= J) {
        for (int32_t t = threadIdx.x; t < T; t += kSelect) {
            kept[t] = t;
            if (nw) nw[t] = __ldg(w + t);
        }
        return;
    }

    // Stretches of whole groups of 128 tokens, four to a lane.  What lies beyond T has the lowest
    // key and comes last: it is never among the J < T that are kept.
    const int32_t groups = (T + 127) / 128, per_warp = (groups + kWarps - 1) / kWarps;
    const int32_t t_lo = min(groups, warp * per_warp) * 128 + 4 * lane, t_hi = min(groups, (warp + 1) * per_warp) * 128;
    auto make = [&](int32_t t) { return t < T ? key_of(__ldg(w + t), t, T, j) : 0u; };
    auto keys = [&](int32_t t) {
        return CACHED ? *reinterpret_cast<const uint4*>(cache + t) : make_uint4(make(t), make(t + 1), make(t + 2), make(t + 3));
    };
    if (CACHED) {
        // Eight loads of a lane in flight (sixteen: 32 layers x 2 requests as fast, two small layers 13.5
        // instead of 11.2 us); left to the loop each waits for the store before it, which might alias.
        for (int32_t t = t_lo - 3 * lane; t < t_hi; t += 256) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = t + 32 * e < min(t_hi, T) ? __ldg(w + t + 32 * e) : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (t + 32 * e < t_hi) cache[t + 32 * e] = t + 32 * e < T ? key_of(x[e], t + 32 * e, T, j) : 0u;
        }
        __syncwarp();
    }
    uint32_t limit = 0, mask = 0, need = J;                      // keep keys above limit in the mask's bits, and `need` of those at it
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : kBins;
#pragma unroll
        for (int b = 0; b < kBins; b += kSelect) hist[b + threadIdx.x] = 0;
        __syncthreads();
#pragma unroll 2
        for (int32_t t = t_lo; t < t_hi; t += 128) {
            const uint4 k = keys(t);
            auto count = [&](uint32_t x) {
                if ((x & mask) == limit) atomicAdd(&hist[x >> shift & (bins - 1)], 1u);
            };
            count(k.x);
            count(k.y);
            count(k.z);
            count(k.w);
        }
        __syncthreads();
        // the bin, from the top, in which the count reaches what is needed: eight bins to a thread
        const int top = kBins - 1 - 8 * (int)threadIdx.x;
        const uint4 hi = *reinterpret_cast<const uint4*>(hist + top - 3), lo = *reinterpret_cast<const uint4*>(hist + top - 7);
        const uint32_t bin[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
        uint32_t sum = 0;
#pragma unroll
        for (int b = 0; b < 8; ++b) sum += bin[b];
        uint32_t before = scan(sum, sums[digit & 1]);
        if (before < need && need <= before + sum) {
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                if (before < need && need <= before + bin[b]) {
                    found[0] = top - b;
                    found[1] = need - before;
                    found[2] = bin[b];
                }
                before += bin[b];
            }
        }
        __syncthreads();
        limit |= found[0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        need = found[1];
        if (need == found[2]) break;                             // the whole bin is kept: its order does not matter
    }
    __syncthreads();
    // how many of each warp's are above and at the limit, then where each goes
    auto classify = [&](const uint4& k, uint32_t (&gt)[4], uint32_t (&eq)[4]) {
        const uint32_t x[4] = {k.x & mask, k.y & mask, k.z & mask, k.w & mask};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            gt[e] = x[e] > limit;
            eq[e] = x[e] == limit;
        }
    };
    uint32_t n_gt = 0, n_eq = 0;
    for (int32_t t = t_lo; t < t_hi; t += 128) {
        uint32_t gt[4], eq[4];
        classify(keys(t), gt, eq);
        n_gt += gt[0] + gt[1] + gt[2] + gt[3];
        n_eq += eq[0] + eq[1] + eq[2] + eq[3];
    }
    n_gt = __reduce_add_sync(0xffffffffu, n_gt);
    n_eq = __reduce_add_sync(0xffffffffu, n_eq);
    if (lane == 0) {
        sums[0][warp] = n_gt;
        sums[1][warp] = n_eq;
    }
    __syncthreads();
    uint32_t g = 0, q = 0;
#pragma unroll
    for (int n = 0; n < kWarps; ++n) {
        g += n < warp ? sums[0][n] : 0;
        q += n < warp ? sums[1][n] : 0;
    }
    for (int32_t t = t_lo; t < t_hi; t += 128) {
        uint32_t gt[4], eq[4];
        const uint4 k = keys(t);
        const uint32_t key[4] = {k.x, k.y, k.z, k.w};
        classify(k, gt, eq);
        const uint32_t both = (gt[0] + gt[1] + gt[2] + gt[3]) | (eq[0] + eq[1] + eq[2] + eq[3]) << 16;
        uint32_t x = both;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        const uint32_t total = __shfl_sync(0xffffffffu, x, 31);
        x -= both;
        uint32_t my_g = g + (x & 0xffffu), my_q = q + (x >> 16);
        float weight[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            weight[e] = weight_of(key[e]);
            if (nw && (gt[e] || eq[e]) && !tells(key[e])) weight[e] = __ldg(w + t + e);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (gt[e] || (eq[e] && my_q < need)) {
                const uint32_t p = my_g + min(my_q, need);
                kept[p] = t + e;
                if (nw) nw[p] = weight[e];
            }
            my_g += gt[e];
            my_q += eq[e];
        }
        g += total & 0xffffu;
        q += total >> 16;
    }
}

constexpr int kMostPlanes = 448;       // plane addresses that a launch carries

struct Planes {
    uint64_t at[kMostPlanes];
};

// A lane per 16-byte vector of a kept row of one head, K and V together; a CTA takes `tokens`
// kept tokens of all heads, whose rows in the new blocks are contiguous, and two vectors of
// each thread are in flight.  Bound by HBM: a kept row is read and written once, 1.05 million rows
// of 256 bytes of K and of V (1.07 GB) in 159 us, 6.7 TB/s.
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
    // The selection.  CTAs without tokens wait too: otherwise a copy of nothing could be over before it.
    grid_wait();
    if (j0 >= J) return;
    const uint32_t items = min(tokens, (uint32_t)(J - j0)) * per_token;
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
    const dim3 units(st.kv_heads, st.requests, j.layers);
    cudaError_t e = cudaSuccess;
    if (st.max_kv <= kCached) {
        e = cudaFuncSetAttribute(kvs_evict_select_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCached * 4);
        if (e == cudaSuccess) kvs_evict_select_kernel<true><<<units, kSelect, (st.max_kv + 127) / 128 * 512, s>>>(j);
    } else {
        kvs_evict_select_kernel<false><<<units, kSelect, 0, s>>>(j);
    }
    if (e == cudaSuccess) e = cudaGetLastError();
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
