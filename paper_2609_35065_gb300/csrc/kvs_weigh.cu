// kvs_weigh.cu -- accumulated attention weight of the cached tokens.
//
//     w_t = decay * w_t + sum over rows of e^(scale q . k_t - lse)
//
// with every row's lse known, so that a key's sum needs no other key.
#include "kvs_async.cuh"
#include "kvs_ops.cuh"

namespace kvs {
namespace {

constexpr int kThreads = 128;
constexpr int kQRows = 16;

// A thread per key, whose dims stay in registers; the rows go by in shared memory.
template <bool HALF, int DP>
__global__ void __launch_bounds__(kThreads) kvs_weigh_kernel(WeighJob j) {
    using N = Num<HALF>;
    __shared__ __align__(16) float rows_q[kQRows][DP];
    __shared__ float rows_lse[kQRows];
    __shared__ int32_t rows_lo[kQRows], rows_hi[kQRows];
    const StepView& st = j.step;
    const int32_t h = blockIdx.y, r = blockIdx.z;
    const Request q = load_request(st, r);
    const int32_t t = blockIdx.x * kThreads + threadIdx.x;
    if ((int32_t)(blockIdx.x * kThreads) >= q.T) return;
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;
    const int64_t row = t < q.T ? row_of(st, table, t) : -1;
    uint32_t k[DP / 2];
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row >= 0 && 8 * c < st.head_dim)
            v = __ldg(reinterpret_cast<const uint4*>(j.k_plane + 2 * (row + (int64_t)h * st.head_dim + 8 * c)));
        k[4 * c] = v.x;
        k[4 * c + 1] = v.y;
        k[4 * c + 2] = v.z;
        k[4 * c + 3] = v.w;
    }
    float sum = 0.0f;
    const int32_t total = q.n * st.group;
    for (int32_t p0 = 0; p0 < total; p0 += kQRows) {
        __syncthreads();
        for (int v = threadIdx.x; v < kQRows * DP; v += kThreads) {
            const int i = v / DP, d = v % DP;
            const int32_t p = p0 + i, tok = q.q0 + p / st.group, head = h * st.group + p % st.group;
            float x = 0.0f;
            if (p < total && d < st.head_dim)
                x = N::to(reinterpret_cast<const typename N::T*>(j.q.base)[(int64_t)tok * j.q.row + (int64_t)head * j.q.head + d]);
            rows_q[i][d] = x;
        }
        if (threadIdx.x < kQRows) {
            const int32_t p = p0 + threadIdx.x;
            Span s{0, 0};
            float e = 0.0f;
            if (p < total) {
                const int32_t i = p / st.group;
                s = seen_by(q, i, i, j.causal, j.window);
                e = j.lse[(int64_t)(q.q0 + i) * (st.kv_heads * st.group) + h * st.group + p % st.group] * 1.4426950408889634f;
            }
            rows_lo[threadIdx.x] = s.lo;
            rows_hi[threadIdx.x] = s.hi;
            rows_lse[threadIdx.x] = e;
        }
        __syncthreads();
        for (int i = 0; i < kQRows; ++i) {
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int c = 0; c < DP / 2; ++c) {
                const float2 kv = N::to2(k[c]);
                a = fmaf(kv.x, rows_q[i][2 * c], a);
                b = fmaf(kv.y, rows_q[i][2 * c + 1], b);
            }
            if (t >= rows_lo[i] && t < rows_hi[i]) sum += exp2_fast((a + b) * j.scale_log2 - rows_lse[i]);
        }
    }
    if (t < q.T) {
        float* w = j.weights + r * j.request_stride + h * j.head_stride + t;
        *w = j.decay == 0.0f ? sum : fmaf(j.decay, *w, sum);
    }
}

template <bool HALF>
cudaError_t weigh(const WeighJob& j, cudaStream_t s) {
    const dim3 grid((j.step.max_kv + kThreads - 1) / kThreads, j.step.kv_heads, j.step.requests);
    if (j.step.head_dim <= 64) kvs_weigh_kernel<HALF, 64><<<grid, kThreads, 0, s>>>(j);
    else kvs_weigh_kernel<HALF, 128><<<grid, kThreads, 0, s>>>(j);
    return cudaGetLastError();
}

}  // namespace

int launch_weigh(const WeighJob& j, bool half, cudaStream_t s) {
    const cudaError_t e = half ? weigh<true>(j, s) : weigh<false>(j, s);
    return e == cudaSuccess ? 1 : -(int)e;
}

}  // namespace kvs
