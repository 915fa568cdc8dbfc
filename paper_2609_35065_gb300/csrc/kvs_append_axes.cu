// kvs_append_axes.cu -- rotary positions on several axes, and the append into the paged planes.
//
// Pair j of a head turns by positions[axis[j]] * turns[j]: (a, b) -> (a cos - b sin, b cos + a sin),
// the same for all heads of a token.  As in kvs_append.cu a lane works out the sines of a few pairs
// of one token once and applies them to every head it is given.  Bound by HBM, each element being
// read and written once.
#include "kvs_append.cuh"

namespace kvs {
namespace {

constexpr int kAxes = KVS_MAX_AXES;
constexpr int kAtOnce = 2;             // heads of a lane in flight

// W 16-bit elements, as words of two (one of one).
template <int W>
struct Piece {
    alignas(W >= 2 ? 2 * W : 4) uint32_t w[(W + 1) / 2];
    __device__ __forceinline__ void load(const char* p) {
        if constexpr (W == 8) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p);
        else if constexpr (W == 4) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
        else if constexpr (W == 2) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    __device__ __forceinline__ void store(char* p) const {
        if constexpr (W == 8) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
        else if constexpr (W == 4) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(w);
        else if constexpr (W == 2) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
};

// A token's positions on all axes, which are loaded before any pair asks for its own.
struct Where {
    int32_t at[kAxes];
    __device__ __forceinline__ int32_t on(const AppendJob& j, int32_t axis) const {
        int32_t p = at[0];
#pragma unroll
        for (int a = 1; a < kAxes; ++a) p = axis == a ? at[a] : p;
        if (axis >= j.axes) {
            record_error(j.step.err, KVS_ERR_BOUNDS);
            p = 0;
        }
        return p;
    }
};

// A warp takes one token (or a share of its heads); a lane owns two pieces of W elements of a head: of
// the rotated part W of its first half and the W that they pair with, of the rest, and of neighbours
// (PAIRS: W is 8 then), 2 W in a row.
template <bool HALF, int W, bool PAIRS>
__global__ void __launch_bounds__(256) kvs_append_axes_kernel(AppendJob j, uint32_t warps_per_token, int32_t groups) {
    const uint32_t w = blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);       // at most 2^31 + 2^11 of them are needed
    const uint32_t own = (uint32_t)j.step.total_q * warps_per_token;
    if (w >= own) {
        check_requests(j.step, w - own);
        return;
    }
    using N = Num<HALF>;
    constexpr int V = (W + 1) / 2;
    const int32_t n = w / warps_per_token, part = w % warps_per_token;
    const int lane = threadIdx.x & 31;
    Where where;
#pragma unroll
    for (int a = 0; a < kAxes; ++a) where.at[a] = a < j.axes ? __ldg(j.positions + a * j.axis_stride + n) : 0;
    const Place pl = place_of(j, n);
    if (!pl.owned) return;
    const int32_t D = j.step.head_dim, rot = j.rot_dim, H = j.step.kv_heads;
    const int32_t lanes = min(32, groups), heads_at_once = 32 / lanes;
    if (lane / lanes >= heads_at_once) return;
    const int32_t first = part * heads_at_once + lane / lanes, step = (int32_t)warps_per_token * heads_at_once;
    const int32_t qh = j.q.base ? j.q_heads : 0, total = qh + 2 * H;
    for (int32_t c0 = lane % lanes; c0 < groups; c0 += lanes) {                    // once, but for odd halves
        int32_t e0, e1;
        bool turned;
        if (PAIRS) {
            e0 = 2 * W * c0;
            e1 = e0 + W;
            turned = e0 < rot;
        } else {
            const int32_t halves = rot / (2 * W);
            turned = c0 < halves;
            e0 = turned ? W * c0 : rot + 2 * W * (c0 - halves);
            e1 = turned ? e0 + rot / 2 : e0 + W;
        }
        const bool has1 = e1 < D;
        float c[2 * V], s[2 * V];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const int32_t pair = (PAIRS ? e0 / 2 : e0) + k;
            c[k] = 1.0f;
            s[k] = 0.0f;
            if (turned && pair < rot / 2) turn(where.on(j, __ldg(j.axis + pair)), __ldg(j.turns + pair), j.scale, c[k], s[k]);
        }
        for (int32_t h0 = first; h0 < total; h0 += kAtOnce * step) {
            Piece<W> a[kAtOnce], b[kAtOnce];
            char* dst[kAtOnce];
            bool rotate[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int32_t h = h0 + i * step, x = h - qh;
                const char* src = nullptr;
                dst[i] = nullptr;
                rotate[i] = turned && x < H;
                if (x < 0) {
                    src = j.q.base + 2 * ((int64_t)n * j.q.row + (int64_t)h * j.q.head);
                    dst[i] = j.q_out.base + 2 * ((int64_t)n * j.q_out.row + (int64_t)h * j.q_out.head);
                } else if (h < total && pl.row >= 0) {
                    const int32_t y = x < H ? x : x - H;
                    const RowsView& rv = x < H ? j.k : j.v;
                    src = rv.base + 2 * ((int64_t)n * rv.row + (int64_t)y * rv.head);
                    dst[i] = (x < H ? j.k_plane : j.v_plane) + 2 * (pl.row + (int64_t)y * D);
                }
                if (src) a[i].load(src + 2 * e0);
                if (src && has1) b[i].load(src + 2 * e1);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (!dst[i]) continue;
                if (rotate[i]) {
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float2 u = N::to2(a[i].w[k]), v = N::to2(b[i].w[k]);
                        if (PAIRS) {
                            // pairs behind the rotated part keep their bits
                            if (e0 / 2 + k < rot / 2) a[i].w[k] = N::pack(u.x * c[k] - u.y * s[k], u.y * c[k] + u.x * s[k]);
                            if (e0 / 2 + V + k < rot / 2) b[i].w[k] = N::pack(v.x * c[V + k] - v.y * s[V + k], v.y * c[V + k] + v.x * s[V + k]);
                        } else {
                            a[i].w[k] = N::pack(u.x * c[2 * k] - v.x * s[2 * k], W == 1 ? 0.0f : u.y * c[2 * k + 1] - v.y * s[2 * k + 1]);
                            b[i].w[k] = N::pack(v.x * c[2 * k] + u.x * s[2 * k], W == 1 ? 0.0f : v.y * c[2 * k + 1] + u.y * s[2 * k + 1]);
                        }
                    }
                }
                a[i].store(dst[i] + 2 * e0);
                if (has1) b[i].store(dst[i] + 2 * e1);
            }
        }
    }
}

template <bool HALF, int W, bool PAIRS>
cudaError_t append_axes(const AppendJob& j, cudaStream_t s) {
    const int32_t D = j.step.head_dim, rot = j.rot_dim;
    const int32_t groups = PAIRS ? (D + 15) / 16 : rot / (2 * W) + (D - rot + 2 * W - 1) / (2 * W);
    const int32_t at_once = 32 / (groups < 32 ? groups : 32), total = (j.q.base ? j.q_heads : 0) + 2 * j.step.kv_heads;
    // Few rows: a warp for every few heads, so that the GPU is filled; many (64 warps for each of
    // the 152 SMs): one warp per row, which works out the sines once.
    const int64_t rows = j.step.total_q;
    int parts = (total + at_once - 1) / at_once;
    while (parts > 1 && rows * parts > 152 * 64) parts = (parts + 1) / 2;
    kvs_append_axes_kernel<HALF, W, PAIRS><<<(warps_of(j.step, rows * parts) + 7) / 8, 256, 0, s>>>(j, parts, groups);
    return cudaGetLastError();
}

template <bool HALF>
cudaError_t append_axes(const AppendJob& j, cudaStream_t s) {
    if (j.interleaved) return append_axes<HALF, 8, true>(j, s);
    // pieces as wide as the halves divide into: neither then crosses into the other
    if (j.rot_dim % 16 == 0) return append_axes<HALF, 8, false>(j, s);
    if (j.rot_dim % 8 == 0) return append_axes<HALF, 4, false>(j, s);
    return j.rot_dim % 4 == 0 ? append_axes<HALF, 2, false>(j, s) : append_axes<HALF, 1, false>(j, s);
}

}  // namespace

cudaError_t launch_append_axes(const AppendJob& j, bool half, cudaStream_t s) { return half ? append_axes<true>(j, s) : append_axes<false>(j, s); }

}  // namespace kvs
