// kvs_append_axes.cu -- rotary positions on several axes, and the append into the paged planes.
//
// Pair j of a head turns by positions[axis[j]] * turns[j]: (a, b) -> (a cos - b sin, b cos + a sin),
// the same for all heads of a token.  As in kvs_append.cu a lane works out the sines of a few pairs
// of one token once and applies them to every head it is given.  Bound by HBM, each element being
// read and written once.
#include "kvs_append.cuh"
#include "kvs_async.cuh"

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

// Request of row n, found by the whole warp 32 entries at a time: the last one that starts at or before it.
__device__ __forceinline__ int32_t request_of(const StepView& st, int32_t n, int lane) {
    if (!st.q_starts) return n;
    int32_t lo = 0, hi = st.requests;                // q_starts[lo] <= n < q_starts[hi], if they are in order
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 31) / 32, at = lo + step * lane;
        const uint32_t behind = __ballot_sync(0xffffffffu, lane > 0 && (at >= hi || st.q_starts[at] > n));
        const int32_t some = behind ? __ffs(behind) - 1 : 32;
        hi = min(hi, lo + step * some);
        lo += step * (some - 1);
    }
    return lo;
}

// A warp takes one token (or a share of its heads); a lane owns two pieces of eight elements of a head: of
// the rotated part eight of its first half and those that they pair with, of the rest, and of neighbours
// (PAIRS), sixteen in a row.  32768 tokens of 32 + 2 x 8 heads of 128 dims (805 MB) on three axes in 125 us, 6.4 TB/s (PAIRS: 131);
// a decode step of 16 tokens 3.8 us in a graph.
template <bool HALF, bool PAIRS>
__global__ void __launch_bounds__(256) kvs_append_axes_kernel(AppendJob j, uint32_t warps_per_token, int32_t groups) {
    grid_wait();
    const uint32_t w = blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);       // at most 2^31 + 2^11 of them are needed
    const uint32_t own = (uint32_t)j.step.total_q * warps_per_token;
    if (w >= own) {
        check_requests<true>(j.step, w - own);
        return;
    }
    using N = Num<HALF>;
    constexpr int W = 8, V = W / 2;
    const int32_t n = w / warps_per_token, part = w % warps_per_token;
    const int lane = threadIdx.x & 31;
    Where where;
#pragma unroll
    for (int a = 0; a < kAxes; ++a) where.at[a] = a < j.axes ? j.positions[a * j.axis_stride + n] : 0;
    const Place pl = place_of<true>(j, n);
    if (!pl.owned) return;
    const int32_t D = j.step.head_dim, rot = j.rot_dim, H = j.step.kv_heads;
    const int32_t lanes = min(32, groups), heads_at_once = 32 / lanes;
    if (lane / lanes >= heads_at_once) return;
    const int32_t first = part * heads_at_once + lane / lanes, step = (int32_t)warps_per_token * heads_at_once;
    const int32_t qh = j.q.base ? j.q_heads : 0, total = qh + 2 * H;
    // One round: there are at most eight groups.  As straight code the compiler gives it 74 registers instead of 64,
    // and those 125 us become 132 (133 where it is held to 64).
    for (int32_t c0 = lane % lanes; c0 < groups; c0 += lanes) {
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
            if (turned && pair < rot / 2) turn(where.on(j, j.axis[pair]), j.turns[pair], j.scale, c[k], s[k]);
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
                            a[i].w[k] = N::pack(u.x * c[2 * k] - v.x * s[2 * k], u.y * c[2 * k + 1] - v.y * s[2 * k + 1]);
                            b[i].w[k] = N::pack(v.x * c[2 * k] + u.x * s[2 * k], v.y * c[2 * k + 1] + u.y * s[2 * k + 1]);
                        }
                    }
                }
                a[i].store(dst[i] + 2 * e0);
                if (has1) b[i].store(dst[i] + 2 * e1);
            }
        }
    }
}

// Halves that begin at no multiple of eight elements: pieces of W elements of them are too narrow for the way
// to and from HBM, so a warp brings `chunk` heads at a time into shared memory in vectors of 16 bytes, turns
// them there and writes them out alike.  11 images of 1225 to 1369 tokens, 2 x 16 + 16 heads of 72 dims (197 MB): 37 us, 5.3 TB/s; 47
// by a kernel as above with pieces of four.
constexpr int kWarps = 8;
template <bool HALF, int W>
__global__ void __launch_bounds__(32 * kWarps) kvs_append_axes_staged_kernel(AppendJob j, uint32_t warps_per_token, int32_t chunk, uint32_t vec_m) {
    extern __shared__ __align__(16) char staged[];
    grid_wait();
    const uint32_t w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const uint32_t all = (uint32_t)j.step.total_q * warps_per_token;
    if (w >= all) {
        check_requests<true>(j.step, w - all);
        return;
    }
    using N = Num<HALF>;
    constexpr int V = (W + 1) / 2;
    const int32_t n = w / warps_per_token, part = w % warps_per_token;
    const int lane = threadIdx.x & 31;
    Where where;
#pragma unroll
    for (int a = 0; a < kAxes; ++a) where.at[a] = a < j.axes ? j.positions[a * j.axis_stride + n] : 0;
    const int32_t D = j.step.head_dim, half = j.rot_dim / 2, H = j.step.kv_heads, vecs = D / 8, pieces = half / W;
    const int32_t qh = j.q.base ? j.q_heads : 0, total = qh + 2 * H, step = (int32_t)warps_per_token * chunk;
    char* own = staged + (threadIdx.x >> 5) * chunk * D * 2;
    const uint32_t own_at = smem_u32(own);
    auto bring = [&](int32_t h0) {
        for (int32_t v = lane; v < min(chunk, total - h0) * vecs; v += 32) {
            const int32_t h = h0 + (int32_t)((uint32_t)v * vec_m >> 16), c = v - (h - h0) * vecs;
            const RowsView& rv = h < qh ? j.q : h < qh + H ? j.k : j.v;
            cp_async16(own_at + 16 * v, rv.base + 2 * ((int64_t)n * rv.row + (int64_t)(h < qh ? h : h < qh + H ? h - qh : h - qh - H) * rv.head) + 16 * c, true);
        }
        cp_commit();
    };
    // what is brought first does not depend on where the row belongs
    if (part * chunk < total) bring(part * chunk);
    // the row's request, then that one's lengths, with the sines in between, then its block
    const int32_t r = request_of(j.step, n, lane);
    const RawRequest fetched = fetch_request<true>(j.step, r);
    // piece c0 % pieces of every at_once-th head is this lane's; of more than 32 pieces (W is 1 then) also c0 + 32
    const int32_t at_once = pieces < 32 ? 32 / pieces : 1;
    float c[2 * V], s[2 * V];
    auto sines = [&](int32_t c0) {
        if (c0 >= pieces * at_once) return;
        const int32_t e = W * (c0 % pieces);
#pragma unroll
        for (int k = 0; k < W; ++k) turn(where.on(j, j.axis[e + k]), j.turns[e + k], j.scale, c[k], s[k]);
    };
    sines(lane);
    const Request q = check_request(j.step, fetched);
    const bool owned = n >= q.q0 && n < q.q0 + q.n;
    const int32_t t = q.T - q.n + (n - q.q0);
    const int64_t row = owned && t >= 0 ? row_of<true>(j.step, j.step.tables + (int64_t)r * j.step.table_stride, t) : -1;
    cp_wait<0>();
    if (!owned) return;
    for (int32_t h0 = part * chunk; h0 < total; h0 += step) {
        __syncwarp();
        const int32_t heads = min(chunk, total - h0), turned = min(heads, qh + H - h0);      // values are not
        auto rotate = [&](int32_t c0) {
            if (c0 >= pieces * at_once) return;
            const int32_t e = W * (c0 % pieces);
            for (int32_t h = c0 / pieces; h < turned; h += at_once) {
                char* at = own + (h * D + e) * 2;
                Piece<W> a, b;
                a.load(at);
                b.load(at + 2 * half);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float2 u = N::to2(a.w[k]), v = N::to2(b.w[k]);
                    a.w[k] = N::pack(u.x * c[2 * k] - v.x * s[2 * k], W == 1 ? 0.0f : u.y * c[2 * k + 1] - v.y * s[2 * k + 1]);
                    b.w[k] = N::pack(v.x * c[2 * k] + u.x * s[2 * k], W == 1 ? 0.0f : v.y * c[2 * k + 1] + u.y * s[2 * k + 1]);
                }
                a.store(at);
                b.store(at + 2 * half);
            }
        };
        rotate(lane);
        if (pieces > 32) {
            sines(lane + 32);
            rotate(lane + 32);
            sines(lane);
        }
        __syncwarp();
        for (int32_t v = lane; v < heads * vecs; v += 32) {
            const int32_t x = (int32_t)((uint32_t)v * vec_m >> 16), h = h0 + x;
            char* dst = nullptr;
            if (h < qh) dst = j.q_out.base + 2 * ((int64_t)n * j.q_out.row + (int64_t)h * j.q_out.head);
            else if (row >= 0) dst = (h < qh + H ? j.k_plane : j.v_plane) + 2 * (row + (int64_t)(h < qh + H ? h - qh : h - qh - H) * D);
            if (dst) *reinterpret_cast<uint4*>(dst + 16 * (v - x * vecs)) = *reinterpret_cast<const uint4*>(own + 16 * v);
        }
        if (h0 + step < total) {
            __syncwarp();
            bring(h0 + step);
            cp_wait<0>();
        }
    }
}

template <bool HALF, int W>
cudaError_t append_staged(const AppendJob& j, cudaStream_t s) {
    const int32_t D = j.step.head_dim, total = (j.q.base ? j.q_heads : 0) + 2 * j.step.kv_heads, vecs = D / 8;
    const int64_t rows = j.step.total_q;
    // Heads of a warp at a time: up to 3.5 KB (7 KB took 40 us for those 37, 2.4 KB 39); few rows are shared out as above.
    const int32_t room = 3500 / (2 * D);
    int parts = (total + 3) / 4;
    while (parts > 1 && rows * parts > 152 * 64) parts = (parts + 1) / 2;
    const int32_t share = (total + parts - 1) / parts, chunk = share < room ? share : room;
    return launch_behind(kvs_append_axes_staged_kernel<HALF, W>, dim3((warps_of(j.step, rows * parts) + kWarps - 1) / kWarps), 32 * kWarps,
                         kWarps * chunk * D * 2, s, j, parts, chunk, (65536 + vecs - 1) / vecs);
}

template <bool HALF, bool PAIRS>
cudaError_t append_axes(const AppendJob& j, cudaStream_t s) {
    const int32_t D = j.step.head_dim, groups = (D + 15) / 16;   // at most 8
    const int32_t at_once = 32 / groups, total = (j.q.base ? j.q_heads : 0) + 2 * j.step.kv_heads;
    // Few rows: a warp for every few heads, so that the GPU is filled; many (64 warps for each of
    // the 152 SMs): one warp per row, which works out the sines once.
    const int64_t rows = j.step.total_q;
    int parts = (total + at_once - 1) / at_once;
    while (parts > 1 && rows * parts > 152 * 64) parts = (parts + 1) / 2;
    return launch_behind(kvs_append_axes_kernel<HALF, PAIRS>, dim3((warps_of(j.step, rows * parts) + 7) / 8), 256, 0, s, j, parts, groups);
}

template <bool HALF>
cudaError_t append_axes(const AppendJob& j, cudaStream_t s) {
    if (j.interleaved) return append_axes<HALF, true>(j, s);
    if (j.rot_dim % 16 == 0) return append_axes<HALF, false>(j, s);
    // pieces as wide as the halves divide into: neither then crosses into the other
    if (j.rot_dim % 8 == 0) return append_staged<HALF, 4>(j, s);
    return j.rot_dim % 4 == 0 ? append_staged<HALF, 2>(j, s) : append_staged<HALF, 1>(j, s);
}

}  // namespace

cudaError_t launch_append_axes(const AppendJob& j, bool half, cudaStream_t s) { return half ? append_axes<true>(j, s) : append_axes<false>(j, s); }

}  // namespace kvs
