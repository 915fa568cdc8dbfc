// kvs_append.cu -- rotary positions of new tokens' queries and keys, and the append of
// keys and values into the paged planes.
//
// (a, b) -> (a cos - b sin, b cos + a sin) with the angle of (token, pair), shared by all
// heads: a thread works out the sines of eight pairs of one token once and applies them to
// every head it is given.  Bound by HBM, each element being read and written once: 32768 tokens
// of 32 + 2 x 8 heads of 128 dims (805 MB) in 131 us, 6.1 TB/s.  A decode step of 16 tokens is
// latency: about 8 us, most of them the call's.
#include "kvs_ops.cuh"

namespace kvs {
namespace {

// cos and sin of pos * (f.x + f.y) turns.  The product with the large part is split exactly
// into its rounded value and the rest, so only the fraction of a turn is ever rounded:
// about 2^-22 of a turn at any position up to 2^24.
__device__ __forceinline__ void turn(int32_t pos, float2 f, float scale, float& c, float& s) {
    const float p = (float)pos;
    const float hi = p * f.x;
    const float rest = fmaf(p, f.x, -hi) + p * f.y;
    const float frac = (hi - rintf(hi)) + rest;
    sincospif(2.0f * frac, &s, &c);
    c *= scale;
    s *= scale;
}

// One token's (row of the tensors) place: its position, its row in the planes (< 0: none), and
// whether it is a request's at all.
struct Place {
    int32_t pos;
    int64_t row;
    bool    owned;
};

// Request of row n: the last one that starts at or before it.
__device__ __forceinline__ Place place_of(const AppendJob& j, int32_t n) {
    const StepView& st = j.step;
    Place pl;
    pl.pos = 0;
    pl.row = -1;
    int32_t r = n;
    if (st.q_starts) {
        int32_t lo = 0, hi = st.requests;            // q_starts[lo] <= n < q_starts[hi], if they are in order
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (__ldg(st.q_starts + mid) <= n) lo = mid;
            else hi = mid;
        }
        r = lo;
    }
    const Request q = load_request(st, r);
    const int32_t t = q.T - q.n + (n - q.q0);
    pl.owned = n >= q.q0 && n < q.q0 + q.n;
    if (pl.owned && t >= 0) pl.row = row_of(st, st.tables + (int64_t)r * st.table_stride, t);
    pl.pos = j.positions ? __ldg(j.positions + n) : max(t, 0);
    return pl;
}

// A request out of bounds may have no row that leads to it (its range falls, or is empty): the
// grid has warps behind the rows' own that look at 32 requests each (looking behind their own work,
// the rows' warps took 1.5% longer).
__device__ __forceinline__ void check_requests(const StepView& st, uint32_t group) {
    const uint32_t r = 32 * group + (threadIdx.x & 31);
    if (st.q_starts && r < (uint32_t)st.requests) load_request(st, r);
}
uint32_t warps_of(const StepView& st, int64_t row_warps) { return (uint32_t)(row_warps + (st.q_starts ? (st.requests + 31) / 32 : 0)); }

// A warp takes one token at a time: its lanes go over (head, vector pair), eight pairs each.
// VEC: halves of the rotated part begin at multiples of eight elements (or pairs are neighbours).
template <bool HALF>
__global__ void __launch_bounds__(256) kvs_append_kernel(AppendJob j, uint32_t warps_per_token, int32_t lanes_per_head) {
    const uint32_t w = blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);       // at most 2^31 + 2^11 of them are needed
    const uint32_t own = (uint32_t)j.step.total_q * warps_per_token;
    if (w >= own) {
        check_requests(j.step, w - own);
        return;
    }
    const int32_t n = w / warps_per_token, part = w % warps_per_token;
    const int lane = threadIdx.x & 31;
    const Place pl = place_of(j, n);
    if (!pl.owned) return;
    const int32_t D = j.step.head_dim, rot = j.rot_dim;
    using N = Num<HALF>;

    const int32_t c0 = lane % lanes_per_head, heads_at_once = 32 / lanes_per_head;
    if (lane / lanes_per_head >= heads_at_once) return;
    const int32_t first = part * heads_at_once + lane / lanes_per_head, step = (int32_t)warps_per_token * heads_at_once;
    const int32_t total = (j.q.base ? j.q_heads : 0) + 2 * j.step.kv_heads;
    // A lane owns two groups of eight elements of a head.  Rotated halves: [8c, 8c + 8) and the
    // eight at rot / 2 behind; neighbours and the rest of the head: sixteen in a row.
    const bool halves = !j.interleaved;
    const int32_t half_groups = rot / 16;            // lanes that own a pair of rotated groups
    int32_t e0, e1;
    bool turned;
    if (halves) {
        turned = c0 < half_groups;
        e0 = turned ? 8 * c0 : rot + 16 * (c0 - half_groups);
        e1 = turned ? e0 + rot / 2 : e0 + 8;
    } else {
        e0 = 16 * c0;
        e1 = e0 + 8;
        turned = e0 < rot;
    }
    const bool has0 = e0 < D, has1 = e1 < D;
    float c[8], s[8];
    if (turned) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int32_t pair = (halves ? e0 : e0 / 2) + k;
            c[k] = 1.0f;
            s[k] = 0.0f;
            if (pair < rot / 2) turn(pl.pos, __ldg(j.turns + pair), j.scale, c[k], s[k]);
        }
    }
    for (int32_t h = first; h < total; h += step) {
        int32_t x = h;
        const char* src;
        char* dst;
        bool rotate = turned;
        if (j.q.base) {
            if (x < j.q_heads) {
                src = j.q.base + 2 * ((int64_t)n * j.q.row + (int64_t)x * j.q.head);
                dst = j.q_out.base + 2 * ((int64_t)n * j.q_out.row + (int64_t)x * j.q_out.head);
                x = -1;
            } else {
                x -= j.q_heads;
            }
        }
        if (x >= 0) {
            if (pl.row < 0) continue;
            const bool key = x < j.step.kv_heads;
            if (!key) x -= j.step.kv_heads;
            const RowsView& rv = key ? j.k : j.v;
            src = rv.base + 2 * ((int64_t)n * rv.row + (int64_t)x * rv.head);
            dst = (key ? j.k_plane : j.v_plane) + 2 * (pl.row + (int64_t)x * D);
            rotate = rotate && key;
        }
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (has0) a = *reinterpret_cast<const uint4*>(src + 2 * e0);
        if (has1) b = *reinterpret_cast<const uint4*>(src + 2 * e1);
        if (rotate) {
            uint32_t* pa = reinterpret_cast<uint32_t*>(&a);
            uint32_t* pb = reinterpret_cast<uint32_t*>(&b);
            if (halves) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 u = N::to2(pa[k]), v = N::to2(pb[k]);
                    pa[k] = N::pack(u.x * c[2 * k] - v.x * s[2 * k], u.y * c[2 * k + 1] - v.y * s[2 * k + 1]);
                    pb[k] = N::pack(v.x * c[2 * k] + u.x * s[2 * k], v.y * c[2 * k + 1] + u.y * s[2 * k + 1]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 u = N::to2(pa[k]), v = N::to2(pb[k]);
                    // pairs past the rotated part keep their bits
                    if (e0 / 2 + k < rot / 2) pa[k] = N::pack(u.x * c[k] - u.y * s[k], u.y * c[k] + u.x * s[k]);
                    if (e0 / 2 + 4 + k < rot / 2) pb[k] = N::pack(v.x * c[4 + k] - v.y * s[4 + k], v.y * c[4 + k] + v.x * s[4 + k]);
                }
            }
        }
        if (has0) *reinterpret_cast<uint4*>(dst + 2 * e0) = a;
        if (has1) *reinterpret_cast<uint4*>(dst + 2 * e1) = b;
    }
}

// Halves that begin at no multiple of eight elements (a rotated part that 16 does not divide):
// a lane per pair, one element at a time, a warp over all heads of a token.  Bound by that: 32768
// tokens of 32 + 2 x 8 heads of 80 dims take 418 us with 20 rotated and 318 with 40, where the
// kernel above takes 94 with all 80; a decode step of 16 tokens 43 us.
template <bool HALF>
__global__ void __launch_bounds__(256) kvs_append_pairs_kernel(AppendJob j) {
    const uint32_t w = blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);
    if (w >= (uint32_t)j.step.total_q) {
        check_requests(j.step, w - (uint32_t)j.step.total_q);
        return;
    }
    const int32_t n = (int32_t)w;
    const int lane = threadIdx.x & 31;
    const Place pl = place_of(j, n);
    if (!pl.owned) return;
    const int32_t D = j.step.head_dim, rot = j.rot_dim, H = j.step.kv_heads;
    using N = Num<HALF>;
    using T = typename N::T;
    const int32_t qh = j.q.base ? j.q_heads : 0, total = qh + 2 * H;
    for (int32_t p = lane; p < D - rot / 2; p += 32) {          // pairs, then the dims behind them
        const bool turned = p < rot / 2;
        const int32_t e0 = turned ? p : p + rot / 2, e1 = p + rot / 2;
        float c = 1.0f, s = 0.0f;
        if (turned) turn(pl.pos, __ldg(j.turns + p), j.scale, c, s);
        for (int32_t h = 0; h < total; ++h) {
            const T* src;
            T* dst;
            bool rotate = turned;
            if (h < qh) {
                src = reinterpret_cast<const T*>(j.q.base) + (int64_t)n * j.q.row + (int64_t)h * j.q.head;
                dst = reinterpret_cast<T*>(j.q_out.base) + (int64_t)n * j.q_out.row + (int64_t)h * j.q_out.head;
            } else {
                if (pl.row < 0) continue;
                const bool key = h < qh + H;
                const int32_t x = key ? h - qh : h - qh - H;
                const RowsView& rv = key ? j.k : j.v;
                src = reinterpret_cast<const T*>(rv.base) + (int64_t)n * rv.row + (int64_t)x * rv.head;
                dst = reinterpret_cast<T*>(key ? j.k_plane : j.v_plane) + pl.row + (int64_t)x * D;
                rotate = rotate && key;
            }
            if (!turned) {
                dst[e0] = src[e0];
            } else {
                const T a = src[e0], b = src[e1];
                const float x = N::to(a), y = N::to(b);
                dst[e0] = rotate ? N::from(x * c - y * s) : a;
                dst[e1] = rotate ? N::from(y * c + x * s) : b;
            }
        }
    }
}

template <bool HALF>
cudaError_t append(const AppendJob& j, cudaStream_t s) {
    const int64_t rows = j.step.total_q;
    if (!j.interleaved && j.rot_dim % 16) {
        kvs_append_pairs_kernel<HALF><<<(warps_of(j.step, rows) + 7) / 8, 256, 0, s>>>(j);
        return cudaGetLastError();
    }
    const int lanes = (j.step.head_dim + 15) / 16;               // at most 8
    const int at_once = 32 / lanes, total = (j.q.base ? j.q_heads : 0) + 2 * j.step.kv_heads;
    // Few rows: a warp for every few heads, so that the GPU is filled; many (64 warps for each of
    // the 152 SMs): one warp per row, which works out the sines once.
    int parts = (total + at_once - 1) / at_once;
    while (parts > 1 && rows * parts > 152 * 64) parts = (parts + 1) / 2;
    kvs_append_kernel<HALF><<<(warps_of(j.step, rows * parts) + 7) / 8, 256, 0, s>>>(j, parts, lanes);
    return cudaGetLastError();
}

}  // namespace

void set_divisors(StepView& st) {
    const FastDiv block = make_fastdiv((uint32_t)st.block_size), group = make_fastdiv((uint32_t)(st.group ? st.group : 1));
    st.block_m = block.m;
    st.block_p = block.p;
    st.group_m = group.m;
    st.group_p = group.p;
}

int launch_append(const AppendJob& j, bool half, cudaStream_t s) {
    const cudaError_t e = half ? append<true>(j, s) : append<false>(j, s);
    return e == cudaSuccess ? 1 : -(int)e;
}

}  // namespace kvs
