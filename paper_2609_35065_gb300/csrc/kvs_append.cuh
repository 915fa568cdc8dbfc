// kvs_append.cuh -- what the append kernels share: a position's sines, a row's place in the cache.
#pragma once

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
template <bool LATE = false>
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
            if (load_of<LATE>(st.q_starts + mid) <= n) lo = mid;
            else hi = mid;
        }
        r = lo;
    }
    const Request q = load_request<LATE>(st, r);
    const int32_t t = q.T - q.n + (n - q.q0);
    pl.owned = n >= q.q0 && n < q.q0 + q.n;
    if (pl.owned && t >= 0) pl.row = row_of<LATE>(st, st.tables + (int64_t)r * st.table_stride, t);
    pl.pos = j.positions ? load_of<LATE>(j.positions + n) : max(t, 0);
    return pl;
}

// A request out of bounds may have no row that leads to it (its range falls, or is empty): the
// grid has warps behind the rows' own that look at 32 requests each (looking behind their own work,
// the rows' warps took 1.5% longer).
template <bool LATE = false>
__device__ __forceinline__ void check_requests(const StepView& st, uint32_t group) {
    const uint32_t r = 32 * group + (threadIdx.x & 31);
    if (st.q_starts && r < (uint32_t)st.requests) load_request<LATE>(st, r);
}
inline uint32_t warps_of(const StepView& st, int64_t row_warps) { return (uint32_t)(row_warps + (st.q_starts ? (st.requests + 31) / 32 : 0)); }

}  // namespace
}  // namespace kvs
