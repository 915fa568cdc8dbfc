// kvs_attend_held.cuh -- what the kernels of a window with sinks share whose CTAs stay: pairs of row tiles,
// which a CTA takes one after the other, and their rows.
#pragma once

#include "kvs_tcgen05.cuh"

namespace kvs {
namespace {

constexpr int kM = 128, kN = 128;                  // rows of a tile, keys of a tile of K or V
constexpr int kTiles = 2;
constexpr int kIssuer = 8 * kTiles;                // the issuing warps, behind the softmax's; then the loading ones
constexpr int kThreads = 256 * kTiles + 128;
constexpr float kNone = -INFINITY;

// What a CTA works on: two tiles of a request's packed rows, of one KV head.
struct Item {
    Request q;
    Span    all;                                   // places that some row sees
    Held    held;
    int32_t r, h, row0, rows, steps, T;            // T: places of the cache; steps of 128 up to the last seen one
};

// The items of a launch, in the order of request, KV head and row tiles.
struct ItemList {
    FastDiv  tiles, heads;
    uint32_t total;
    int32_t  boxes;                                // whether K and V come by boxes
};

// Goes over this CTA's items; every role does so by itself.
struct Walk {
    const AttendJob& j;
    const ItemList&  list;
    const int32_t    per, unit;                    // rows of a tile; tokens that places are held in
    uint32_t at;

    __device__ __forceinline__ Walk(const AttendJob& job, const ItemList& l)
        : j(job), list(l), per(tile_rows_of(job.step.group)), unit(l.boxes ? min(job.step.block_size, kN) : 1), at(blockIdx.x) {}
    // Whole units up to t: divided as block_of divides, or by 128.
    __device__ __forceinline__ int32_t units(int32_t t) const {
        return unit == 1 ? t : unit == j.step.block_size ? (int32_t)block_of(j.step, t) : t >> 7;
    }
    __device__ __forceinline__ bool next(Item& it) {
        const StepView& st = j.step;
        while (at < list.total) {
            const uint32_t p = fdiv(at, list.tiles), tile = at - p * list.tiles.d;
            at += gridDim.x;
            it.r = fdiv(p, list.heads);
            it.h = p - it.r * list.heads.d;
            it.row0 = (int32_t)tile * kTiles * per;
            it.q = load_request(st, it.r);
            it.rows = min(kTiles * per, it.q.n * st.group - it.row0);
            if (it.rows <= 0) continue;
            int32_t g;
            const int32_t tok = token_of(st, it.row0, g);
            it.all = seen_by(it.q, tok, token_of(st, it.row0 + it.rows - 1, g), j.causal, j.window);
            // as held_of
            const int32_t first = units(it.all.lo) * unit;
            it.held.cut = min(units(min(j.sinks, it.all.lo) + unit - 1) * unit, first);
            it.held.shift = first - it.held.cut;
            it.all = in_places(it.held, it.all);
            it.T = it.q.T - it.held.shift;
            it.steps = it.all.hi > it.all.lo ? (it.all.hi + kN - 1) / kN : 0;
            return true;
        }
        return false;
    }
    // ... of those whose rows see something
    __device__ __forceinline__ bool next_active(Item& it) {
        bool some;
        do some = next(it);
        while (some && it.steps == 0);
        return some;
    }
};

// A thread's row of an item: whether there is one, what it sees (in places), where its results go -- its first
// element in `out` and its entry of lse.
struct RowOf {
    Span    see;
    char*   out;
    int64_t lse;
    bool    live;
};
__device__ __forceinline__ RowOf row_of_item(const AttendJob& j, const Item& it, int32_t per, int tl, int t) {
    const StepView& st = j.step;
    int32_t g;
    const int32_t tok = token_of(st, it.row0 + tl * per + t, g);
    // a tile's rows without a token see everything, so that their warp need not mask for them
    RowOf r{Span{0, INT32_MAX}, nullptr, 0, t < per && tl * per + t < it.rows};
    if (r.live) {
        r.see = in_places(it.held, seen_by(it.q, tok, tok, j.causal, j.window));
        r.out = j.out.base + 2 * ((int64_t)(it.q.q0 + tok) * j.out.row + (int64_t)(it.h * st.group + g) * j.out.head);
        r.lse = (int64_t)(it.q.q0 + tok) * (st.kv_heads * st.group) + it.h * st.group + g;
    }
    return r;
}

// Bits below x of the 32 from 0 on.
__device__ __forceinline__ uint32_t bits_below(int32_t x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1; }

// Whether each of the tile's places from t0 on is seen by some row: where not, V has to be zeros.
__device__ __forceinline__ bool tile_whole(const Item& it, int32_t t0, int32_t sinks) {
    return (t0 >= it.all.lo || min(t0 + kN, it.all.lo) <= sinks) && t0 + kN <= it.T;
}

}  // namespace
}  // namespace kvs
