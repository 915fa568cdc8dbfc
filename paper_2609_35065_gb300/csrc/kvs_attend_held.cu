// kvs_attend_held.cu -- attention of many packed rows over a window with sinks, on the tensor cores.
//
// The products and the softmax are those of kvs_attend_tc.cu: two tiles of 128 packed rows against 128
// keys a step, S = Q K^T in tensor memory -> P = 2^(c S - c m) back over it -> O += P V.  A window leaves
// a tile few steps (nine for 1024 tokens, two for 128), so that there a CTA's start and end took as long
// as its steps.  Here a CTA stays and takes one pair of tiles after the other, and every role runs ahead
// into the next: the loading warps fill the ring with its keys; the issuing warp sends for its rows as soon
// as the products that read the last ones are done, and issues its first S behind the last product with V;
// the softmax warps work out its rows' places beside that product, before they write the results.
//
// Steps go over the places of the cache (Held): the sinks' blocks, then those from the window's first token on.
// Of V, blocks with places that no row sees come row by row (cp.async), with zeros for those.  Where no box fits the cache's
// blocks, everything does: with blocks of one token the calls below take 1870 and 504 us.
//
// 16 suffixes of 2048 tokens behind 2048, 32 query heads of 128 dims on 8 and a window of 1024 with four
// sinks (0.55 TFLOP) take 446 to 481 us by card and power, 1.15 to 1.24 PFLOP/s; with a CTA to each pair of tiles 616.  Four prompts of 4001
// to 4096 tokens, 64 heads of 64 dims on 8 and a window of 128 (34 GFLOP, 303 MB) take 125 to 128 us (276).  What bounds
// them is the chain of a pair's hand-overs: with 128 dims the tensor cores are busy for 51% of the time and the issue
// slots for 48%, with 64 for 22% and 56%.  Of 15 steps or more (a window of 4096) 1.5 PFLOP/s are reached.
// Without the softmax's arithmetic the first took 395 of then 503 us and the second 112 of 151.
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

constexpr int kSoftmaxRegs = 104, kOtherRegs = 64;     // of a thread

template <int DP>
struct Plan {
    static constexpr int tile = kN * DP * 2;       // bytes of a tile of Q, K or V
    static constexpr int stages = 4;
    static constexpr int columns = 512;            // of tensor memory: S of each tile, then O
    // Issuing and loading warps.  A narrow tile's products and loads are both short, and a warp to each tile's products
    // keeps one tile from waiting for the other (four prompts of 4096 tokens with 64 dims and a window of 128: 123 us,
    // with one for both 131); a wide tile's 16 boxes want three warps to load (16 suffixes of 2048 tokens with 128 dims
    // and a window of 1024: 446 us, with two 482).
    static constexpr int issuers = DP == 128 ? 1 : 2, loaders = 4 - issuers;
    static_assert(loaders < stages, "a loading warp is less than a round ahead of the others");
    static constexpr bool staged = DP == 128;
    static constexpr int out = (kTiles + stages) * tile;             // [warp][32 rows][64 bytes], if staged
    static constexpr int bars = out + (staged ? 8 * kTiles * 2048 : 0);
    static constexpr int tops = bars + 256;        // [2][kTiles][128] binary32: maxima, sums that a row's threads exchange
    static constexpr int bytes = tops + 1024 * kTiles;
};

// q, s, p and o: one of each tile.
struct Bars {
    uint32_t q, s, p, o, full, free, done;
    __device__ Bars(uint32_t at, int stages) : q(at), s(at + 16), p(at + 32), o(at + 48), full(at + 64), free(full + 8 * stages), done(free + 8 * stages) {}
};

template <bool HALF, int DP>
__global__ void __launch_bounds__(kThreads, 1) kvs_attend_held_kernel(AttendJob j, const __grid_constant__ CUtensorMap k_map,
                                                                            const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map,
                                                                            ItemList list, int32_t q_boxes) {
    extern __shared__ __align__(1024) char raw[];
    using N = Num<HALF>;
    using P = Plan<DP>;
    constexpr float kMost = HALF ? 65504.0f : 1048576.0f;            // of a thread's weights of a step (half: of either sum)
    const StepView& st = j.step;
    const uint32_t base = smem_u32(raw);
    if (base & 1023) {                               // the swizzle needs it; there is no room to round it up
        record_error(st.err, KVS_ERR_UNSUPPORTED);
        return;
    }
    const uint32_t ring = base + kTiles * P::tile, ctl = base + P::bars;
    const Bars bar(ctl, P::stages);
    const uint32_t tmem_at = bar.done + 16;
    const int warp = warp_number(), wg = warp >> 2, lane = threadIdx.x & 31;
    const bool boxes = list.boxes;
    Walk walk(j, list);
    const int32_t per = walk.per;

    if (warp == kIssuer) tmem_alloc(tmem_at, P::columns);
    if (threadIdx.x == 0) {
        for (int t = 0; t < kTiles; ++t) {
            mbar_init(bar.q + 8 * t, q_boxes ? 1 : 256);
            mbar_init(bar.s + 8 * t, 1);
            mbar_init(bar.p + 8 * t, 8);
            mbar_init(bar.o + 8 * t, 1);
        }
        for (int i = 0; i < P::stages; ++i) {
            mbar_init(bar.full + 8 * i, 1);
            mbar_init(bar.free + 8 * i, P::issuers);
        }
        for (int i = 0; i < P::issuers; ++i) mbar_init(bar.done + 8 * i, 1);
        mbar_init_fence();
    }
    constexpr int kLoader = kIssuer + P::issuers;
    if (warp == kLoader && lane == 0) {
        if (boxes) {
            prefetch_map(&k_map);
            prefetch_map(&v_map);
        }
        if (q_boxes) prefetch_map(&q_map);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_at) : "memory");
    auto s_at = [&](int t) { return tmem + 128u * t; };
    auto o_at = [&](int t) { return tmem + 128u * kTiles + (uint32_t)DP * t; };

    // A wait that does not end is recorded; every role then leaves its loop (the others' waits end too).
    auto wait = [&](uint32_t b, uint32_t parity) {
        if (mbar_wait(b, parity, kWaitLimitNs)) return true;
        record_error(st.err, KVS_ERR_TIMEOUT);
        return false;
    };

    // The softmax's warps get registers of the others' (512 x 104 + 128 x 64 = 640 x 96).
    if (warp >= kIssuer) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kOtherRegs));
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kSoftmaxRegs));
    if (warp >= kLoader) {
        // ---- K and V: the ring's tile i is K (even) or V (odd) of step i / 2 of all items' -----
        // A warp brings every P::loaders-th tile whole: its waits and look-ups are beside the others' then.  A stage is
        // free in the order of the ring, so that a wait for a stage's last user follows those before it.
        const int w = warp - kLoader;
        int pending = -1;                                    // tile with cp.async rows, not yet announced
        auto announce = [&]() {
            cp_wait<0>();
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.full + 8 * pending);
            pending = -1;
        };
        // The tile at hand, k of an item, and whether there is one.
        struct Cursor {
            Item    it;
            int32_t k;
            bool    have;
        };
        auto ahead = [&](Cursor& c, int32_t n) {
            c.k += n;
            while (c.have && c.k >= 2 * c.it.steps) {
                c.k -= 2 * c.it.steps;
                c.have = walk.next_active(c.it);
            }
        };
        auto look_up = [&](const Cursor& c) {
            return c.have && boxes ? box_of<DP, 1>(st, st.tables + (int64_t)c.it.r * st.table_stride, c.it.held, (c.k >> 1) * kN, c.it.T, 0, lane) : Box{};
        };
        Cursor now{{}, 0, false};
        now.have = walk.next_active(now.it);
        ahead(now, w);
        Box box = look_up(now);
        uint32_t i = w;
        bool ok = true;
        while (now.have && ok) {
            Cursor next = now;
            ahead(next, P::loaders);
            const Box after = look_up(next);
            const uint32_t stage = i % P::stages, round = i / P::stages;
            if (round > 0) {
                ok = __all_sync(0xffffffffu, lane != 0 || wait(bar.free + 8 * stage, (round - 1) & 1));
                if (!ok) break;
            }
            const Item& it = now.it;
            const uint32_t dst = ring + stage * P::tile;
            const int32_t t0 = (now.k >> 1) * kN;
            const bool is_v = now.k & 1;
            if (boxes && (!is_v || tile_whole(it, t0, j.sinks))) {
                tile_boxes<DP>(dst, is_v ? &v_map : &k_map, st, it.h, box, bar.full + 8 * stage, lane);
                if (pending >= 0) announce();
            } else {
                if (pending >= 0) announce();
                if (boxes) tile_mixed<DP>(dst, &v_map, j.v_plane, st, it.h, box, bar.full + 8 * stage, t0, it.all.lo, it.T, j.sinks, lane);
                else tile_rows<DP, 32>(dst, is_v ? j.v_plane : j.k_plane, st, st.tables + (int64_t)it.r * st.table_stride, it.h, it.held, t0, it.all.lo, it.T, j.sinks, lane);
                cp_commit();
                pending = stage;
            }
            // A tile of V may wait for its rows until this warp's next tile is sent for: what frees that one's stage does not
            // need it.  Of tiles of K by rows that would not hold.
            if (pending >= 0 && !boxes) announce();
            i += P::loaders;
            now = next;
            box = after;
        }
        if (pending >= 0) announce();
        // Before the CTA leaves, every load has landed (all of them have when the products are done).
        if (!ok) {
            for (uint32_t k = w; k <= i; k += P::loaders)
                if (k + P::stages > i) mbar_wait(bar.full + 8 * (k % P::stages), (k / P::stages) & 1, kWaitLimitNs);
        }
    } else if (warp >= kIssuer) {
        // ---- the products of tiles t0 to t1: the warp waits together, one lane issues ---
        const int t0 = P::issuers == 2 ? warp - kIssuer : 0, t1 = P::issuers == 2 ? t0 + 1 : kTiles;
        // a negative scale's sign goes into the products, so that maxima of S are those of the scores
        const uint32_t id_s = tc_idesc(HALF, kN, false) | (j.scale_log2 < 0.0f ? kNegA : 0u);
        constexpr uint32_t id_o = tc_idesc(HALF, DP, true);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t q_desc = tc_desc(base, 16, 1024), k_desc = tc_desc(ring, 16, 1024), v_desc = tc_desc(ring, kN * 128, 1024);
        auto issue_s = [&](int t, int stage) {
            const uint64_t a = tc_ahead(q_desc, t * P::tile), b = tc_ahead(k_desc, stage * P::tile);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                const uint32_t off = (k >> 2) * kN * 128 + (k & 3) * 32;
                tc_mma_ss(tm + 128 * t, tc_ahead(a, off), tc_ahead(b, off), id_s, k > 0);
            }
            tc_commit(bar.s + 8 * t);
        };
        // An item's rows to a tile's place, when the products that read the last ones are done.
        auto send_rows = [&](const Item& x, int t) {
            if (elect_one()) {
                mbar_expect_tx(bar.q + 8 * t, (uint32_t)per * DP * 2);
#pragma unroll
                for (int c = 0; c < DP / 64; ++c)
                    tma_load_3d(base + t * P::tile + c * kM * 128, &q_map, 64 * c, x.h * st.group, x.q.q0 + (x.row0 + t * per) / st.group, bar.q + 8 * t);
            }
            __syncwarp();
        };
        auto issue_o = [&](int t, int stage, bool add) {
            const uint64_t b = tc_ahead(v_desc, stage * P::tile);
#pragma unroll
            for (int k = 0; k < kN / 16; ++k)
                tc_mma_ts(tm + 128 * kTiles + DP * t, tm + 128 * t + 8 * k, tc_ahead(b, k * 2048), id_o, add || k > 0);
        };
        int32_t stage = 0, round = 0;                        // of the next tile of the ring
        auto take = [&](int32_t& s, int32_t& r) {
            s = stage;
            r = round;
            if (++stage == P::stages) {
                stage = 0;
                ++round;
            }
        };
        auto filled = [&](int32_t stage, int32_t round) { return wait(bar.full + 8 * stage, round & 1); };
        Item it;
        bool have = walk.next_active(it);
        int32_t steps = it.steps;
        uint32_t gone = 0, items = 0;                        // steps and items that are done with
        bool ok = true;
        if (have) {
            int32_t ks, kr;
            take(ks, kr);
            if (q_boxes)
                for (int t = t0; t < t1; ++t) send_rows(it, t);
            for (int t = t0; t < t1; ++t) ok = wait(bar.q + 8 * t, 0) && ok;
            ok = __all_sync(0xffffffffu, filled(ks, kr) && ok);
            if (ok) {
                tc_fence_after();
                if (elect_one()) {
                    for (int t = t0; t < t1; ++t) issue_s(t, ks);
                    tc_commit(bar.free + 8 * ks);
                }
                __syncwarp();
            }
        }
        while (have && ok) {
            Item after;
            const bool follows = walk.next_active(after);
            for (int32_t k = 0; ok && k < steps; ++k, ++gone) {
                const bool last = k + 1 == steps, more = !last || follows;
                int32_t vs, vr, ks = 0, kr = 0;
                take(vs, vr);
                if (more) take(ks, kr);
                if (last && more && q_boxes) {
                    for (int t = t0; t < t1; ++t) {
                        ok = wait(bar.s + 8 * t, gone & 1) && ok;
                        if (__all_sync(0xffffffffu, ok)) send_rows(after, t);
                    }
                }
                // V of this step and K of the next were loaded long ago; P is what is waited for.  A wait
                // that ran out ends the loop at the next vote.
                ok = filled(vs, vr) && (!more || filled(ks, kr)) && ok;
                // the next item's rows, where the softmax warps bring them, come behind this one's results
                const bool later = last && more && !q_boxes;
                auto next_s = [&](int t) {
                    if (last) ok = wait(bar.q + 8 * t, (items + 1) & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
                    if (elect_one()) {
                        issue_s(t, ks);
                        if (t == t1 - 1) tc_commit(bar.free + 8 * ks);
                    }
                };
                for (int t = t0; t < t1; ++t) {
                    ok = wait(bar.p + 8 * t, gone & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
                    if (elect_one()) {
                        issue_o(t, vs, k > 0);
                        if (last) tc_commit(bar.o + 8 * t);
                        if (t == t1 - 1) tc_commit(bar.free + 8 * vs);
                    }
                    if (more && !later) next_s(t);
                }
                if (later)
                    for (int t = t0; t < t1; ++t) next_s(t);
                ok = __all_sync(0xffffffffu, ok);
            }
            ++items;
            steps = after.steps;
            have = follows;
        }
        if (!ok && elect_one()) {
            // what was issued is done before the CTA leaves
            tc_commit(bar.done + 8 * (warp - kIssuer));
            mbar_wait(bar.done + 8 * (warp - kIssuer), 0, kWaitLimitNs);
            for (int t = t0; t < t1; ++t) {
                mbar_wait(bar.q + 8 * t, 0, kWaitLimitNs);
                mbar_wait(bar.q + 8 * t, 1, kWaitLimitNs);
            }
        }
        __syncwarp();
    } else {
        // ---- softmax of tile tl: row t, keys 64 half ... of a step -----------------------
        const int tl = wg >> 1, half = wg & 1, t = threadIdx.x & 127;
        const uint32_t own = base + tl * P::tile;                    // the tile's Q
        // The warps of a row's two halves agree, and wait for one another, under a barrier of their
        // own.  After a wait that ran out, both still go through all steps (on whatever is there).
        const int pair = 1 + tl * 4 + (warp & 3);
        float* tops = reinterpret_cast<float*>(raw + P::tops);
        const float c = fmaxf(fabsf(j.scale_log2), 1e-36f);         // a zero scale keeps -infinity * c what it is
        const float c_low = j.scale_log2 < 0.0f ? -j.scale_low : j.scale_low;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;          // lane 32 (warp % 4) of tensor memory
        const uint32_t s_own = s_at(tl) + lanes + 64 * half, o_own = o_at(tl) + lanes + DP / 2 * half;
        uint32_t gone = 0, items = 0;
        bool ok = true;
        RowOf row{};                                                 // this thread's of the item at hand
        int32_t steps = 0;
        auto take = [&]() {
            Item it;
            if (!walk.next(it)) return false;
            steps = it.steps;
            if (!q_boxes && steps > 0) {
                constexpr int CH = DP / 8;
#pragma unroll 4
                for (int v = threadIdx.x & 255; v < kM * CH; v += 256) {
                    const int i = v / CH, d = v % CH;
                    const bool there = i < per && tl * per + i < it.rows && 8 * d < st.head_dim;
                    int32_t g;
                    const int32_t tok = token_of(st, there ? it.row0 + tl * per + i : 0, g);
                    cp_async16(own + (d >> 3) * kM * 128 + i * 128 + (((d & 7) ^ (i & 7)) << 4),
                               j.q.base + (there ? 2 * ((int64_t)(it.q.q0 + tok) * j.q.row + (int64_t)(it.h * st.group + g) * j.q.head + 8 * d) : 0), there);
                }
                cp_commit();
                cp_wait<0>();
                fence_async_smem();
                mbar_arrive(bar.q + 8 * tl);
            }
            row = row_of_item(j, it, per, tl, t);
            return true;
        };
        bool have = take();
        while (have) {
            // log2 of a weight at the reference
            const float top_at = HALF ? half_top(steps * kN, 3) : 0.0f;
            float m = kNone, l0 = 0.0f, l1 = 0.0f;
            for (int32_t k = 0; k < steps; ++k, ++gone) {
                ok = ok && __all_sync(0xffffffffu, wait(bar.s + 8 * tl, gone & 1));
                tc_fence_after();
                // the keys of this half that the row sees, a bit to each
                const int32_t t0 = k * kN + 64 * half;
                auto below = [&](int32_t x) { return x - t0 <= 0 ? 0ull : x - t0 >= 64 ? ~0ull : (1ull << (x - t0)) - 1; };
                const uint64_t seen = below(row.see.hi) & (~below(row.see.lo) | below(j.sinks));
                const uint32_t bits[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
                // of either 32: whether some of the warp's rows do not see all of them, and whether some see any
                bool edge[2], some[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    edge[b] = __any_sync(0xffffffffu, bits[b] != ~0u);
                    some[b] = __any_sync(0xffffffffu, row.live && bits[b]);
                }
                auto load_s = [&](uint32_t* sr, int b) {
                    tmem_ld32(sr, s_own + 32 * b);
                    tmem_wait_ld();
                    tmem_loaded32(sr);
                    float* s = reinterpret_cast<float*>(sr);
                    if (edge[b]) {
#pragma unroll
                        for (int n = 0; n < 32; ++n) s[n] = bits[b] >> n & 1 ? s[n] : kNone;
                    }
                };
                if (k == 0) {
                    // The first reference is the maximum of the first 32 places, the sinks among them, which both
                    // halves take for themselves: one that both shared of all 128 had the row wait twice as long.
                    const uint32_t first = bits_below(row.see.hi) & (~bits_below(row.see.lo) | bits_below(j.sinks));
                    uint32_t sr[32];
                    tmem_ld32(sr, s_at(tl) + lanes);
                    tmem_wait_ld();
                    tmem_loaded32(sr);
                    float* s = reinterpret_cast<float*>(sr);
#pragma unroll
                    for (int n = 0; n < 32; ++n) s[n] = first >> n & 1 ? s[n] : kNone;
#pragma unroll
                    for (int n = 0; n < 32; n += 2) m = max3(m, s[n], s[n + 1]);
                }
                // Against this step's own maximum: the first step that rows see any key of.
                bool exact = __any_sync(0xffffffffu, row.live && m == kNone && (row.see.lo < (k + 1) * kN || j.sinks > k * kN) && row.see.hi > k * kN);
                uint32_t pk[32];
                float a0, a1;
                while (true) {
                    if (exact) {
                        float top = kNone;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            if (!some[b]) continue;
                            uint32_t sr[32];
                            load_s(sr, b);
                            float* s = reinterpret_cast<float*>(sr);
#pragma unroll
                            for (int n = 0; n < 32; n += 2) top = max3(top, s[n], s[n + 1]);
                        }
                        tops[half * 128 * kTiles + tl * 128 + t] = top;
                        bar_some(pair, 64);
                        top = fmaxf(top, tops[(half ^ 1) * 128 * kTiles + tl * 128 + t]);
                        // m = -infinity: nothing was summed yet, and O is zero or not yet written
                        const bool raise = top > m;
                        const float f = raise && m != kNone ? exp2_fast((m - top) * c) : 1.0f;
                        if (raise) m = top;
                        l0 *= f;
                        l1 *= f;
                        if (k > 0 && __any_sync(0xffffffffu, f != 1.0f)) {
                            // the products before are done: this step's S was issued behind them
#pragma unroll
                            for (int b = 0; b < DP / 32; ++b) {
                                uint32_t o[16];
                                tmem_ld16(o, o_own + 16 * b);
                                tmem_wait_ld();
                                tmem_loaded16(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16(o_own + 16 * b, o);
                            }
                        }
                    }
                    const float off = m == kNone ? 0.0f : top_at - m * c;
                    a0 = a1 = 0.0f;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (!some[b]) {
#pragma unroll
                            for (int n = 0; n < 16; ++n) pk[16 * b + n] = 0;
                            continue;
                        }
                        uint32_t sr[32];
                        load_s(sr, b);
                        float* s = reinterpret_cast<float*>(sr);
#pragma unroll
                        for (int n = 0; n < 16; ++n) {
                            float x = s[2 * n], y = s[2 * n + 1];
                            fma2(x, y, c, off);
                            x = exp2_fast(x);
                            y = exp2_fast(y);
                            add2(a0, a1, x, y);
                            pk[16 * b + n] = N::pack(x, y);
                        }
                    }
                    // No weight is above its sum.  Both halves of S are read behind this: P goes over the
                    // first one's columns.
                    const bool again = bar_or(pair, 64, !exact && row.live && (HALF ? fmaxf(a0, a1) : a0 + a1) > kMost);
                    if (!again) break;
                    exact = true;
                }
                add2(l0, l1, a0, a1);
                tmem_st32(s_at(tl) + lanes + 32 * half, pk);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.p + 8 * tl);
            }
            // ---- the rows' results --------------------------------------------------------
            float l = l0 + l1;
            tops[half * 128 * kTiles + tl * 128 + t] = l;
            bar_some(pair, 64);
            l = tops[tl * 128 + t] + tops[128 * kTiles + tl * 128 + t];
            bar_some(pair, 64);                                      // the next item's maxima go over them
            if (row.live && ok && half == 0 && j.lse) j.lse[row.lse] = l == 0.0f ? kNone : ((m == kNone ? kNone : fmaf(m, c_low, m * c - top_at)) + log2f(l)) * 0.69314718055994531f;
            const bool some_o = steps > 0;
            char* to = ok ? row.out : nullptr;
            if (some_o) ++items;
            // the next item's rows while the last product with V is under way (its queries, where these warps bring
            // them, go to a place that the last S has left)
            have = take();
            if (some_o && !__all_sync(0xffffffffu, !ok || wait(bar.o + 8 * tl, (items - 1) & 1))) ok = false;
            if (!ok) to = nullptr;
            tc_fence_after();
            const float f = l > 0.0f ? 1.0f / l : l;
            // Through shared memory, 64 bytes of 32 rows at a time, so that four lanes write a row's piece.
            // Narrow rows are written as they are: by way of shared memory four prompts of 4096 tokens with 64 dims take 157 us, 148 so.
            const uint32_t stage = base + P::out + warp * 2048;
#pragma unroll
            for (int b = 0; b < DP / 64; ++b) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    uint32_t o[16];
                    if (some_o) {
                        tmem_ld16(o, o_own + 32 * b + 16 * x);
                        tmem_wait_ld();
                        tmem_loaded16(o);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = some_o && l != 0.0f ? __float_as_uint(__uint_as_float(o[e]) * f) : 0u;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t y[4];
#pragma unroll
                        for (int n = 0; n < 4; ++n) y[n] = N::pack(__uint_as_float(o[8 * e + 2 * n]), __uint_as_float(o[8 * e + 2 * n + 1]));
                        const int d = DP / 2 * half + 32 * b + 16 * x + 8 * e;
                        if (!P::staged) {
                            if (to && d < st.head_dim) *reinterpret_cast<uint4*>(to + 2 * d) = make_uint4(y[0], y[1], y[2], y[3]);
                        } else st_shared16(stage + lane * 64 + (((2 * x + e) ^ (lane >> 1 & 3)) << 4), y[0], y[1], y[2], y[3]);
                    }
                }
                if (!P::staged) continue;
                __syncwarp();
                const int d = DP / 2 * half + 32 * b + 8 * (lane & 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * i + (lane >> 2);
                    char* dst = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, (unsigned long long)to, r));
                    if (dst && d < st.head_dim) *reinterpret_cast<uint4*>(dst + 2 * d) = ld_shared16(stage + r * 64 + (((lane & 3) ^ (r >> 1 & 3)) << 4));
                }
                __syncwarp();
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssuer) tmem_dealloc(tmem, P::columns);
}

template <bool HALF, int DP>
cudaError_t attend_held(const AttendJob& j, int sms, cudaStream_t s) {
    using P = Plan<DP>;
    CUtensorMap km{}, vm{}, qm{};
    const bool boxes = plane_map(&km, j.step, j.k_plane, HALF) && plane_map(&vm, j.step, j.v_plane, HALF), q_boxes = rows_map(&qm, j.step, j.q, HALF);
    const int64_t total = held_items(j.step), tiles = total / ((int64_t)j.step.kv_heads * j.step.requests);
    const ItemList list{make_fastdiv((uint32_t)tiles), make_fastdiv((uint32_t)j.step.kv_heads), (uint32_t)total, boxes};
    const unsigned grid = (unsigned)(total < sms ? total : sms);
    auto* k = kvs_attend_held_kernel<HALF, DP>;
    // What the warps take on and give up has to be what the CTA was launched with, or they would wait for ever.
    static const bool enough = [&] {
        cudaFuncAttributes a{};
        return cudaFuncGetAttributes(&a, k) == cudaSuccess && a.numRegs * kThreads >= kSoftmaxRegs * 32 * kIssuer + kOtherRegs * 128;
    }();
    if (!enough) return launch_attend_tc(j, HALF, s);
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, P::bytes);
    if (e != cudaSuccess) return e;
    // Not by launch_behind: an item's lengths, loaded coherently, wait where they now come ahead (the four prompts
    // 129 us for 125, and among other calls the 4 that are saved between them).
    k<<<grid, kThreads, P::bytes, s>>>(j, km, vm, qm, list, (int32_t)q_boxes);
    return cudaGetLastError();
}

}  // namespace

int64_t held_items(const StepView& st) {
    const int64_t rows = kTiles * tile_rows_of(st.group), tiles = ((int64_t)st.max_q * st.group + rows - 1) / rows;
    return tiles * st.kv_heads * st.requests;
}

cudaError_t launch_attend_held(const AttendJob& j, bool half, int sms, cudaStream_t s) {
    if (j.step.head_dim <= 64) return half ? attend_held<true, 64>(j, sms, s) : attend_held<false, 64>(j, sms, s);
    return half ? attend_held<true, 128>(j, sms, s) : attend_held<false, 128>(j, sms, s);
}

}  // namespace kvs
