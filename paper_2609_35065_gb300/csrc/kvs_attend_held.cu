// kvs_attend_held.cu -- attention of many packed rows over a window with sinks, on the tensor cores.
//
// The products and the softmax are those of kvs_attend_tc.cu: two tiles of 128 packed rows against 128
// keys a step, S = Q K^T in tensor memory -> P = 2^(c S - c m) back over it -> O += P V.  A window leaves
// a tile few steps (nine for 1024 tokens, two for 128), so that there a CTA's start and end took as long
// as its steps.  Here a CTA stays and takes one pair of tiles after the other, and every role runs ahead
// into the next: the loading warps fill the ring with its keys and, once S of the last step is done, Q's
// place with its rows; the issuing warp sends its first S behind the last product with V, while the softmax
// warps still write the results.
//
// Steps go over the places of the cache (Held): the sinks' blocks, then those from the window's first token on.
#include "kvs_tcgen05.cuh"

namespace kvs {
namespace {

constexpr int kM = 128, kN = 128;                  // rows of a tile, keys of a step
constexpr int kTiles = 2;
constexpr int kLoaders = 3;
constexpr int kIssuer = 8 * kTiles;                // the issuing warp, behind the softmax's; then the loading ones
constexpr float kNone = -INFINITY;

template <int DP>
struct Plan {
    static constexpr int threads = 256 * kTiles + 128;
    static constexpr int tile = kN * DP * 2;       // bytes of a tile of Q, K or V
    static constexpr int stages = 4;
    static constexpr int columns = 512;            // of tensor memory: S of each tile, then O
    static constexpr bool staged = DP == 128;
    static constexpr int out = (kTiles + stages) * tile;             // [warp][32 rows][64 bytes], if staged
    static constexpr int bars = out + (staged ? 8 * kTiles * 2048 : 0);
    static constexpr int tops = bars + 256;        // [2][kTiles][128] binary32: maxima, sums that a row's threads exchange
    static constexpr int bytes = tops + 1024 * kTiles;
};

// q, q_free, s, p and o: one of each tile.
struct Bars {
    uint32_t q, q_free, s, p, o, full, free, done;
    __device__ Bars(uint32_t at, int stages)
        : q(at), q_free(at + 16), s(at + 32), p(at + 48), o(at + 64), full(at + 80), free(full + 8 * stages), done(free + 8 * stages) {}
};

// What a CTA works on: two tiles of a request's packed rows, of one KV head.
struct Item {
    Request q;
    Span    all;                                   // places that some row sees
    Held    held;
    int32_t r, h, row0, rows, steps, T;            // T: places of the cache
};

template <bool HALF, int DP>
__global__ void __launch_bounds__(Plan<DP>::threads, 1) kvs_attend_held_kernel(AttendJob j, const __grid_constant__ CUtensorMap k_map,
                                                                            const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map,
                                                                            int32_t boxes, int32_t q_boxes, FastDiv tiles, FastDiv heads_of, uint32_t total) {
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
    const uint32_t tmem_at = bar.done + 8;
    const int warp = warp_number(), wg = warp >> 2, lane = threadIdx.x & 31;
    const int32_t per = tile_rows_of(st.group);

    uint32_t at_item = blockIdx.x;
    const int32_t unit = boxes ? min(st.block_size, kN) : 1;
    // floor and ceiling in units, of which there is one to a box: divided as block_of divides, or by 128
    auto units = [&](int32_t t) { return unit == 1 ? t : unit == st.block_size ? (int32_t)block_of(st, t) : t >> 7; };
    auto next_item = [&](Item& it) {
        while (at_item < total) {
            // the item's pair of request and KV head, and its pair of row tiles
            const uint32_t p = fdiv(at_item, tiles), tile = at_item - p * tiles.d;
            at_item += gridDim.x;
            it.r = fdiv(p, heads_of);
            it.h = p - it.r * heads_of.d;
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
    };
    // ... of those whose rows see something
    auto next_active = [&](Item& it) {
        bool some;
        do some = next_item(it);
        while (some && it.steps == 0);
        return some;
    };

    if (warp == kIssuer) tmem_alloc(tmem_at, P::columns);
    if (threadIdx.x == 0) {
        for (int t = 0; t < kTiles; ++t) {
            mbar_init(bar.q + 8 * t, q_boxes ? 1 : 256);
            mbar_init(bar.q_free + 8 * t, 1);
            mbar_init(bar.s + 8 * t, 1);
            mbar_init(bar.p + 8 * t, 8);
            mbar_init(bar.o + 8 * t, 1);
        }
        for (int i = 0; i < P::stages; ++i) {
            mbar_init(bar.full + 8 * i, kLoaders);
            mbar_init(bar.free + 8 * i, 1);
        }
        mbar_init(bar.done, 1);
        mbar_init_fence();
    }
    if (warp == kIssuer + 1 && lane == 0) {
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
    if (warp >= kIssuer) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    if (warp > kIssuer) {
        // ---- K and V: the ring's tile i is K (even) or V (odd) of step i / 2 of all items' -----
        const int t = threadIdx.x - 32 * (kIssuer + 1), w = warp - kIssuer - 1;
        int pending = -1;                                    // cp.async tile not yet announced
        auto announce = [&]() {
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.full + 8 * pending);
            pending = -1;
        };
        Item it, after;
        bool have = next_active(it), ok = true;
        Box box{}, next{};
        if (have && boxes) next = box_of<DP, kLoaders>(st, st.tables + (int64_t)it.r * st.table_stride, it.held, 0, it.T, w, lane);
        uint32_t i = 0, stage = 0, round = 0, items = 0, rows_of[kTiles] = {};        // items whose rows each tile's place was sent
        while (have && ok) {
            const bool more = next_active(after);
            const int32_t* table = st.tables + (int64_t)it.r * st.table_stride;
            for (int32_t k = 0; k < 2 * it.steps; ++k, ++i) {
                if (boxes && !(k & 1)) {
                    // K's and V's tiles of a step are in the same blocks; the next step's are looked up a step ahead
                    box = next;
                    if (k + 2 < 2 * it.steps) next = box_of<DP, kLoaders>(st, table, it.held, ((k >> 1) + 1) * kN, it.T, w, lane);
                    else if (more) next = box_of<DP, kLoaders>(st, st.tables + (int64_t)after.r * st.table_stride, after.held, 0, after.T, w, lane);
                }
                if (round > 0) {
                    ok = __all_sync(0xffffffffu, lane != 0 || wait(bar.free + 8 * stage, (round - 1) & 1));
                    if (!ok) break;
                }
                const uint32_t dst = ring + stage * P::tile;
                const int32_t t0 = (k >> 1) * kN;
                const bool is_v = k & 1;
                // Where no row sees anything V has to be zeros; K may be anything there.
                const bool whole = (t0 >= it.all.lo || min(t0 + kN, it.all.lo) <= j.sinks) && t0 + kN <= it.T;
                if (boxes && (whole || !is_v)) {
                    tile_boxes<DP>(dst, is_v ? &v_map : &k_map, st, it.h, box, bar.full + 8 * stage, lane);
                    if (pending >= 0) {
                        cp_wait<0>();
                        announce();
                    }
                } else {
                    if (boxes) {
                        tile_mixed<DP>(dst, &v_map, j.v_plane, st, it.h, box, bar.full + 8 * stage, t0, it.all.lo, it.T, j.sinks, lane);
                    } else {
                        tile_rows<DP, 32 * kLoaders>(dst, is_v ? j.v_plane : j.k_plane, st, table, it.h, it.held, t0, it.all.lo, it.T, j.sinks, t);
                    }
                    cp_commit();
                    if (pending >= 0) {
                        cp_wait<1>();
                        announce();
                    }
                    pending = stage;
                }
                if (k == 0 && w == 0 && q_boxes) {
                    // the item's rows, where the last one's lay
                    for (int x = 0; ok && x < kTiles; ++x) {
                        if (items > 0) ok = __all_sync(0xffffffffu, lane != 0 || wait(bar.q_free + 8 * x, (items - 1) & 1));
                        if (!ok) break;
                        rows_of[x] = items + 1;
                        if (lane == 0) {
                            mbar_expect_tx(bar.q + 8 * x, (uint32_t)per * DP * 2);
#pragma unroll
                            for (int c = 0; c < DP / 64; ++c)
                                tma_load_3d(base + x * P::tile + c * kM * 128, &q_map, 64 * c, it.h * st.group, it.q.q0 + (it.row0 + x * per) / st.group, bar.q + 8 * x);
                        }
                        __syncwarp();
                    }
                }
                if (++stage == P::stages) {
                    stage = 0;
                    ++round;
                }
                if (!ok) {
                    ++i;
                    break;
                }
            }
            ++items;
            it = after;
            have = more;
        }
        cp_wait<0>();
        if (pending >= 0) announce();
        // Before the CTA leaves, every load has landed (all of them have when the products are done).
        if (!ok) {
            for (uint32_t k = i < P::stages ? 0 : i - P::stages; k < i; ++k) mbar_wait(bar.full + 8 * (k % P::stages), (k / P::stages) & 1, kWaitLimitNs);
            for (int x = 0; x < kTiles; ++x)
                if (rows_of[x] > 0) mbar_wait(bar.q + 8 * x, (rows_of[x] - 1) & 1, kWaitLimitNs);
        }
    } else if (warp == kIssuer) {
        // ---- the products: the warp waits together, one lane issues ------------------
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
        bool have = next_active(it);
        int32_t steps = it.steps;
        uint32_t gone = 0, items = 0;                        // steps and items that are done with
        bool ok = true;
        if (have) {
            int32_t ks, kr;
            take(ks, kr);
            ok = __all_sync(0xffffffffu, wait(bar.q, 0) && wait(bar.q + 8, 0) && filled(ks, kr));
            if (ok) {
                tc_fence_after();
                if (elect_one()) {
                    for (int t = 0; t < kTiles; ++t) {
                        issue_s(t, ks);
                        if (steps == 1) tc_commit(bar.q_free + 8 * t);
                    }
                    tc_commit(bar.free + 8 * ks);
                }
                __syncwarp();
            }
        }
        while (have && ok) {
            Item after;
            const bool follows = next_active(after);
            for (int32_t k = 0; ok && k < steps; ++k, ++gone) {
                const bool last = k + 1 == steps, more = !last || follows;
                // whether Q is done with when the next step's S is
                const bool frees = last ? after.steps == 1 : k + 2 == steps;
                int32_t vs, vr, ks = 0, kr = 0;
                take(vs, vr);
                if (more) take(ks, kr);
                // V of this step and K of the next were loaded long ago; P is what is waited for.  A wait
                // that ran out ends the loop at the next vote.
                ok = filled(vs, vr) && (!more || filled(ks, kr));
                // the next item's rows, where the softmax warps bring them, come behind this one's results
                const bool later = last && more && !q_boxes;
                auto next_s = [&](int t) {
                    if (last) ok = wait(bar.q + 8 * t, (items + 1) & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
                    if (elect_one()) {
                        issue_s(t, ks);
                        if (frees) tc_commit(bar.q_free + 8 * t);
                        if (t == kTiles - 1) tc_commit(bar.free + 8 * ks);
                    }
                };
                for (int t = 0; t < kTiles; ++t) {
                    ok = wait(bar.p + 8 * t, gone & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
                    if (elect_one()) {
                        issue_o(t, vs, k > 0);
                        if (last) tc_commit(bar.o + 8 * t);
                        if (t == kTiles - 1) tc_commit(bar.free + 8 * vs);
                    }
                    if (more && !later) next_s(t);
                }
                if (later)
                    for (int t = 0; t < kTiles; ++t) next_s(t);
                ok = __all_sync(0xffffffffu, ok);
            }
            ++items;
            steps = after.steps;
            have = follows;
        }
        if (!ok && elect_one()) {
            // what was issued is done before the CTA leaves
            tc_commit(bar.done);
            mbar_wait(bar.done, 0, kWaitLimitNs);
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
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;          // lane 32 (warp % 4) of tensor memory
        const uint32_t s_own = s_at(tl) + lanes + 64 * half, o_own = o_at(tl) + lanes + DP / 2 * half;
        const int32_t heads = st.kv_heads * st.group;
        uint32_t gone = 0, items = 0;
        bool ok = true;
        // Of the item at hand: this thread's row -- whether there is one, what it sees, where its results go
        // (of rows of all tensors: its first element in `out`, its entry of lse) -- and the steps.
        Span see{};
        char* row_at = nullptr;
        int64_t lse_at = 0;
        int32_t steps = 0;
        bool live = false;
        auto take = [&]() {
            Item it;
            if (!next_item(it)) return false;
            steps = it.steps;
            if (!q_boxes && steps > 0) {
                if (items > 0) ok = ok && __all_sync(0xffffffffu, wait(bar.q_free + 8 * tl, (items - 1) & 1));
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
            int32_t g;
            const int32_t tok = token_of(st, it.row0 + tl * per + t, g);
            live = t < per && tl * per + t < it.rows;
            // a tile's rows without a token see everything, so that their warp need not mask for them
            see = Span{0, INT32_MAX};
            row_at = nullptr;
            if (live) {
                see = in_places(it.held, seen_by(it.q, tok, tok, j.causal, j.window));
                row_at = j.out.base + 2 * ((int64_t)(it.q.q0 + tok) * j.out.row + (int64_t)(it.h * st.group + g) * j.out.head);
                lse_at = (int64_t)(it.q.q0 + tok) * heads + it.h * st.group + g;
            }
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
                const uint64_t seen = below(see.hi) & (~below(see.lo) | below(j.sinks));
                const uint32_t bits[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
                // of either 32: whether some of the warp's rows do not see all of them, and whether some see any
                bool edge[2], some[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    edge[b] = __any_sync(0xffffffffu, bits[b] != ~0u);
                    some[b] = __any_sync(0xffffffffu, live && bits[b]);
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
                    auto up_to = [](int32_t x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1; };
                    const uint32_t first = up_to(see.hi) & (~up_to(see.lo) | up_to(j.sinks));
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
                bool exact = __any_sync(0xffffffffu, live && m == kNone && see.lo < (k + 1) * kN && see.hi > k * kN);
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
                    const bool again = bar_or(pair, 64, !exact && live && (HALF ? fmaxf(a0, a1) : a0 + a1) > kMost);
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
            if (live && ok && half == 0 && j.lse) j.lse[lse_at] = l == 0.0f ? kNone : ((m == kNone ? kNone : m * c - top_at) + log2f(l)) * 0.69314718055994531f;
            const bool some_o = steps > 0;
            char* to = ok ? row_at : nullptr;
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
                    const int row = 8 * i + (lane >> 2);
                    char* dst = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, (unsigned long long)to, row));
                    if (dst && d < st.head_dim) *reinterpret_cast<uint4*>(dst + 2 * d) = ld_shared16(stage + row * 64 + (((lane & 3) ^ (row >> 1 & 3)) << 4));
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
    auto* k = kvs_attend_held_kernel<HALF, DP>;
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, P::bytes);
    if (e != cudaSuccess) return e;
    CUtensorMap km{}, vm{}, qm{};
    const bool boxes = plane_map(&km, j.step, j.k_plane, HALF) && plane_map(&vm, j.step, j.v_plane, HALF), q_boxes = rows_map(&qm, j.step, j.q, HALF);
    const int64_t total = held_items(j.step), tiles = total / ((int64_t)j.step.kv_heads * j.step.requests);
    k<<<(unsigned)(total < sms ? total : sms), P::threads, P::bytes, s>>>(j, km, vm, qm, (int32_t)boxes, (int32_t)q_boxes, make_fastdiv((uint32_t)tiles),
                                                                             make_fastdiv((uint32_t)j.step.kv_heads), (uint32_t)total);
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
