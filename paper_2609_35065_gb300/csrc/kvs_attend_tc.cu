// kvs_attend_tc.cu -- attention of many packed rows: the products on the tensor cores.
//
// A CTA holds up to 256 packed rows (row = token * group + head) of one KV head as two tiles of
// whole tokens (or one, where a request has no more) and goes over the keys 128 at a time:
//
//     S = Q K^T  (tensor memory)  ->  P = 2^(c S - c m)  (registers, back over S)  ->  O += P V
//
// While one tile's softmax runs, the tensor cores work on the other's.  Two warpgroups do a
// tile's softmax, half of a row's 64 + 64 keys to a thread: a step's softmax has to be done
// within the other tile's two products, which one warp to a scheduler cannot do.  Of the fifth
// warpgroup three warps load K and V through a ring of 32 KiB tiles -- TMA boxes of whole
// blocks where the block size allows, cp.async row by row otherwise and for the tiles that
// hold the ends of what may be read (there, rows outside become zeros) -- and one issues the
// products.
//
// The running maximum m that O and the sums refer to is raised only when weights outgrow it by
// 2^20: until then P is up to that instead of 1, which costs the relative precision of P and of
// binary32 sums nothing, and O need not be rescaled, which hardly any step then does (at 2^8
// every third step of a long cache had a row that did).  Half holds multiples of 2^-24 up to 2^16
// only: P is 2^3 to 2^10 at the maximum there, by the number of keys, so that the light ones of
// many are not lost, and may outgrow it up to 2^16.
//
// P is rounded to the 16-bit type of V, as the products take both operands of one such type:
// what that takes would need a second product with V, half again of all of them (relative error
// of the outputs 0.0023, with weights of 32 bits 0.0017).
//
// So a step takes its exponentials against the m at hand and sees by their sum that none was
// too large; the rare step that had such a one is done again with m raised.
//
// 16 suffixes of 2048 tokens behind 2048, 32 query heads of 128 dims on 8 (1.65 TFLOP) take
// 1075 to 1117 us, 1.48 to 1.53 PFLOP/s, at the GPU's power cap (1.36 kW, where its clock falls
// from 2070 to 1860 MHz).  A question of 293 tokens about 12288, 40 query heads on 8, takes 62 to
// 64 (75 GFLOP in 144 CTAs of 33 steps; some 53 of it are this kernel, whose products keep the
// tensor cores busy for 62%; of the rest a CTA's start was measured at 1.6 us, what the other 18
// wait for was not; 9 are the binary32 parts and their join).  35 rows over 4000 to 10000 tokens
// for each of 8 requests and 2 heads take 18.4: with one tile nothing runs beside the softmax, S of
// the next step being issued behind the product that reads P from the same columns, so that
// S, softmax, P and O are one chain of about 1 us a step.
//
// Products run in the order in which one thread issues them, which the reuse of S's columns
// for P relies on: S of the next tile is issued behind the product that reads P.
#include "kvs_tcgen05.cuh"

namespace kvs {
namespace {

constexpr int kM = 128, kN = 128;                  // rows of a tile, keys of a step
constexpr int kLoaders = 3;
constexpr float kNone = -INFINITY;

template <int DP, int TILES>
struct Plan {
    static constexpr int threads = 256 * TILES + 128;
    static constexpr int tile = kN * DP * 2;       // bytes of a tile of Q, K or V
    static constexpr int stages = DP == 128 ? 5 : TILES == 2 ? 8 : 5;
    static constexpr int ctas = DP == 64 && TILES == 1 ? 2 : 1;       // to an SM
    static constexpr int columns = 256 * TILES;    // of tensor memory: S of each tile, then O
    static constexpr int bars = (TILES + stages) * tile;
    static constexpr int tops = bars + 256;        // [2][TILES][128] binary32: maxima, sums that a row's threads exchange
    static constexpr int bytes = tops + 1024 * TILES;
    // for a cluster's join, in the ring: [tile's row][DP] binary32 and [tile's row] (m, l)
    static constexpr int part = TILES * tile, part_ml = part + TILES * 128 * DP * 4;
    static_assert(part_ml + TILES * 1024 <= bars, "the ring holds a CTA's part");
};

struct Bars {
    uint32_t q, full, free, s, p, o;
    __device__ Bars(uint32_t at, int stages) : q(at), full(at + 8), free(full + 8 * stages), s(free + 8 * stages), p(s + 16), o(p + 16) {}
};

// HELD: a window with sinks; the steps go over its places, units of which are boxes' tokens.
template <bool HALF, int DP, int TILES, bool HELD>
__global__ void __launch_bounds__(Plan<DP, TILES>::threads, Plan<DP, TILES>::ctas) kvs_attend_tc_kernel(AttendJob j, const __grid_constant__ CUtensorMap k_map,
                                                                    const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map,
                                                                    int32_t boxes, int32_t q_boxes) {
    extern __shared__ __align__(1024) char raw[];
    using N = Num<HALF>;
    using P = Plan<DP, TILES>;
    constexpr int kIssuer = 8 * TILES;               // the issuing warp, behind the softmax's; then the loading ones
    constexpr float kMost = HALF ? 65504.0f : 1048576.0f;            // of a thread's weights of a step (half: of either sum)
    if (HELD) grid_wait();                           // HELD: launched behind the kernel before
    const StepView& st = j.step;
    const bool cluster = (TILES == 1 || HELD) && j.cluster;      // parts of two tiles: only of places
    const uint32_t base = smem_u32(raw);
    if (base & 1023) {                               // the swizzle needs it; there is no room to round it up
        record_error(st.err, KVS_ERR_UNSUPPORTED);
        return;
    }
    const uint32_t ring = base + TILES * P::tile, ctl = base + P::bars;
    const Bars bar(ctl, P::stages);
    const uint32_t tmem_at = bar.o + 8;
    const int warp = warp_number(), wg = warp >> 2, lane = threadIdx.x & 31;

    const int32_t tiles = gridDim.x / j.splits, split = blockIdx.x % j.splits;
    const int32_t r = blockIdx.z, h = blockIdx.y;
    const int32_t per = tile_rows_of(st.group);
    // The last rows see the most keys: they come first, so that no long CTA starts last.
    const int32_t row0 = (tiles - 1 - (int32_t)(blockIdx.x / j.splits)) * TILES * per;
    // Set-up while the request's lengths are on their way.
    const RawRequest fetched = fetch_request<HELD>(st, r);
    if (warp == kIssuer) tmem_alloc(tmem_at, P::columns);
    if (threadIdx.x == 0) {
        mbar_init(bar.q, q_boxes ? 1 : 256 * TILES);
        for (int i = 0; i < P::stages; ++i) {
            mbar_init(bar.full + 8 * i, kLoaders);
            mbar_init(bar.free + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar.s + 8 * i, 1);
            mbar_init(bar.p + 8 * i, 8);
        }
        mbar_init(bar.o, 1);
        mbar_init_fence();
    }
    if (warp == kIssuer + 1 && lane == 0) {
        if (boxes) {
            prefetch_map(&k_map);
            prefetch_map(&v_map);
        }
        if (q_boxes) prefetch_map(&q_map);
    }
    const Request q = check_request(st, fetched);
    const int32_t rows = min(TILES * per, q.n * st.group - row0);
    if (rows <= 0) {
        if (warp == kIssuer) {
            __syncwarp();
            uint32_t at;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(at) : "r"(tmem_at) : "memory");
            tmem_dealloc(at, P::columns);
        }
        return;
    }
    Span all = seen_by(q, row0 / st.group, (row0 + rows - 1) / st.group, j.causal, j.window);
    Held held{};
    int32_t T = q.T;                                 // places (without HELD: tokens) of the cache
    if (HELD) {
        held = held_of(all.lo, j.sinks, boxes ? min(st.block_size, kN) : 1);
        T -= held.shift;
        all = in_places(held, all);
    }
    const int32_t first = HELD ? 0 : all.lo / kN, steps_all = all.hi > all.lo ? (all.hi + kN - 1) / kN - first : 0;
    const int32_t j0 = first + (int32_t)((int64_t)steps_all * split / j.splits);
    const int32_t steps = first + (int32_t)((int64_t)steps_all * (split + 1) / j.splits) - j0;
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;
    // K's and V's tiles of a step are in the same blocks; the loading warps look the next step's up a step ahead
    Box next{};
    if (boxes && steps > 0 && warp > kIssuer) next = box_of<DP, kLoaders, HELD>(st, table, held, j0 * kN, T, warp - kIssuer - 1, lane);

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_at) : "memory");
    auto s_at = [&](int t) { return tmem + 128u * t; };
    auto o_at = [&](int t) { return tmem + 128u * TILES + (uint32_t)DP * t; };

    // A wait that does not end is recorded; every role then leaves its loop (the others' waits end too).
    auto wait = [&](uint32_t b, uint32_t parity) {
        if (mbar_wait(b, parity, kWaitLimitNs)) return true;
        record_error(st.err, KVS_ERR_TIMEOUT);
        return false;
    };

    if (warp > kIssuer) {
        // ---- K and V: tile i is K (even) or V (odd) of step i / 2 ------------------
        const int t = threadIdx.x - 32 * (kIssuer + 1), w = warp - kIssuer - 1;
        int pending = -1;                                    // cp.async tile not yet announced
        auto announce = [&]() {
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.full + 8 * pending);
            pending = -1;
        };
        int32_t i = 0;
        Box box{};
        for (; i < 2 * steps; ++i) {
            const int stage = i % P::stages;
            if (boxes && !(i & 1)) {
                box = next;
                if (i + 2 < 2 * steps) next = box_of<DP, kLoaders, HELD>(st, table, held, (j0 + (i >> 1) + 1) * kN, T, w, lane);
            }
            if (i >= P::stages) {
                const bool ok = lane != 0 || wait(bar.free + 8 * stage, (i / P::stages - 1) & 1);
                if (!__all_sync(0xffffffffu, ok)) break;
            }
            const uint32_t dst = ring + stage * P::tile;
            const int32_t t0 = (j0 + (i >> 1)) * kN;
            const bool is_v = i & 1;
            // Beyond the cache, and before what the rows see, V has to be zeros; K may be anything there.
            const bool whole = (t0 >= all.lo || (HELD && min(t0 + kN, all.lo) <= j.sinks)) && t0 + kN <= T;
            if (boxes && (whole || !is_v)) {
                if (pending >= 0) {
                    cp_wait<0>();
                    announce();
                }
                tile_boxes<DP>(dst, is_v ? &v_map : &k_map, st, h, box, bar.full + 8 * stage, lane);
            } else {
                tile_rows<DP, 32 * kLoaders, HELD>(dst, is_v ? j.v_plane : j.k_plane, st, table, h, held, t0, all.lo, T, HELD ? j.sinks : 0, t);
                cp_commit();
                if (pending >= 0) {
                    cp_wait<1>();
                    announce();
                }
                pending = stage;
            }
        }
        cp_wait<0>();
        if (pending >= 0) announce();
        // Before the CTA leaves, every load has landed (all of them have when the products are done).
        if (i < 2 * steps)
            for (int k = i - P::stages < 0 ? 0 : i - P::stages; k < i; ++k)
                mbar_wait(bar.full + 8 * (k % P::stages), (k / P::stages) & 1, kWaitLimitNs);
    } else if (warp == kIssuer) {
        if (steps > 0) {
            // ---- the products: the warp waits together, one lane issues ------------------
            // a negative scale's sign goes into the products, so that maxima of S are those of the scores
            const uint32_t id_s = tc_idesc(HALF, kN, false) | (j.scale_log2 < 0.0f ? kNegA : 0u);
            constexpr uint32_t id_o = tc_idesc(HALF, DP, true);
            if (q_boxes && elect_one()) {
                mbar_expect_tx(bar.q, (uint32_t)per * DP * 2 * TILES);
#pragma unroll
                for (int k = 0; k < TILES * (DP / 64); ++k) {
                    const int t = k / (DP / 64), c = k % (DP / 64);
                    tma_load_3d(base + t * P::tile + c * kM * 128, &q_map, 64 * c, h * st.group, q.q0 + (row0 + t * per) / st.group, bar.q);
                }
            }
            __syncwarp();
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
                    tc_mma_ts(tm + 128 * TILES + DP * t, tm + 128 * t + 8 * k, tc_ahead(b, k * 2048), id_o, add || k > 0);
            };
            auto filled = [&](int32_t stage, int32_t round) { return wait(bar.full + 8 * stage, round & 1); };
            bool ok = __all_sync(0xffffffffu, wait(bar.q, 0) && filled(0, 0));
            if (ok) {
                tc_fence_after();
                if (elect_one()) {
                    issue_s(0, 0);
                    if (TILES == 2) issue_s(1, 0);
                    tc_commit(bar.free);
                }
                __syncwarp();
            }
            int32_t stage = 1, round = 0;                    // of the next tile of the ring
            for (int32_t k = 0; ok && k < steps; ++k) {
                const bool more = k + 1 < steps;
                const int32_t vs = stage, vr = round;
                if (++stage == P::stages) {
                    stage = 0;
                    ++round;
                }
                const int32_t ks = stage, kr = round;
                if (more && ++stage == P::stages) {
                    stage = 0;
                    ++round;
                }
                // V of this step and K of the next were loaded long ago; P is what is waited for.  A wait
                // that ran out ends the loop at the next vote.
                ok = filled(vs, vr) && (!more || filled(ks, kr));
                ok = wait(bar.p, k & 1) && ok;
                __syncwarp();
                tc_fence_after();
                if (elect_one()) {
                    issue_o(0, vs, k > 0);
                    if (TILES == 1) tc_commit(bar.free + 8 * vs);
                    if (more) issue_s(0, ks);
                    if (TILES == 1 && more) tc_commit(bar.free + 8 * ks);
                }
                if (TILES == 2) {
                    ok = wait(bar.p + 8, k & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
                    if (elect_one()) {
                        issue_o(1, vs, k > 0);
                        tc_commit(bar.free + 8 * vs);
                        if (more) {
                            issue_s(1, ks);
                            tc_commit(bar.free + 8 * ks);
                        }
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
            }
            if (elect_one()) {
                tc_commit(bar.o);
                if (!ok) {
                    mbar_wait(bar.q, 0, kWaitLimitNs);
                    mbar_wait(bar.o, 0, kWaitLimitNs);
                }
            }
        }
        __syncwarp();
    } else {
        // ---- softmax of tile tl: row t, keys 64 half ... of a step -----------------------
        const int tl = wg >> 1, half = wg & 1, t = threadIdx.x & 127;
        const uint32_t own = base + tl * P::tile;                    // the tile's Q, and at the end its results
        if (!q_boxes && steps > 0) {
            constexpr int CH = DP / 8;
#pragma unroll 4
            for (int v = threadIdx.x & 255; v < kM * CH; v += 256) {
                const int i = v / CH, c = v % CH;
                const bool there = i < per && tl * per + i < rows && 8 * c < st.head_dim;
                int32_t g;
                const int32_t tok = token_of(st, there ? row0 + tl * per + i : 0, g);
                cp_async16(own + (c >> 3) * kM * 128 + i * 128 + (((c & 7) ^ (i & 7)) << 4),
                           j.q.base + (there ? 2 * ((int64_t)(q.q0 + tok) * j.q.row + (int64_t)(h * st.group + g) * j.q.head + 8 * c) : 0), there);
            }
            cp_commit();
            cp_wait<0>();
            fence_async_smem();
            mbar_arrive(bar.q);
        }
        // The warps of a row's two halves agree, and wait for one another, under a barrier of their
        // own.  After a wait that ran out, both still go through all steps (on whatever is there).
        const int pair = 1 + tl * 4 + (warp & 3);
        float* tops = reinterpret_cast<float*>(raw + P::tops);
        const float c = fmaxf(fabsf(j.scale_log2), 1e-36f);         // a zero scale keeps -infinity * c what it is
        const float c_low = j.scale_log2 < 0.0f ? -j.scale_low : j.scale_low;
        int32_t g;
        const int32_t tok = token_of(st, row0 + tl * per + t, g);
        const bool live = t < per && tl * per + t < rows;
        // a tile's rows without a token see everything, so that their warp need not mask for them
        Span see{0, INT32_MAX};
        if (live) {
            see = seen_by(q, tok, tok, j.causal, j.window);
            if (HELD) see = in_places(held, see);
        }
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;          // lane 32 (warp % 4) of tensor memory
        const uint32_t s_own = s_at(tl) + lanes + 64 * half, o_own = o_at(tl) + lanes + DP / 2 * half;
        // log2 of a weight at the reference: at 3 half's time over 4096 and 12581 tokens is that at 0, at 8 it is 8 and 12% more
        const float top_at = HALF ? half_top(steps * kN, 3) : 0.0f;
        float m = kNone, l0 = 0.0f, l1 = 0.0f;
        bool ok = true;
        for (int32_t k = 0; k < steps; ++k) {
            ok = ok && __all_sync(0xffffffffu, wait(bar.s + 8 * tl, k & 1));
            tc_fence_after();
            const int32_t t0 = (j0 + k) * kN + 64 * half;
            const int32_t lo = see.lo - t0, hi = see.hi - t0, sinks = HELD ? j.sinks - t0 : 0;
            const bool edge = __any_sync(0xffffffffu, lo > 0 || hi < 64);
            auto masked = [&](float* s, int b) {
#pragma unroll
                for (int n = 0; n < 32; ++n) s[n] = (32 * b + n >= lo || (HELD && 32 * b + n < sinks)) && 32 * b + n < hi ? s[n] : kNone;
            };
            // Against this step's own maximum: the first step, and the first that rows see any key of.
            bool exact = k == 0 || __any_sync(0xffffffffu, live && m == kNone && (see.lo < (j0 + k + 1) * kN || (HELD && j.sinks > (j0 + k) * kN)) && see.hi > (j0 + k) * kN);
            uint32_t pk[32];
            float a0, a1;
            while (true) {
                if (exact) {
                    float top = kNone;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint32_t sr[32];
                        tmem_ld32(sr, s_own + 32 * b);
                        tmem_wait_ld();
                        tmem_loaded32(sr);
                        float* s = reinterpret_cast<float*>(sr);
                        if (edge) masked(s, b);
#pragma unroll
                        for (int n = 0; n < 32; n += 2) top = max3(top, s[n], s[n + 1]);
                    }
                    tops[half * 128 * TILES + tl * 128 + t] = top;
                    bar_some(pair, 64);
                    top = fmaxf(top, tops[(half ^ 1) * 128 * TILES + tl * 128 + t]);
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
                    uint32_t sr[32];
                    tmem_ld32(sr, s_own + 32 * b);
                    tmem_wait_ld();
                    tmem_loaded32(sr);
                    float* s = reinterpret_cast<float*>(sr);
                    if (edge) masked(s, b);
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
        if (steps > 0 && ok) ok = __all_sync(0xffffffffu, wait(bar.o, 0));
        tc_fence_after();
        float l = l0 + l1;
        tops[half * 128 * TILES + tl * 128 + t] = l;
        bar_some(pair, 64);
        l = tops[tl * 128 + t] + tops[128 * TILES + tl * 128 + t];
        const int32_t heads = st.kv_heads * st.group;
        const int64_t all_rows = (int64_t)st.total_q * heads;
        if (ok) {
            if (live && half == 0) {
                const float m2 = m == kNone ? kNone : HELD ? fmaf(m, c_low, m * c - top_at) : m * c - top_at;
                const int64_t row = (int64_t)(q.q0 + tok) * heads + h * st.group + g;
                if (cluster) reinterpret_cast<float2*>(raw + P::part_ml)[128 * tl + t] = make_float2(m2, l);
                else if (j.splits > 1) reinterpret_cast<float2*>(j.partial + (int64_t)j.splits * all_rows * st.head_dim)[split * all_rows + row] = make_float2(m2, l);
                else if (j.lse) j.lse[row] = l == 0.0f ? kNone : (m2 + log2f(l)) * 0.69314718055994531f;
            }
            // Through shared memory (32 rows of DP bytes to a warp, in Q's place), so that a row's
            // bytes leave in one piece: 16-bit results at once, binary32 parts in two passes.
            const bool parts = j.splits > 1;
            if (cluster) {
                // binary32 rows over the ring, which nothing needs any more, for the cluster's CTAs to read
                const uint32_t at = base + P::part + (128 * tl + t) * DP * 4;
#pragma unroll
                for (int b = 0; b < DP / 32; ++b) {
                    uint32_t o[16];
                    if (steps > 0) {
                        tmem_ld16(o, o_own + 16 * b);
                        tmem_wait_ld();
                        tmem_loaded16(o);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int v = DP / 8 * half + 4 * b + e;
                        const bool some = steps > 0 && l != 0.0f;
                        st_shared16(at + ((v ^ (t & 7)) << 4), some ? o[4 * e] : 0u, some ? o[4 * e + 1] : 0u, some ? o[4 * e + 2] : 0u, some ? o[4 * e + 3] : 0u);
                    }
                }
            }
            const float f = parts ? 1.0f : (l > 0.0f ? 1.0f / l : l);
            const uint32_t stage = own + half * (P::tile / 2) + (warp & 3) * (P::tile / 8);
            constexpr int VR = DP / 16;                                                  // 16-byte vectors of a staged row
            const int vec0 = parts ? DP / 8 * half : VR * half;                          // of the whole row, where this half's begin
            const int vecs = (parts ? st.head_dim * 4 : st.head_dim * 2) / 16;
            // where this thread's row goes; the row's writers get it from here
            char* row_at = nullptr;
            if (live) {
                if (parts) row_at = reinterpret_cast<char*>(j.partial + (split * all_rows + (int64_t)(q.q0 + tok) * heads + h * st.group + g) * st.head_dim);
                else row_at = j.out.base + 2 * ((int64_t)(q.q0 + tok) * j.out.row + (int64_t)(h * st.group + g) * j.out.head);
            }
            for (int pass = 0; pass < (cluster ? 0 : parts ? 2 : 1); ++pass) {
#pragma unroll
                for (int b = 0; b < DP / 32; ++b) {
                    // 16 columns: two vectors of 16-bit numbers, or four of binary32
                    if (parts && b / (DP / 64) != pass) continue;
                    uint32_t o[16];
                    if (steps > 0) {
                        tmem_ld16(o, o_own + 16 * b);
                        tmem_wait_ld();
                        tmem_loaded16(o);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = steps > 0 && l != 0.0f ? __float_as_uint(__uint_as_float(o[e]) * f) : 0u;
                    if (parts) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int v = 4 * (b % (DP / 64)) + e;
                            st_shared16(stage + lane * VR * 16 + ((v ^ (lane & (VR - 1))) << 4), o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t w[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) w[x] = N::pack(__uint_as_float(o[8 * e + 2 * x]), __uint_as_float(o[8 * e + 2 * x + 1]));
                            st_shared16(stage + lane * VR * 16 + (((2 * b + e) ^ (lane & (VR - 1))) << 4), w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < VR; ++i) {
                    const int row = i * (32 / VR) + lane / VR, v = lane % VR, vec = vec0 + pass * VR + v;
                    char* dst = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, (unsigned long long)row_at, row));
                    if (dst && vec < vecs) *reinterpret_cast<uint4*>(dst + 16 * vec) = ld_shared16(stage + row * VR * 16 + ((v ^ (row & (VR - 1))) << 4));
                }
                __syncwarp();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssuer) tmem_dealloc(tmem, P::columns);
    if (!cluster) return;
    // The cluster's CTAs share out the rows, four dims to a thread, and read one another's parts in order.
    constexpr int kParts = TILES == 1 ? kCluster : kClusterPairs;
    cluster_sync();
    const int32_t share = (rows + j.splits - 1) / j.splits, row_end = min(rows, (split + 1) * share);
    for (int32_t v = threadIdx.x; v < share * (DP / 4); v += P::threads) {
        const int32_t x = split * share + v / (DP / 4), d = v % (DP / 4);
        if (x >= row_end || 4 * d >= st.head_dim) continue;
        const int32_t at = x + (x < per ? 0 : 128 - per);        // among the rows of tiles
        float2 ml[kParts];
        float4 p[kParts];
        float M = kNone, L = 0.0f;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            ml[k] = make_float2(kNone, 0.0f);
            p[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (k < j.splits) {
                ml[k] = cluster_ld2(cluster_at(base + P::part_ml + 8 * at, k));
                p[k] = cluster_ld4(cluster_at(base + P::part + at * DP * 4 + ((d ^ (at & 7)) << 4), k));
            }
            M = fmaxf(M, ml[k].x);
        }
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const float f = ml[k].y == 0.0f ? 0.0f : exp2_fast(ml[k].x - M);
            L += f * ml[k].y;
            o.x += f * p[k].x;
            o.y += f * p[k].y;
            o.z += f * p[k].z;
            o.w += f * p[k].w;
        }
        int32_t g;
        const int32_t tok = q.q0 + token_of(st, row0 + x, g), head = h * st.group + g;
        const float inv = L > 0.0f ? 1.0f / L : L;
        *reinterpret_cast<uint2*>(j.out.base + 2 * ((int64_t)tok * j.out.row + (int64_t)head * j.out.head + 4 * d)) =
            make_uint2(N::pack(o.x * inv, o.y * inv), N::pack(o.z * inv, o.w * inv));
        if (d == 0 && j.lse) j.lse[(int64_t)tok * (st.kv_heads * st.group) + head] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
    }
    // no CTA leaves while another may read its parts
    cluster_sync();
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
    static const EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        cudaGetLastError();
        return (EncodeFn)f;
    }();
    return fn;
}

}  // namespace

bool plane_map(void* map, const StepView& st, const void* plane, bool half) {
    const int B = st.block_size;
    if (B % 8 || (128 % B && B % 128) || st.head_dim < 64 || !encoder()) return false;
    const cuuint64_t d = st.head_dim, h = st.kv_heads;
    const cuuint64_t dims[4] = {d, h, (cuuint64_t)B, (cuuint64_t)st.num_blocks};
    const cuuint64_t strides[3] = {d * 2, d * h * 2, d * h * 2 * B};
    if (strides[2] >= 1ull << 40) return false;
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)(B < 128 ? B : 128), 1}, one[4] = {1, 1, 1, 1};
    return encoder()((CUtensorMap*)map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(plane), dims, strides, box,
                     one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool rows_map(void* map, const StepView& st, const RowsView& rows, bool half) {
    if (st.group > 128 || st.head_dim < 64 || !encoder()) return false;
    const int heads = st.kv_heads * st.group;
    const cuuint64_t d = st.head_dim;
    const cuuint64_t dims[3] = {d, (cuuint64_t)heads, (cuuint64_t)st.total_q};
    // a dimension of one entry has no stride of its own
    const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)rows.head * 2 : d * 2, st.total_q > 1 ? (cuuint64_t)rows.row * 2 : d * 2 * heads};
    if (!strides[0] || !strides[1] || strides[0] >= 1ull << 40 || strides[1] >= 1ull << 40) return false;
    const cuuint32_t box[3] = {64, (cuuint32_t)st.group, (cuuint32_t)(128 / st.group)}, one[3] = {1, 1, 1};
    return encoder()((CUtensorMap*)map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, rows.base, dims, strides, box,
                     one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <bool HALF, int DP, int TILES, bool HELD>
cudaError_t attend_tc(const AttendJob& j, cudaStream_t s) {
    using P = Plan<DP, TILES>;
    auto* k = kvs_attend_tc_kernel<HALF, DP, TILES, HELD>;
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, P::bytes);
    if (e != cudaSuccess) return e;
    CUtensorMap km{}, vm{}, qm{};
    const bool boxes = plane_map(&km, j.step, j.k_plane, HALF) && plane_map(&vm, j.step, j.v_plane, HALF), q_boxes = rows_map(&qm, j.step, j.q, HALF);
    const int64_t rows = TILES * tile_rows_of(j.step.group), tiles = ((int64_t)j.step.max_q * j.step.group + rows - 1) / rows;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * j.splits), j.step.kv_heads, j.step.requests);
    cfg.blockDim = dim3(P::threads);
    cfg.dynamicSmemBytes = P::bytes;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    cfg.attrs = at;
    cfg.numAttrs = launch_attributes(at, j.cluster ? j.splits : 1, HELD);
    return cudaLaunchKernelEx(&cfg, k, j, km, vm, qm, (int32_t)boxes, (int32_t)q_boxes);
}

template <bool HALF, bool HELD>
cudaError_t attend_tiles(const AttendJob& j, cudaStream_t s) {
    if (j.step.head_dim <= 64) return j.row_tiles == 1 ? attend_tc<HALF, 64, 1, HELD>(j, s) : attend_tc<HALF, 64, 2, HELD>(j, s);
    return j.row_tiles == 1 ? attend_tc<HALF, 128, 1, HELD>(j, s) : attend_tc<HALF, 128, 2, HELD>(j, s);
}
template <bool HALF>
cudaError_t attend_tiles(const AttendJob& j, cudaStream_t s) { return j.held ? attend_tiles<HALF, true>(j, s) : attend_tiles<HALF, false>(j, s); }

}  // namespace

cudaError_t launch_attend_tc(const AttendJob& j, bool half, cudaStream_t s) { return half ? attend_tiles<true>(j, s) : attend_tiles<false>(j, s); }

}  // namespace kvs
