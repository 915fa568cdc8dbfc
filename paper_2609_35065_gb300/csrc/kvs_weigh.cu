// kvs_weigh.cu -- accumulated attention weight of the cached tokens.
//
//     w_t = decay * w_t + sum over rows of 2^(c q . k_t - lse'),  c = scale log2(e), lse' = lse log2(e)
//
// The exponent is one binary32 number, whose rounding a weight shows: 8e-7 of it where 12288 tokens
// share it, against 2e-7 for a difference taken before it is scaled.
//
// With every row's lse known a key's sum needs no other key: keys go to different CTAs, warps
// or lanes, and no sum is shared.  Rows are packed as in attention (row = token * group + head).
#include "kvs_tcgen05.cuh"

namespace kvs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Packed rows [first, end) that see any of the cached tokens t_lo .. t_hi (all of them do
// between, of one token).  Their number is below 2^30.
struct RowSpan {
    int32_t first, end;
};
__device__ __forceinline__ RowSpan rows_seeing(const StepView& st, const Request& q, int32_t t_lo, int32_t t_hi, int32_t causal, int32_t window) {
    const int64_t base = q.T - q.n;                              // position of new token 0
    int64_t first = 0, end = q.n;
    if (causal) first = min(end, max((int64_t)0, t_lo - base));
    if (window > 0) end = min(end, t_hi + window - base);
    return RowSpan{(int32_t)first * st.group, (int32_t)max(first, end) * st.group};
}

__device__ __forceinline__ void add_weight(const WeighJob& j, int32_t r, int32_t h, int32_t t, float sum) {
    float* w = j.weights + r * j.request_stride + h * j.head_stride + t;
    *w = j.decay == 0.0f ? sum : j.decay * *w + sum;
}

// ---------------------------------------------------------------------------
// Many rows: S^T = K Q^T on the tensor cores, one or two tiles of 128 keys (the accumulators'
// lanes) per CTA and the rows in tiles of at most 128 (their columns), so that a thread sums its
// key's weights in registers.  The keys stay in tensor memory: read from shared memory for every
// product they took as much of its 128 bytes a cycle as the rows, and both together all of it.
// Two warpgroups share a key tile, half of each row tile's columns to each; in the last
// warpgroup one warp issues the products, one loads the next row tiles (TMA boxes of whole
// tokens; cp.async by three warps where the rows have no such boxes) and two their lse, in a
// ring of its own: a tile's rows are done with when the products are, its lse with the sums.
//
// Two CTAs of one key tile share an SM, and while one starts or ends the other works; of many row
// tiles, two key tiles read each of them once for both.
//
// 128 x 128 scores take the tensor cores about 570 cycles and the exponentials 512; what bounds
// it is their hand-over, some 850 cycles: 5120 rows against 13312 keys of 8 heads of 128 dims
// (134 GFLOP) in 120.5 us, 1.12 PFLOP/s.  With a quarter of the exponentials it takes 115, with
// half the products 118, without lse 118.  Slower were: a key of both tiles to a thread, so that
// lse is read once (128); loads of the scores ahead of their use (122); three sets of warps
// with an accumulator each (128).
//
// Where there are fewer key tiles than SMs, a cluster of CTAs shares a key tile's row tiles
// and joins its sums, in the CTAs' order, through distributed shared memory.
// ---------------------------------------------------------------------------
constexpr int kSlots = 8;

// KT: key tiles of a CTA.
template <int DP, int KT>
struct WPlan {
    static constexpr int issuer = 8 * KT;                        // the issuing warp, behind the sums'; then the loading ones
    static constexpr int threads = 32 * (issuer + 4), keys = 128 * KT;
    static constexpr int stages = KT == 2 ? 4 : 2, accs = KT == 2 ? 3 : 1, columns = 256 * KT;
    static constexpr int tile = 128 * DP * 2;
    static constexpr int lse = tile * (KT + stages);             // [kSlots][128] binary32, times -log2(e)
    static constexpr int sums = lse + kSlots * 512;              // [KT][2][128]
    static constexpr int bars = sums + 1024 * KT;
    static constexpr int bytes = bars + 512 + 1024;
};

template <bool HALF, int DP, int KT>
__global__ void __launch_bounds__(WPlan<DP, KT>::threads, 3 - KT) kvs_weigh_tc_kernel(WeighJob j, const __grid_constant__ CUtensorMap k_map,
                                                                   const __grid_constant__ CUtensorMap q_map, int32_t k_boxes, int32_t q_boxes, int32_t share) {
    extern __shared__ char raw[];
    using P = WPlan<DP, KT>;
    constexpr int kThreads = P::threads, kStages = P::stages, kAccs = P::accs, kKeysTc = P::keys, kIssuer = P::issuer;
    const StepView& st = j.step;
    const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
    char* mem = raw + (base - smem_u32(raw));
    const uint32_t ring = base + KT * P::tile, ctl = base + P::bars;
    const uint32_t b_k = ctl, b_full = ctl + 8, b_free = b_full + 8 * kStages, b_s = b_free + 8 * kStages, b_e = b_s + 8 * kAccs, b_done = b_e + 8 * kAccs,
                   b_load = b_done + 8, b_lse = b_load + 8, b_read = b_lse + 8 * kSlots, tmem_at = b_read + 8 * kSlots;
    const int warp = warp_number(), lane = threadIdx.x & 31, wg = warp >> 2;
    const int32_t r = blockIdx.z, h = blockIdx.y, rank = blockIdx.x % share, t0 = (blockIdx.x / share) * kKeysTc;
    const Request q = load_request(st, r);
    if (t0 >= q.T) return;                                       // the whole cluster
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;
    const int32_t per = tile_rows_of(st.group);                  // rows of a tile
    const int32_t key_tiles = KT == 2 && t0 + 128 < q.T ? 2 : 1;
    const RowSpan any = rows_seeing(st, q, t0, min(t0 + kKeysTc, q.T) - 1, j.causal, j.window);
    const int32_t tile0 = any.first / per, tiles = any.end > any.first ? (any.end + per - 1) / per - tile0 : 0;
    const int32_t mine = (tiles - rank + share - 1) / share;     // row tiles tile0 + rank + share * i
    const int32_t total = q.n * st.group;

    if (threadIdx.x == 0) {
        mbar_init(b_load, 3 * key_tiles);
        mbar_init(b_k, 8 * KT);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(b_full + 8 * i, q_boxes ? 1 : 3);          // the loading warps
            mbar_init(b_free + 8 * i, 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(b_lse + 8 * i, q_boxes ? 2 : 3);
            mbar_init(b_read + 8 * i, 8 * key_tiles);            // the key tiles' warps
        }
        for (int i = 0; i < kAccs; ++i) {
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_e + 8 * i, 8);
        }
        mbar_init(b_done, 1);
        mbar_init_fence();
    }
    if (warp == kIssuer) tmem_alloc(tmem_at, P::columns);
    // rows that no box fills are zeros for good, and weigh nothing
    for (int i = threadIdx.x; i < (128 - per) * (DP / 8) * kStages; i += kThreads) {
        const int stage = i / ((128 - per) * (DP / 8)), v = i % ((128 - per) * (DP / 8)), row = per + v / (DP / 8), c = v % (DP / 8);
        *reinterpret_cast<uint4*>(mem + P::tile * (KT + stage) + (c >> 3) * 128 * 128 + row * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_at) : "memory");
    auto wait = [&](uint32_t b, uint32_t parity) {
        if (mbar_wait(b, parity, kWaitLimitNs)) return true;
        record_error(st.err, KVS_ERR_TIMEOUT);
        return false;
    };

    float sum = 0.0f;
    const int t = threadIdx.x & 127;
    if (warp == kIssuer) {
        // ---- the products: the warp waits together, one lane issues ----------------------
        constexpr uint32_t id = tc_idesc(HALF, 128, false);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), keys = tm + 128 * kAccs;     // 64 columns to a key tile
        const uint64_t q_desc = tc_desc(ring, 16, 1024);
        bool ok = mine <= 0 || __all_sync(0xffffffffu, wait(b_k, 0));
        int32_t stage = 0, round = 0, acc = 0, uses = 0;         // of the next row tile; of the next product
        // A wait that ran out ends the loop at the next vote: what is issued meanwhile works on whatever is there.
        for (int32_t i = 0; ok && i < mine; ++i) {
            ok = wait(b_full + 8 * stage, round & 1);
            const uint64_t b = tc_ahead(q_desc, stage * P::tile);
            for (int32_t kt = 0; kt < key_tiles; ++kt) {
                if (uses > 0) ok = wait(b_e + 8 * acc, (uses - 1) & 1) && ok;
                __syncwarp();
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
                        tc_mma_ts(tm + 128 * acc, keys + 64 * kt + 8 * k, tc_ahead(b, (k >> 2) * 128 * 128 + (k & 3) * 32), id, k > 0);
                    tc_commit(b_s + 8 * acc);
                    if (kt + 1 == key_tiles) tc_commit(b_free + 8 * stage);
                }
                if (++acc == kAccs) {
                    acc = 0;
                    ++uses;
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (++stage == kStages) {
                stage = 0;
                ++round;
            }
        }
        // the last products are waited for by their readers; after a failure, here
        if (!ok && elect_one()) {
            tc_commit(b_done);
            mbar_wait(b_done, 0, kWaitLimitNs);
        }
        __syncwarp();
    } else if (warp > kIssuer) {
        // ---- loads: one warp the rows, two their lse; by rows all three both ------
        const int u = threadIdx.x - (kIssuer + 1) * 32;                     // 0 to 95
        uint32_t pending = 0;
        auto announce = [&]() {
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(pending);
            pending = 0;
        };
        if (mine > 0) {
            for (int32_t kt = 0; kt < key_tiles; ++kt) {
                if (k_boxes) tile_boxes<DP>(base + kt * P::tile, &k_map, st, h, box_of<DP, 3>(st, table, t0 + 128 * kt, q.T, warp - kIssuer - 1, lane), b_load, lane);
                else tile_rows<DP, 96>(base + kt * P::tile, j.k_plane, st, table, h, t0 + 128 * kt, 0, q.T, u);
            }
            if (!k_boxes) {
                cp_commit();
                cp_wait<0>();
                __syncwarp();
                if (lane == 0)
                    for (int32_t kt = 0; kt < key_tiles; ++kt) mbar_arrive(b_load);
            }
        }
        // lse of the rows u and u + 96 (by boxes: of u - 32 and u + 32, by two warps) of tile i
        const int a0 = q_boxes ? u - 32 : u, a1 = q_boxes ? u + 32 : u + 96;
        auto lse_of = [&](int32_t i, int row) {
            const int64_t p = (int64_t)(tile0 + rank + share * i) * per + row;
            float x = INFINITY;                                  // weighs nothing
            int32_t g;
            const int32_t tok = token_of(st, (int32_t)min(p, (int64_t)total), g);
            if (i < mine && row >= 0 && row < per && p < total) x = __ldg(j.lse + (int64_t)(q.q0 + tok) * (st.kv_heads * st.group) + h * st.group + g);
            return x;                                            // as it is: a product here would wait for the load
        };
        auto stage_free = [&](int32_t stage, int32_t round) {
            const bool ok = round == 0 || lane != 0 || wait(b_free + 8 * stage, (round - 1) & 1);
            return __all_sync(0xffffffffu, ok);
        };
        int32_t stage = 0, round = 0, i = 0;
        auto slot_free = [&](int32_t i) {
            const bool ok = i < kSlots || lane != 0 || wait(b_read + 8 * (i % kSlots), (i / kSlots - 1) & 1);
            return __all_sync(0xffffffffu, ok);
        };
        auto put_lse = [&](int32_t i, float e0, float e1) {
            float* lse = reinterpret_cast<float*>(mem + P::lse) + (i % kSlots) * 128;
            lse[a0] = -kLog2e * e0;
            if (a1 < 128) lse[a1] = -kLog2e * e1;
            __syncwarp();
            if (lane == 0) mbar_arrive(b_lse + 8 * (i % kSlots));
        };
        auto next_stage = [&]() {
            if (++stage == kStages) {
                stage = 0;
                ++round;
            }
        };
        if (q_boxes && warp > kIssuer + 1) {
            // four tiles' lse ahead of the four that are announced: a load takes longer than a tile
            float now[4][2], next[4][2];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                now[e][0] = lse_of(e, a0);
                now[e][1] = lse_of(e, a1);
            }
            bool ok = true;
            for (; ok && i < mine; i += 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    next[e][0] = lse_of(i + 4 + e, a0);
                    next[e][1] = lse_of(i + 4 + e, a1);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!ok || i + e >= mine) break;
                    ok = slot_free(i + e);
                    if (ok) put_lse(i + e, now[e][0], now[e][1]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    now[e][0] = next[e][0];
                    now[e][1] = next[e][1];
                }
            }
        } else if (q_boxes) {
            for (; i < mine; ++i) {
                if (!stage_free(stage, round)) break;
                if (lane == 0) {
                    const int32_t p0 = (tile0 + rank + share * i) * per;
                    mbar_expect_tx(b_full + 8 * stage, (uint32_t)per * DP * 2);
#pragma unroll
                    for (int c = 0; c < DP / 64; ++c)
                        tma_load_3d(ring + stage * P::tile + c * 128 * 128, &q_map, 64 * c, h * st.group, q.q0 + p0 / st.group, b_full + 8 * stage);
                }
                __syncwarp();
                next_stage();
            }
        } else {
            float e0 = lse_of(0, a0), e1 = lse_of(0, a1);
            for (; i < mine; ++i) {
                if (!stage_free(stage, round) || !slot_free(i)) break;
                const int32_t p0 = (tile0 + rank + share * i) * per;
                const uint32_t dst = ring + stage * P::tile;
                put_lse(i, e0, e1);
                e0 = lse_of(i + 1, a0);
                e1 = lse_of(i + 1, a1);
                constexpr int CH = DP / 8;
#pragma unroll 4
                for (int v = u; v < 128 * CH; v += 96) {
                    const int k = v / CH, c = v % CH;
                    const bool there = p0 + k < total && 8 * c < st.head_dim;
                    int32_t g;
                    const int32_t tok = token_of(st, min(p0 + k, total - 1), g);
                    cp_async16(dst + (c >> 3) * 128 * 128 + k * 128 + (((c & 7) ^ (k & 7)) << 4),
                               j.q.base + (there ? 2 * ((int64_t)(q.q0 + tok) * j.q.row + (int64_t)(h * st.group + g) * j.q.head + 8 * c) : 0), there);
                }
                cp_commit();
                if (pending) {
                    cp_wait<1>();
                    announce();
                }
                pending = b_full + 8 * stage;
                next_stage();
            }
        }
        cp_wait<0>();
        if (pending) announce();
        // every load has landed when its sums are done; after a failure, wait for them here
        if (mine > 0) mbar_wait(b_load, 0, kWaitLimitNs);
        if (i < mine && warp == kIssuer + 1)
            for (int k = i < kStages ? 0 : i - kStages; k < i; ++k) mbar_wait(b_full + 8 * (k % kStages), (k / kStages) & 1, kWaitLimitNs);
    } else {
        // ---- sums: a key to a thread ---------------------------------------------------
        const int kt = wg >> 1, half = wg & 1;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const int32_t key = t0 + 128 * kt + t;
        const bool live = key < q.T;
        RowSpan see = rows_seeing(st, q, key, key, j.causal, j.window);
        if (!live) see.end = see.first;
        const float c = j.scale_log2;
        const int32_t columns = min(64, per - 64 * half);
        if (kt < key_tiles) {
            // this thread's key, DP / 2 of its dims, into tensor memory: lane = key, two dims to a column
            if (mine > 0) wait(b_load, 0);
            __syncwarp();
            uint32_t w[DP / 4];
#pragma unroll
            for (int v = 0; v < DP / 16; ++v) {
                const int d = DP / 16 * half + v;
                const uint4 x = ld_shared16(base + kt * P::tile + (d >> 3) * 128 * 128 + t * 128 + (((d & 7) ^ (t & 7)) << 4));
                w[4 * v] = x.x;
                w[4 * v + 1] = x.y;
                w[4 * v + 2] = x.z;
                w[4 * v + 3] = x.w;
            }
            const uint32_t to = tmem + 128 * kAccs + lanes + 64 * kt + DP / 4 * half;
            if (DP == 128) tmem_st32(to, w);
            else tmem_st16(to, w);
            tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_k);
        for (int32_t i = kt < key_tiles ? 0 : mine; i < mine; ++i) {
            const int32_t n = i * key_tiles + kt;
            const int slot = i % kSlots, acc = n % kAccs;
            if (!__all_sync(0xffffffffu, wait(b_lse + 8 * slot, (i / kSlots) & 1) && wait(b_s + 8 * acc, (n / kAccs) & 1))) break;
            tc_fence_after();
            const int32_t p0 = (tile0 + rank + share * i) * per + 64 * half;
            const int32_t a = see.first - p0, b = see.end - p0;      // columns that see this thread's key
            const bool edge = __any_sync(0xffffffffu, a > 0 || b < columns);
            const float4* lse = reinterpret_cast<const float4*>(mem + P::lse) + slot * 32 + 16 * half;
            float x0 = 0.0f, x1 = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t sr[32];
                tmem_ld32(sr, tmem + 128 * acc + lanes + 64 * half + 32 * k);
                tmem_wait_ld();
                tmem_loaded32(sr);
                if (k == 1) {
                    // the accumulator is read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_e + 8 * acc);
                }
                float* s = reinterpret_cast<float*>(sr);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float4 z = lse[8 * k + e];
                    fma2(s[4 * e], s[4 * e + 1], c, z.x, z.y);
                    fma2(s[4 * e + 2], s[4 * e + 3], c, z.z, z.w);
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) s[e] = exp2_fast(s[e]);
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) s[e] = 32 * k + e >= a && 32 * k + e < b ? s[e] : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 32; e += 2) add2(x0, x1, s[e], s[e + 1]);
            }
            sum += x0 + x1;
            __syncwarp();
            if (lane == 0) mbar_arrive(b_read + 8 * slot);
        }
        reinterpret_cast<float*>(mem + P::sums)[threadIdx.x] = sum;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssuer) tmem_dealloc(tmem, P::columns);
    const float* sums = reinterpret_cast<const float*>(mem + P::sums);        // [key tile][half][128]
    const int32_t at_sum = (threadIdx.x >> 7) * 256 + t;
    const int32_t key = t0 + (int32_t)threadIdx.x;               // of the first 256 threads: key tile by key tile
    const bool mine_to_write = threadIdx.x < kKeysTc && key < q.T;
    if (share == 1) {
        if (mine_to_write) add_weight(j, r, h, key, sums[at_sum] + sums[at_sum + 128]);
        return;
    }
    cluster_sync();
    if (rank == 0 && mine_to_write) {
        float x = 0.0f;
        for (int32_t k = 0; k < share; ++k) {
            const uint32_t at = cluster_at(base + P::sums + 4 * at_sum, k);
            float u, v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u) : "r"(at) : "memory");
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at + 512) : "memory");
            x += u + v;
        }
        add_weight(j, r, h, key, x);
    }
    cluster_sync();
}

// ---------------------------------------------------------------------------
// Few rows (a decode step): a warp takes 16 keys at a time straight into the fragments of
// mma.m16n8k16, keys in its 16 rows, the next 16 in flight meanwhile, and the packed rows eight
// at a time in its columns.  The sum over a head's dims has no order, so lane 4 i + c takes 16
// contiguous bytes of key i (dims 32 k + 8 c ...) for what the instruction calls dims 2c, 2c + 1,
// 2c + 8 and 2c + 9 of two of its steps, for keys and rows alike: no shared memory.  Bound by
// HBM, K being read once: a decode step of 16 requests with 4000 to 8000 cached tokens (201 MB
// of K) in 40.7 us, 4.9 TB/s; two CTAs to an SM hold 128 registers a thread, most of them keys
// in flight, and a third tile of them spills (55 us).  With the packed rows in the
// instruction's 16 rows, half of them empty, it took 49 us.
//
// A window leaves tokens out of the sums, but not out of the loads and products: four requests
// with 131072 tokens and a window of 4096 take 180 us, with caches of 4096 tokens 9.3.
// ---------------------------------------------------------------------------
constexpr int kRowWarps = 8, kRowKeys = 16;

template <bool HALF>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight packed rows: fragments of row p0 + lane / 4; lse and span of rows p0 + 2 c + e.
template <int K>
struct RowFrags {
    uint4 q[K];
    float lse[2];                // times -log2(e)
    Span  see[2];
};
template <int K>
__device__ __forceinline__ void load_rows(RowFrags<K>& f, const WeighJob& j, const Request& q, int32_t h, int32_t p0, int lane) {
    const StepView& st = j.step;
    const int32_t total = q.n * st.group, c = lane & 3, p = p0 + (lane >> 2);
    int32_t g = 0;
    const int32_t tok = token_of(st, p < total ? p : 0, g);
    const char* row = j.q.base + 2 * ((int64_t)(q.q0 + tok) * j.q.row + (int64_t)(h * st.group + g) * j.q.head);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        f.q[k] = make_uint4(0, 0, 0, 0);
        const int32_t d = 32 * k + 8 * c;
        if (p < total && d < st.head_dim) f.q[k] = __ldg(reinterpret_cast<const uint4*>(row + 2 * d));
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int32_t x = p0 + 2 * c + e;
        f.see[e] = Span{0, 0};
        f.lse[e] = 0.0f;
        if (x < total) {
            const int32_t t = token_of(st, x, g);
            f.see[e] = seen_by(q, t, t, j.causal, j.window);
            f.lse[e] = -kLog2e * __ldg(j.lse + (int64_t)(q.q0 + t) * (st.kv_heads * st.group) + h * st.group + g);
        }
    }
}

// STAY: the requests have at most eight times as many rows, whose fragments stay.  0: any number,
// whose fragments are loaded (from L1) for every 16 keys; 16 rows take 27 us with and 38 without
// them staying (8 requests x 8 heads of 64 dims, 8000 tokens), with 128 dims 45 and 48 (where two
// of them spill some 150 bytes, and what a call cannot do without is 19 us).
template <bool HALF, int DP, int STAY>
__global__ void __launch_bounds__(kRowWarps * 32, 2) kvs_weigh_rows_kernel(WeighJob j) {
    constexpr int K = DP / 32;                                   // 16-byte vectors of a lane and key
    const StepView& st = j.step;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 3, i = lane >> 2;
    const int32_t h = blockIdx.y, r = blockIdx.z;
    const Request q = load_request(st, r);
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;
    // this CTA's tiles of 16 keys, of which its warps take every eighth
    const int32_t all = (q.T + kRowKeys - 1) / kRowKeys;
    const int32_t first = (int32_t)((int64_t)all * blockIdx.x / gridDim.x), end = (int32_t)((int64_t)all * (blockIdx.x + 1) / gridDim.x);
    const int32_t mine = (end - first - warp + kRowWarps - 1) / kRowWarps;
    if (mine <= 0) return;
    auto key0 = [&](int32_t n) { return (first + warp + kRowWarps * n) * kRowKeys; };
    // a lane looks keys i and i + 8 of a tile up two tiles ahead, and loads them one ahead
    auto look_up = [&](int32_t n, int64_t (&row)[2]) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int32_t t = key0(n) + i + 8 * e;
            row[e] = n < mine && t < q.T ? row_of(st, table, t) : -1;
        }
    };
    // lanes 4 i and 4 i + 1 add to the weights of keys i and i + 8, which they load with the keys
    float* weights = j.weights + r * j.request_stride + h * j.head_stride;
    auto load = [&](int32_t n, const int64_t (&row)[2], uint4 (&kv)[2][K], float& old) {
        const int32_t t = key0(n) + i + 8 * c;
        old = 0.0f;
        if (j.decay != 0.0f && n < mine && c < 2 && t < q.T) old = weights[t];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                kv[e][k] = make_uint4(0, 0, 0, 0);
                const int32_t d = 32 * k + 8 * c;
                if (row[e] >= 0 && d < st.head_dim) kv[e][k] = *reinterpret_cast<const uint4*>(j.k_plane + 2 * (row[e] + (int64_t)h * st.head_dim + d));
            }
    };
    const int32_t total = q.n * st.group;
    RowFrags<K> stay[STAY ? STAY : 1];
    auto weigh = [&](int32_t n, const uint4 (&kv)[2][K], float old) {
        const int32_t t = key0(n) + i;
        float sum[2] = {0.0f, 0.0f};                             // keys t and t + 8, of this lane's rows
        auto add = [&](const RowFrags<K>& f) {
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                mma<HALF>(s, kv[0][k].x, kv[1][k].x, kv[0][k].y, kv[1][k].y, f.q[k].x, f.q[k].y);
                mma<HALF>(u, kv[0][k].z, kv[1][k].z, kv[0][k].w, kv[1][k].w, f.q[k].z, f.q[k].w);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t key = t + 8 * (e >> 1);
                if (key >= f.see[e & 1].lo && key < f.see[e & 1].hi) sum[e >> 1] += exp2_fast(fmaf(s[e] + u[e], j.scale_log2, f.lse[e & 1]));
            }
        };
#pragma unroll
        for (int x = 0; x < STAY; ++x) add(stay[x]);
        if (STAY == 0) {
            for (int32_t p0 = 0; p0 < total; p0 += 8) {
                RowFrags<K> f;
                load_rows<K>(f, j, q, h, p0, lane);
                add(f);
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
            sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
        }
        if (c < 2 && t + 8 * c < q.T) weights[t + 8 * c] = j.decay * old + (c ? sum[1] : sum[0]);
    };
    uint4 ka[2][K], kb[2][K];
    float wa, wb;
    int64_t row[2];
    look_up(0, row);
    load(0, row, ka, wa);
    look_up(1, row);
#pragma unroll
    for (int x = 0; x < STAY; ++x) load_rows<K>(stay[x], j, q, h, 8 * x, lane);
    for (int32_t n = 0; n < mine; n += 2) {
        load(n + 1, row, kb, wb);
        look_up(n + 2, row);
        weigh(n, ka, wa);
        load(n + 2, row, ka, wa);
        look_up(n + 3, row);
        if (n + 1 < mine) weigh(n + 1, kb, wb);
    }
}

template <bool HALF, int DP, int KT>
cudaError_t weigh_tc(const WeighJob& j, int sms, cudaStream_t s) {
    using P = WPlan<DP, KT>;
    const StepView& st = j.step;
    const int64_t rows = (int64_t)st.max_q * st.group;
    auto* k = kvs_weigh_tc_kernel<HALF, DP, KT>;
    cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, P::bytes);
    if (e != cudaSuccess) return e;
    CUtensorMap km{}, qm{};
    const bool k_boxes = plane_map(&km, st, j.k_plane, HALF), q_boxes = rows_map(&qm, st, j.q, HALF);
    const int64_t x = (st.max_kv + P::keys - 1) / P::keys, tiles = x * st.kv_heads * st.requests, row_tiles = (rows + 127) / 128;
    int share = 1;
    while (share < 8 && tiles * share * 2 <= sms && share * 2 <= row_tiles) share *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(x * share), st.kv_heads, st.requests);
    cfg.blockDim = dim3(P::threads);
    cfg.dynamicSmemBytes = P::bytes;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = share;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = share > 1;
    return cudaLaunchKernelEx(&cfg, k, j, km, qm, (int32_t)k_boxes, (int32_t)q_boxes, (int32_t)share);
}

template <bool HALF, int DP>
cudaError_t weigh(const WeighJob& j, int sms, cudaStream_t s) {
    const StepView& st = j.step;
    const int64_t rows = (int64_t)st.max_q * st.group;
    // Up to 32 rows: 8 requests x 8 heads of 128 dims with 8000 tokens take 68 us at 32 rows and 90 at
    // 48 (on the tensor cores' kernel 72); of 64 dims 54 and 70 (66).
    if (rows <= 32) {
        // CTAs for two rounds of two to an SM (weigh of a decode step: one round 45.2 us, two 40.5,
        // three 41.1, six 45.1), but not more than leave a warp four tiles.
        const int64_t pairs = (int64_t)st.kv_heads * st.requests, most = (st.max_kv + kRowWarps * kRowKeys * 4 - 1) / (kRowWarps * kRowKeys * 4);
        int64_t x = (4 * sms + pairs - 1) / pairs;
        x = x > most ? most : x;
        const dim3 grid((unsigned)x, st.kv_heads, st.requests);
        if (rows <= 8) kvs_weigh_rows_kernel<HALF, DP, 1><<<grid, kRowWarps * 32, 0, s>>>(j);
        else if (rows <= 16) kvs_weigh_rows_kernel<HALF, DP, 2><<<grid, kRowWarps * 32, 0, s>>>(j);
        else kvs_weigh_rows_kernel<HALF, DP, 0><<<grid, kRowWarps * 32, 0, s>>>(j);
        return cudaGetLastError();
    }
    // One key tile to a CTA up to 2560 rows: against 8000 tokens of 8 requests x 8 heads of 128 dims 64 rows
    // take 72 us (two tiles: 92), 256 79 (99), 1024 149 (167), 2048 250 (261), 4096 467 (450).
    return rows <= 2560 ? weigh_tc<HALF, DP, 1>(j, sms, s) : weigh_tc<HALF, DP, 2>(j, sms, s);
}

}  // namespace

int launch_weigh(const WeighJob& j, bool half, int sms, cudaStream_t s) {
    cudaError_t e;
    if (j.step.head_dim <= 64) e = half ? weigh<true, 64>(j, sms, s) : weigh<false, 64>(j, sms, s);
    else e = half ? weigh<true, 128>(j, sms, s) : weigh<false, 128>(j, sms, s);
    return e == cudaSuccess ? 1 : -(int)e;
}

}  // namespace kvs
