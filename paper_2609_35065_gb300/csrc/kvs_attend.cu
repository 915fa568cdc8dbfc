// kvs_attend.cu -- attention of new tokens over the paged cache.
//
//     o = sum_t e^(s_t - m) v_t / sum_t e^(s_t - m),   s_t = scale * q . k_t
//
// in one pass over the keys: partial results (m, l, o) of any two sets of keys join as
// m = max(m1, m2), l = l1 e^(m1 - m) + l2 e^(m2 - m), o alike.  Scores are kept times
// log2(e), so that every exponential is one ex2.
//
// The query heads of a KV head and the new tokens are packed into the rows of one matrix
// (row = token * group + head), which reads each key and value once for all of them.
#include "kvs_async.cuh"
#include "kvs_ops.cuh"

namespace kvs {
namespace {

constexpr int kRows = 16;              // packed rows of a CTA
constexpr int kKeys = 16;              // keys of a warp's stage
constexpr float kNone = -INFINITY;

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool HALF>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The 8 x 8 matrix of 16-bit elements whose rows lie two elements to a lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Byte offset of the 16-byte vector `c` of row `r` in a tile of rows of PITCH bytes: the
// vectors of eight neighbouring rows lie in different banks.
template <int PITCH>
__device__ __forceinline__ uint32_t swz(uint32_t r, uint32_t c) {
    return r * PITCH + ((c ^ (r & 7)) << 4);
}

// Splits cut what a tile sees into parts of whole units of keys.
__device__ __forceinline__ Span split_of(Span s, int32_t split, int32_t splits, int32_t unit) {
    const int32_t units = (s.hi - s.lo + unit - 1) / unit;
    const int32_t a = (int32_t)((int64_t)units * split / splits), b = (int32_t)((int64_t)units * (split + 1) / splits);
    Span o;
    o.lo = min(s.hi, s.lo + a * unit);
    o.hi = min(s.hi, s.lo + b * unit);
    return o;
}

// ---------------------------------------------------------------------------
// Up to 16 packed rows (a decode step): the warps of a CTA take stages of 16 keys in
// turn, each with its own running maximum, sum and output in registers and its own ring of
// stages, filled by cp.async: no barrier between warps until they join at the end.  Bound by
// HBM: a key's K and V are read once for all query heads of its KV head.
//
// The products are S^T = K Q^T and O^T = V^T P^T, keys and dims in the 16 rows of mma.m16n8k16
// and the packed rows in its 8 columns: with the rows in the 16, most of them padding, the same
// work took twice the instructions, and those of a decode step as long as its loads.  As on the
// tensor cores the running maximum may lag behind, so that a stage need not exchange it.
//
// A weight goes into the product with V as the 16-bit number next to it and, in a second product,
// what that rounding took: in the shadow of the loads up to eight rows (0.2% of those 207 us), 2% with
// nine to sixteen, and the outputs are as near as with weights of 32 bits.
//
// Where a head's parts are up to eight and all clusters run at once, they are CTAs of a cluster
// that join through distributed shared memory; otherwise a second kernel joins them.
//
// 14 warps with two stages each: 64 requests over 2k to 8k tokens take 207 us (1.34 GB, 6.5 TB/s);
// 8 warps with three stages took 211, 5 with five 262 (with the products the other way round).
// ---------------------------------------------------------------------------
template <int DP, int WARPS, int STAGES>
struct RowsPlan {
    static constexpr int ring = WARPS * STAGES * 2 * kKeys * DP * 2;
    static constexpr int join = WARPS * kRows * ((DP + 4) * 4 + 8);
    // [row][DP] and [row] (m, l) of the CTA, for its cluster
    static constexpr int part = kRows * (DP * 4 + 8);
    static constexpr int bytes = ring > join + part ? ring : join + part;
};

// NT: column tiles of eight rows.
template <bool HALF, int DP, int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32) kvs_attend_rows_kernel(AttendJob j) {
    extern __shared__ __align__(1024) char smem[];
    using N = Num<HALF>;
    constexpr int PITCH = DP * 2, CH = DP / 8;                 // 16-byte vectors of a row
    constexpr int STAGE = 2 * kKeys * PITCH;                   // K, then V
    constexpr float kLag = HALF ? 15.0f : 20.0f;               // log2 that a weight may reach before the reference is raised
    const StepView& st = j.step;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 3, i8 = lane >> 2;
    const int32_t split = blockIdx.x, r = blockIdx.z, h = blockIdx.y;
    if (j.splits > 1 && !j.cluster) grid_trigger();            // the join may come and wait
    const Request q = load_request(st, r);
    const int32_t rows = q.n * st.group;
    if (rows <= 0) return;
    const Span all = seen_by(q, 0, q.n - 1, j.causal, j.window);
    const Span keys = split_of(all, split, j.splits, kKeys * WARPS);
    const float top_at = HALF ? half_top(keys.hi - keys.lo, 8) : 0.0f;       // log2 of the maximum's weight then (8 costs nothing here)
    const uint32_t base = smem_u32(smem);
    const int32_t vecs = st.head_dim / 8;
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;

    // Queries: through shared memory into the fragments of every warp.
    for (int v = threadIdx.x; v < 8 * NT * CH; v += WARPS * 32) {
        const int i = v / CH, d = v % CH;
        const bool there = i < rows && d < vecs;
        int32_t g;
        const int32_t tok = token_of(st, there ? i : 0, g);
        const char* src = j.q.base + (there ? 2 * ((int64_t)(q.q0 + tok) * j.q.row + (int64_t)(h * st.group + g) * j.q.head + d * 8) : 0);
        cp_async16(base + swz<PITCH>(i, d), src, there);
    }
    cp_commit();
    // This warp's stages: keys lo + 16 (warp + 8 i).  The row of this lane's key of a stage is
    // looked up a stage before it is loaded.
    const uint32_t ring = base + warp * STAGES * STAGE;
    const int32_t count = (keys.hi - keys.lo + kKeys - 1) / kKeys;
    const int32_t mine = (count - warp + WARPS - 1) / WARPS;
    auto look_up = [&](int32_t i) {
        const int32_t t = keys.lo + kKeys * (warp + WARPS * i) + (lane & 15);
        return i < mine && t < keys.hi ? row_of(st, table, t) : (int64_t)-1;
    };
    int64_t mrow = look_up(0);
    auto load = [&](int32_t i) {
        if (i < mine) {
            const uint32_t at = ring + (i % STAGES) * STAGE;
            const int64_t ahead = look_up(i + 1);
#pragma unroll
            for (int v = lane; v < kKeys * CH; v += 32) {
                const int k = v / CH, d = v % CH;
                const int64_t row = __shfl_sync(0xffffffffu, mrow, k);
                const bool there = row >= 0 && d < vecs;
                const int64_t off = there ? 2 * (row + (int64_t)h * st.head_dim + d * 8) : 0;
                cp_async16(at + swz<PITCH>(k, d), j.k_plane + off, there);
                cp_async16(at + kKeys * PITCH + swz<PITCH>(k, d), j.v_plane + off, there);
            }
            mrow = ahead;
        }
        cp_commit();
    };
    cp_wait<0>();
    __syncthreads();
    uint32_t qf[NT][DP / 16][2];                                 // columns: rows 8 n + i8, dims 16 k + 2 c and + 8
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < DP / 16; k += 2) {
            uint32_t x[4];
            ldsm4(x, base + swz<PITCH>(8 * n + (lane & 7), 2 * k + (lane >> 3)));
            qf[n][k][0] = x[0];
            qf[n][k][1] = x[1];
            qf[n][k + 1][0] = x[2];
            qf[n][k + 1][1] = x[3];
        }
    __syncthreads();                                             // the ring may go over them
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load(i);

    // This lane's rows 8 n + 2 c + e: reference maximum, sum (of its keys), span; output at dims i8 and i8 + 8 of each 16.
    float o[NT][DP / 16][4], m[NT][2], l[NT][2];
    int32_t lo[NT][2], hi[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][d][e] = 0.0f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = 8 * n + 2 * c + e;
            m[n][e] = kNone;
            l[n][e] = 0.0f;
            int32_t g;
            const int32_t tok = token_of(st, i, g);
            const Span s = seen_by(q, tok, tok, j.causal, j.window);
            lo[n][e] = i < rows ? s.lo : 0;
            hi[n][e] = i < rows ? min(s.hi, keys.hi) : 0;
        }
    }
    for (int32_t i = 0; i < mine; ++i) {
        cp_wait<STAGES - 2>();
        __syncwarp();
        load(i + STAGES - 1);                                    // into the slot read last time
        const uint32_t at = ring + (i % STAGES) * STAGE;
        float s[NT][2][4];                                       // two sums, of even and odd dims' steps
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][b][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            uint32_t a[4];                                       // keys 0-7 and 8-15, dims 16 k and + 8
            ldsm4(a, at + swz<PITCH>(lane & 15, 2 * k + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816<HALF>(s[n][k & 1], a, qf[n][k][0], qf[n][k][1]);
        }
        // keys t0 + i8 and + 8 of rows 2 c, 2 c + 1: elements 0, 1 and 2, 3
        const int32_t t0 = keys.lo + kKeys * (warp + WARPS * i) + i8;
        bool above = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t t = t0 + 8 * (e >> 1);
                const float x = (s[n][0][e] + s[n][1][e]) * j.scale_log2;
                s[n][0][e] = t >= lo[n][e & 1] && t < hi[n][e & 1] ? x : kNone;
                above = above || s[n][0][e] > m[n][e & 1] + kLag;
            }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(s[n][0][e], s[n][0][e + 2]);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                    const float to = fmaxf(m[n][e], top - top_at), f = to == m[n][e] ? 1.0f : exp2_fast(m[n][e] - to);
                    m[n][e] = to;
                    l[n][e] *= f;
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d) {
                        o[n][d][e] *= f;
                        o[n][d][e + 2] *= f;
                    }
                }
        }
        uint32_t p[NT][2], rest[NT][2];                          // columns: rows 8 n + i8, keys 2 c and + 8; what rounding took of them
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][0][e] = s[n][0][e] == kNone ? 0.0f : exp2_fast(s[n][0][e] - m[n][e & 1]);
                l[n][e & 1] += s[n][0][e];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = s[n][0][2 * e], y = s[n][0][2 * e + 1];
                const uint32_t w = N::pack(x, y);
                const float2 r = N::to2(w);
                p[n][e] = transposed(w);
                rest[n][e] = transposed(N::pack(x - r.x, y - r.y));
            }
        }
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            uint32_t a[4];                                       // dims 16 d and + 8, keys 0-7 and 8-15
            ldsm4t(a, at + kKeys * PITCH + swz<PITCH>((lane & 7) + ((lane >> 4) << 3), 2 * d + ((lane >> 3) & 1)));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma16816<HALF>(o[n][d], a, p[n][0], p[n][1]);
                mma16816<HALF>(o[n][d], a, rest[n][0], rest[n][1]);
            }
        }
        __syncwarp();
    }
    cp_wait<0>();
    __syncthreads();                                             // the rings become the join's buffers

    // Join: every warp writes its part, then each thread sums the warps' for its outputs.
    constexpr int OP = DP + 4;                                   // floats of a row
    float* po = reinterpret_cast<float*>(smem);                  // [warp][row][OP]
    float2* pml = reinterpret_cast<float2*>(smem + WARPS * kRows * OP * 4);
    float* part = reinterpret_cast<float*>(smem + RowsPlan<DP, WARPS, STAGES>::join);
    float2* part_ml = reinterpret_cast<float2*>(part + kRows * DP);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = 8 * n + 2 * c + e;
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                po[(warp * kRows + i) * OP + 16 * d + i8] = o[n][d][e];
                po[(warp * kRows + i) * OP + 16 * d + 8 + i8] = o[n][d][e + 2];
            }
            if (i8 == 0) pml[warp * kRows + i] = make_float2(m[n][e], l[n][e]);
        }
    __syncthreads();
    for (int v = threadIdx.x; v < rows * (DP / 2); v += WARPS * 32) {
        const int i = v / (DP / 2), d = 2 * (v % (DP / 2));
        float M = kNone, L = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, pml[w * kRows + i].x);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 ml = pml[w * kRows + i];
            const float f = ml.y == 0.0f ? 0.0f : exp2_fast(ml.x - M);
            const float2 p = *reinterpret_cast<const float2*>(po + (w * kRows + i) * OP + d);
            L += f * ml.y;
            x += f * p.x;
            y += f * p.y;
        }
        if (d >= st.head_dim) continue;
        int32_t g;
        const int32_t tok = q.q0 + token_of(st, i, g), head = h * st.group + g;
        const int64_t row = (int64_t)tok * (st.kv_heads * st.group) + head;
        if (j.splits == 1) {
            const float inv = L > 0.0f ? 1.0f / L : L;
            *reinterpret_cast<uint32_t*>(j.out.base + 2 * ((int64_t)tok * j.out.row + (int64_t)head * j.out.head + d)) = N::pack(x * inv, y * inv);
            if (d == 0 && j.lse) j.lse[row] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
        } else if (j.cluster) {
            *reinterpret_cast<float2*>(part + i * DP + d) = make_float2(x, y);
            if (d == 0) part_ml[i] = make_float2(M, L);
        } else {
            const int64_t all_rows = (int64_t)st.total_q * st.kv_heads * st.group, to = split * all_rows + row;
            *reinterpret_cast<float2*>(j.partial + to * st.head_dim + d) = make_float2(x, y);
            if (d == 0) reinterpret_cast<float2*>(j.partial + (int64_t)j.splits * all_rows * st.head_dim)[to] = make_float2(M, L);
        }
    }
    if (!j.cluster) return;
    // The cluster's CTAs share out the outputs and read one another's parts of them, in order.
    cluster_sync();
    const int total = rows * (DP / 2), share = (total + j.splits - 1) / j.splits;
    for (int v = split * share + threadIdx.x; v < min(total, (split + 1) * share); v += WARPS * 32) {
        const int i = v / (DP / 2), d = 2 * (v % (DP / 2));
        if (d >= st.head_dim) continue;
        float2 ml[kCluster], p[kCluster];
        float M = kNone, L = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
            ml[k] = make_float2(kNone, 0.0f);
            p[k] = make_float2(0.0f, 0.0f);
            if (k < j.splits) {
                ml[k] = cluster_ld2(cluster_at(smem_u32(part_ml + i), k));
                p[k] = cluster_ld2(cluster_at(smem_u32(part + i * DP + d), k));
            }
            M = fmaxf(M, ml[k].x);
        }
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
            const float f = ml[k].y == 0.0f ? 0.0f : exp2_fast(ml[k].x - M);
            L += f * ml[k].y;
            x += f * p[k].x;
            y += f * p[k].y;
        }
        int32_t g;
        const int32_t tok = q.q0 + token_of(st, i, g), head = h * st.group + g;
        const float inv = L > 0.0f ? 1.0f / L : L;
        *reinterpret_cast<uint32_t*>(j.out.base + 2 * ((int64_t)tok * j.out.row + (int64_t)head * j.out.head + d)) = N::pack(x * inv, y * inv);
        if (d == 0 && j.lse) j.lse[(int64_t)tok * (st.kv_heads * st.group) + head] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
    }
    // no CTA leaves while another may read its part
    cluster_sync();
}

// Joins the splits' parts: a warp per row of a request, whose lanes weigh a split each and whose
// loads of the parts go out eight at a time.  Rows of no request have no parts and are left alone.
constexpr int kJoinWarps = 4;
template <bool HALF>
__global__ void __launch_bounds__(32 * kJoinWarps) kvs_attend_join_kernel(AttendJob j) {
    const StepView& st = j.step;
    using N = Num<HALF>;
    const int32_t heads = st.kv_heads * st.group;
    const int64_t all_rows = (int64_t)st.total_q * heads, own = (int64_t)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    // ranges and lengths were there before the parts' kernel began: no need to wait for it
    const Request q = load_request(st, blockIdx.y);
    grid_wait();
    if (own >= (int64_t)q.n * heads) return;
    const int64_t row = (int64_t)q.q0 * heads + own;
    const float2* ml = reinterpret_cast<const float2*>(j.partial + (int64_t)j.splits * all_rows * st.head_dim);
    float M = kNone;
    for (int k = lane; k < j.splits; k += 32) M = fmaxf(M, ml[k * all_rows + row].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float L = 0.0f;
    const bool has = 4 * lane < st.head_dim;
    const float* part = j.partial + row * st.head_dim + 4 * lane;
    for (int k0 = 0; k0 < j.splits; k0 += 32) {
        float2 v = make_float2(kNone, 0.0f);
        if (k0 + lane < j.splits) v = ml[(k0 + lane) * all_rows + row];
        const float f = v.y == 0.0f ? 0.0f : exp2_fast(v.x - M), g = f * v.y;
        for (int k = 0; k < min(32, j.splits - k0); k += 8) {
            float4 p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (has && k0 + k + e < j.splits) p[e] = *reinterpret_cast<const float4*>(part + (k0 + k + e) * all_rows * st.head_dim);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __shfl_sync(0xffffffffu, f, k + e);
                L += __shfl_sync(0xffffffffu, g, k + e);
                o.x += w * p[e].x;
                o.y += w * p[e].y;
                o.z += w * p[e].z;
                o.w += w * p[e].w;
            }
        }
    }
    const float inv = L > 0.0f ? 1.0f / L : L;
    const int64_t tok = row / heads, head = row % heads;
    if (has) {
        uint2 w;
        w.x = N::pack(o.x * inv, o.y * inv);
        w.y = N::pack(o.z * inv, o.w * inv);
        *reinterpret_cast<uint2*>(j.out.base + 2 * (tok * j.out.row + head * j.out.head + 4 * lane)) = w;
    }
    if (lane == 0 && j.lse) j.lse[row] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
}

template <bool HALF, int DP, int NT>
cudaError_t attend_rows(const AttendJob& j, cudaStream_t s) {
    // 14 warps of two column tiles of wide heads would have too few registers
    constexpr int WARPS = DP == 128 && NT == 2 ? 12 : 14, STAGES = 2, smem = RowsPlan<DP, WARPS, STAGES>::bytes;
    auto* k = kvs_attend_rows_kernel<HALF, DP, NT, WARPS, STAGES>;
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)j.splits, j.step.kv_heads, j.step.requests);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = j.splits;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = j.cluster;
    return cudaLaunchKernelEx(&cfg, k, j);
}

template <bool HALF>
cudaError_t attend_few(const AttendJob& j, cudaStream_t s) {
    const bool eight = j.step.max_q * j.step.group <= 8;
    if (j.step.head_dim <= 64) return eight ? attend_rows<HALF, 64, 1>(j, s) : attend_rows<HALF, 64, 2>(j, s);
    return eight ? attend_rows<HALF, 128, 1>(j, s) : attend_rows<HALF, 128, 2>(j, s);
}

}  // namespace

AttendPlan attend_plan(const StepView& st, int sms) {
    const int64_t rows = (int64_t)st.max_q * st.group, units = (int64_t)st.kv_heads * st.requests;
    // Up to 16 rows: mma.sync, whose work is in the shadow of the loads; above, the tensor cores (at
    // 20 rows over 3000 to 8000 tokens 62 to 79 us against 65 to 91, at 48 rows 62 to 80 against 97 to 169).
    AttendPlan p{rows > 16, 1, 1, 0};
    const int32_t tile = tile_rows_of(st.group);
    if (p.tc && rows > tile) p.row_tiles = 2;
    // One CTA to an SM (two of one narrow tile); steps of 128 keys, and about four of start and end.
    const int64_t per = p.tc ? (int64_t)tile * p.row_tiles : 16, tiles = (rows + per - 1) / per * units, steps = (st.max_kv + 127) / 128, start = 4, join = p.row_tiles == 2 ? 6 : p.tc ? 3 : 5;
    if (p.tc && p.row_tiles == 1 && st.head_dim <= 64) sms *= 2;
    // As many parts as keep the number of waves times a part's steps lowest.  The join of parts of
    // few rows costs about five steps of theirs, within a cluster one (8 heads of 128 dims, captured
    // in a graph: one decoding request over 2000 tokens 7.3 us with a cluster and 8.4 without, over
    // 4000 9.8 and 11.2, over 8000 12.4 and 13.4, over 16000, in 19 parts, 18.2); of one tile three,
    // or one (20 rows over 2000 tokens 10.0 us with a cluster, 11.8 without, over 4000 12.7 and 14.3;
    // of eight requests and two heads over 1000 10.3 and 12.1), of two tiles six, where a cluster
    // loses (293 tokens over 4000 37 us, 33 without, both before the join went by requests).
    // The plan goes by max_kv, whatever the window: four decoding requests with a window of 4096
    // in 131072 tokens take 32 us, with caches of 4096 tokens 18.5.
    int64_t best = -1;
    for (int64_t n = 1; n <= 256 && n <= (steps + 1) / 2; ++n) {
        // Clusters have room where all of their CTAs run at once: a cluster's lie on neighbouring SMs, and
        // of each such group up to n - 1 stay unused (16 clusters of 7 did not fit on 152 SMs: 16 us for 10).
        const bool cluster = p.row_tiles == 1 && n > 1 && n <= kCluster && tiles * n <= sms - 10 * (n - 1);
        const int64_t cost = (tiles * n + sms - 1) / sms * ((steps + n - 1) / n + start) + (n == 1 ? 0 : cluster ? 1 : join);
        if (best < 0 || cost < best) {
            best = cost;
            p.splits = (int)n;
            p.cluster = cluster;
        }
    }
    return p;
}

int launch_attend(const AttendJob& j, bool half, cudaStream_t s) {
    cudaError_t e = j.tc ? launch_attend_tc(j, half, s) : half ? attend_few<true>(j, s) : attend_few<false>(j, s);
    if (e != cudaSuccess) return -(int)e;
    if (j.splits == 1 || j.cluster) return 1;
    // The join is launched programmatically: its CTAs are in place when the parts are done.
    const int64_t rows = (int64_t)j.step.max_q * j.step.kv_heads * j.step.group;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((rows + kJoinWarps - 1) / kJoinWarps), j.step.requests);
    cfg.blockDim = dim3(32 * kJoinWarps);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, half ? kvs_attend_join_kernel<true> : kvs_attend_join_kernel<false>, j);
    return e == cudaSuccess ? 2 : -(int)e;
}

}  // namespace kvs
