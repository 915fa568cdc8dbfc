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

constexpr int kWarps = 8;
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

// Byte offset of the 16-byte vector `c` of row `r` in a tile of rows of PITCH bytes: the
// vectors of eight neighbouring rows lie in different banks.
template <int PITCH>
__device__ __forceinline__ uint32_t swz(uint32_t r, uint32_t c) {
    return r * PITCH + ((c ^ (r & 7)) << 4);
}

struct Tile {
    int32_t r, h;          // request, KV head
    Request q;
    int32_t row0, rows;    // packed rows of the request
    Span    keys;          // that the tile's rows see, of this split
};

// Splits cut what a tile sees into parts of whole kKeys * kWarps keys.
__device__ __forceinline__ Span split_of(Span s, int32_t split, int32_t splits, int32_t unit) {
    const int32_t units = (s.hi - s.lo + unit - 1) / unit;
    const int32_t a = (int32_t)((int64_t)units * split / splits), b = (int32_t)((int64_t)units * (split + 1) / splits);
    Span o;
    o.lo = min(s.hi, s.lo + a * unit);
    o.hi = min(s.hi, s.lo + b * unit);
    return o;
}

// ---------------------------------------------------------------------------
// Few packed rows (a decode step): 16 rows to a CTA, whose eight warps take stages of 16
// keys in turn, each with its own running maximum, sum and output in registers and its own
// ring of stages, filled by cp.async: no barrier between warps until they join at the end.
// Bound by HBM: a key's K and V are read once for all query heads of its KV head.
// ---------------------------------------------------------------------------
template <bool HALF, int DP, int STAGES>
__global__ void __launch_bounds__(kWarps * 32) kvs_attend_rows_kernel(AttendJob j) {
    extern __shared__ __align__(1024) char smem[];
    using N = Num<HALF>;
    constexpr int PITCH = DP * 2, CH = DP / 8;                 // 16-byte vectors of a row
    constexpr int STAGE = 2 * kKeys * PITCH;                   // K, then V
    const StepView& st = j.step;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int32_t split = blockIdx.x % j.splits, r = blockIdx.z, h = blockIdx.y;
    const int32_t row0 = (blockIdx.x / j.splits) * kRows;
    const Request q = load_request(st, r);
    const int32_t rows = min(kRows, q.n * st.group - row0);
    if (rows <= 0) return;
    const Span all = seen_by(q, row0 / st.group, (row0 + rows - 1) / st.group, j.causal, j.window);
    const Span keys = split_of(all, split, j.splits, kKeys * kWarps);
    const uint32_t base = smem_u32(smem);
    const int32_t vecs = st.head_dim / 8;
    const int32_t* table = st.tables + (int64_t)r * st.table_stride;

    // Queries: the rows of the tile, through shared memory into the fragments of every warp.
    for (int v = threadIdx.x; v < kRows * CH; v += kWarps * 32) {
        const int i = v / CH, c = v % CH;
        const int32_t p = row0 + i, tok = p / st.group, head = h * st.group + p % st.group;
        const bool there = i < rows && c < vecs;
        const char* src = j.q.base + (there ? 2 * ((int64_t)(q.q0 + tok) * j.q.row + (int64_t)head * j.q.head + c * 8) : 0);
        cp_async16(base + swz<PITCH>(i, c), src, there);
    }
    cp_commit();
    cp_wait<0>();
    __syncthreads();
    uint32_t qf[DP / 16][4];
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) ldsm4(qf[k], base + swz<PITCH>(lane & 15, 2 * k + (lane >> 4)));
    __syncthreads();

    // This warp's stages: keys lo + 16 (warp + 8 i).
    const uint32_t ring = base + warp * STAGES * STAGE;
    const int32_t count = (keys.hi - keys.lo + kKeys - 1) / kKeys;
    const int32_t mine = (count - warp + kWarps - 1) / kWarps;
    auto load = [&](int32_t i) {
        if (i < mine) {
            const int32_t t0 = keys.lo + kKeys * (warp + kWarps * i);
            const uint32_t at = ring + (i % STAGES) * STAGE;
            // lane's key, looked up once
            const int32_t t = t0 + (lane & 15);
            const int64_t mrow = t < keys.hi ? row_of(st, table, t) : -1;
#pragma unroll
            for (int v = lane; v < kKeys * CH; v += 32) {
                const int k = v / CH, c = v % CH;
                const int64_t row = __shfl_sync(0xffffffffu, mrow, k);
                const bool there = row >= 0 && c < vecs;
                const int64_t off = there ? 2 * (row + (int64_t)h * st.head_dim + c * 8) : 0;
                cp_async16(at + swz<PITCH>(k, c), j.k_plane + off, there);
                cp_async16(at + kKeys * PITCH + swz<PITCH>(k, c), j.v_plane + off, there);
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load(i);

    float o[DP / 8][4];
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
    float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};
    // rows of this lane, and what each sees
    int32_t lo[2], hi[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int32_t p = row0 + (lane >> 2) + 8 * k;
        if ((lane >> 2) + 8 * k < rows) {
            const Span s = seen_by(q, p / st.group, p / st.group, j.causal, j.window);
            lo[k] = s.lo;
            hi[k] = s.hi;
        } else {
            lo[k] = 0;
            hi[k] = 0;
        }
    }
    for (int32_t i = 0; i < mine; ++i) {
        cp_wait<STAGES - 2>();
        __syncwarp();
        load(i + STAGES - 1);                                   // into the slot read last time
        const uint32_t at = ring + (i % STAGES) * STAGE;
        float s[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            uint32_t b[4];                                       // keys 0-7 and 8-15, dims 16k and 16k + 8
            ldsm4(b, at + swz<PITCH>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
            mma16816<HALF>(s[0], qf[k], b[0], b[1]);
            mma16816<HALF>(s[1], qf[k], b[2], b[3]);
        }
        const int32_t t0 = keys.lo + kKeys * (warp + kWarps * i) + 2 * (lane & 3);
        float mx[2] = {kNone, kNone};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t t = t0 + 8 * n + (e & 1);
                const bool seen = t >= lo[e >> 1] && t < min(hi[e >> 1], keys.hi);
                s[n][e] = seen ? s[n][e] * j.scale_log2 : kNone;
                mx[e >> 1] = fmaxf(mx[e >> 1], s[n][e]);
            }
        float f[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            mx[k] = fmaxf(mx[k], __shfl_xor_sync(0xffffffffu, mx[k], 1));
            mx[k] = fmaxf(mx[k], __shfl_xor_sync(0xffffffffu, mx[k], 2));
            const float to = fmaxf(m[k], mx[k]);
            f[k] = to == m[k] ? 1.0f : exp2_fast(m[k] - to);
            m[k] = to;
        }
        if (__any_sync(0xffffffffu, f[0] != 1.0f || f[1] != 1.0f)) {
            l[0] *= f[0];
            l[1] *= f[1];
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = s[n][e] == kNone ? 0.0f : exp2_fast(s[n][e] - m[e >> 1]);
                l[e >> 1] += s[n][e];
            }
        const uint32_t a[4] = {N::pack(s[0][0], s[0][1]), N::pack(s[0][2], s[0][3]),
                               N::pack(s[1][0], s[1][1]), N::pack(s[1][2], s[1][3])};
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
            uint32_t b[4];                                       // dims 16n and 16n + 8, keys 0-7 and 8-15
            ldsm4t(b, at + kKeys * PITCH + swz<PITCH>(lane & 15, 2 * n + (lane >> 4)));
            mma16816<HALF>(o[2 * n], a, b[0], b[1]);
            mma16816<HALF>(o[2 * n + 1], a, b[2], b[3]);
        }
        __syncwarp();
    }
    cp_wait<0>();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
    }
    __syncthreads();                                             // the rings become the join's buffers

    // Join: every warp writes its part, then each thread sums the warps' for its outputs.
    constexpr int OP = DP + 4;                                   // floats of a row
    float* po = reinterpret_cast<float*>(smem);                  // [warp][row][OP]
    float2* pml = reinterpret_cast<float2*>(smem + kWarps * kRows * OP * 4);
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            *reinterpret_cast<float2*>(po + (warp * kRows + (lane >> 2) + 8 * k) * OP + 8 * n + 2 * (lane & 3)) =
                make_float2(o[n][2 * k], o[n][2 * k + 1]);
    if ((lane & 3) == 0) {
        pml[warp * kRows + (lane >> 2)] = make_float2(m[0], l[0]);
        pml[warp * kRows + (lane >> 2) + 8] = make_float2(m[1], l[1]);
    }
    __syncthreads();
    for (int v = threadIdx.x; v < rows * (DP / 2); v += kWarps * 32) {
        const int i = v / (DP / 2), d = 2 * (v % (DP / 2));
        float M = kNone, L = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, pml[w * kRows + i].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = pml[w * kRows + i];
            const float f = ml.y == 0.0f ? 0.0f : exp2_fast(ml.x - M);
            const float2 p = *reinterpret_cast<const float2*>(po + (w * kRows + i) * OP + d);
            L += f * ml.y;
            x += f * p.x;
            y += f * p.y;
        }
        if (d >= st.head_dim) continue;
        const int32_t p = row0 + i, tok = q.q0 + p / st.group, head = h * st.group + p % st.group;
        const int64_t row = (int64_t)tok * (st.kv_heads * st.group) + head;
        if (j.splits == 1) {
            const float inv = L > 0.0f ? 1.0f / L : (L == 0.0f ? 0.0f : L);
            *reinterpret_cast<uint32_t*>(j.out.base + 2 * ((int64_t)tok * j.out.row + (int64_t)head * j.out.head + d)) =
                N::pack(x * inv, y * inv);
            if (d == 0 && j.lse) j.lse[row] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
        } else {
            const int64_t all_rows = (int64_t)st.total_q * st.kv_heads * st.group, at = split * all_rows + row;
            *reinterpret_cast<float2*>(j.partial + at * st.head_dim + d) = make_float2(x, y);
            if (d == 0) reinterpret_cast<float2*>(j.partial + (int64_t)j.splits * all_rows * st.head_dim)[at] = make_float2(M, L);
        }
    }
}

// Joins the splits' parts: a warp per row.
template <bool HALF>
__global__ void __launch_bounds__(128) kvs_attend_join_kernel(AttendJob j) {
    const StepView& st = j.step;
    using N = Num<HALF>;
    const int32_t heads = st.kv_heads * st.group;
    const int64_t all_rows = (int64_t)st.total_q * heads;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= all_rows) return;
    const float2* ml = reinterpret_cast<const float2*>(j.partial + (int64_t)j.splits * all_rows * st.head_dim);
    float M = kNone;
    for (int k = lane; k < j.splits; k += 32) M = fmaxf(M, ml[k * all_rows + row].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float L = 0.0f;
    const bool has = 4 * lane < st.head_dim;
    for (int k = 0; k < j.splits; ++k) {
        const float2 v = ml[k * all_rows + row];
        const float f = v.y == 0.0f ? 0.0f : exp2_fast(v.x - M);
        L += f * v.y;
        if (has) {
            const float4 p = *reinterpret_cast<const float4*>(j.partial + (k * all_rows + row) * st.head_dim + 4 * lane);
            o.x += f * p.x;
            o.y += f * p.y;
            o.z += f * p.z;
            o.w += f * p.w;
        }
    }
    const float inv = L > 0.0f ? 1.0f / L : (L == 0.0f ? 0.0f : L);
    const int64_t tok = row / heads, head = row % heads;
    if (has) {
        uint2 w;
        w.x = N::pack(o.x * inv, o.y * inv);
        w.y = N::pack(o.z * inv, o.w * inv);
        *reinterpret_cast<uint2*>(j.out.base + 2 * (tok * j.out.row + head * j.out.head + 4 * lane)) = w;
    }
    if (lane == 0 && j.lse) j.lse[row] = L == 0.0f ? kNone : (M + log2f(L)) * 0.69314718055994531f;
}

template <bool HALF, int DP, int STAGES>
cudaError_t attend_rows(const AttendJob& j, cudaStream_t s) {
    constexpr int ring = kWarps * STAGES * 2 * kKeys * DP * 2;
    constexpr int join = kWarps * kRows * ((DP + 4) * 4 + 8);
    constexpr int smem = ring > join ? ring : join;
    auto* k = kvs_attend_rows_kernel<HALF, DP, STAGES>;
    cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const int tiles = (int)(((int64_t)j.step.max_q * j.step.group + kRows - 1) / kRows);
    k<<<dim3((unsigned)(tiles * j.splits), j.step.kv_heads, j.step.requests), kWarps * 32, smem, s>>>(j);
    return cudaGetLastError();
}

}  // namespace

AttendPlan attend_plan(const StepView& st, int sms) {
    const int64_t rows = (int64_t)st.max_q * st.group, units = (int64_t)st.kv_heads * st.requests;
    AttendPlan p{rows > 32, 1};
    if (p.tc) {
        // One CTA of two row tiles to an SM: as many parts as keep the number of waves times a
        // part's steps (of 128 keys, and about four of start and end) lowest.
        const int64_t pair = 2 * tile_rows_of(st.group), tiles = (rows + pair - 1) / pair * units, steps = (st.max_kv + 127) / 128;
        int64_t best = -1;
        for (int64_t n = 1; n <= 64 && n <= (steps + 1) / 2; ++n) {
            const int64_t cost = (tiles * n + sms - 1) / sms * ((steps + n - 1) / n + 4);
            if (best < 0 || cost < best) {
                best = cost;
                p.splits = (int)n;
            }
        }
        return p;
    }
    const int64_t tiles = (rows + kRows - 1) / kRows * units, most = (st.max_kv + 255) / 256;      // a part of at least 256 keys
    if (tiles > 0) {
        int64_t n = (2 * (int64_t)sms + tiles - 1) / tiles;
        n = n > most ? most : n;
        p.splits = (int)(n < 1 ? 1 : n > 256 ? 256 : n);
    }
    return p;
}

int launch_attend(const AttendJob& j, bool half, cudaStream_t s) {
    cudaError_t e;
    if (j.tc) e = launch_attend_tc(j, half, s);
    else if (j.step.head_dim <= 64) e = half ? attend_rows<true, 64, 3>(j, s) : attend_rows<false, 64, 3>(j, s);
    else e = half ? attend_rows<true, 128, 3>(j, s) : attend_rows<false, 128, 3>(j, s);
    if (e != cudaSuccess) return -(int)e;
    if (j.splits == 1) return 1;
    const int64_t rows = (int64_t)j.step.total_q * j.step.kv_heads * j.step.group;
    if (half) kvs_attend_join_kernel<true><<<(unsigned)((rows + 3) / 4), 128, 0, s>>>(j);
    else kvs_attend_join_kernel<false><<<(unsigned)((rows + 3) / 4), 128, 0, s>>>(j);
    e = cudaGetLastError();
    return e == cudaSuccess ? 2 : -(int)e;
}

}  // namespace kvs
