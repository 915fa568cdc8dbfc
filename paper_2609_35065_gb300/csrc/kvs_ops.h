// kvs_ops.h -- what the C entries of the model operators (kvs_ops_api.cpp) hand to their
// kernels.  Not part of the public ABI.
#pragma once

#include <cmath>
#include <cstdint>
#include <cuda_runtime.h>

#include "kvs.h"
#include "kvs_internal.h"

namespace kvs {

// The device's part of a step: geometry of the planes, and the requests' device arrays.
struct StepView {
    const int32_t* tables;
    const int32_t* kv_lens;
    const int32_t* q_starts;         // nullptr: request r has the one row r
    int32_t*       err;              // device error word (first error wins)
    int32_t  requests, table_stride, total_q, max_q, max_kv;
    int32_t  block_size;
    uint32_t block_m, block_p;       // t / block_size = (t * block_m) >> block_p (FastDiv)
    int32_t  num_blocks;
    int32_t  kv_heads, head_dim;
    int32_t  group;                  // query heads per KV head
    uint32_t group_m, group_p;       // p / group = (p * group_m) >> group_p
};

struct RowsView {
    char*   base;
    int64_t row, head;               // strides in elements
};

struct AppendJob {
    StepView step;
    RowsView q, q_out, k, v;
    char *k_plane, *v_plane;
    const int32_t* positions;
    const float2*  turns;
    float    scale;
    int32_t  rot_dim, interleaved, q_heads;
    const uint8_t* axis;             // of each pair
    int32_t  axes;                   // 0: positions has one entry to a row; else [axes][...] at axis_stride
    int64_t  axis_stride;
};

struct AttendJob {
    StepView step;
    RowsView q, out;
    const char *k_plane, *v_plane;
    float*   lse;
    float*   partial;                // splits > 1: [splits][rows of total_q * heads][head_dim], then their (m, l) pairs
    float    scale_log2;             // scale * log2(e)
    float    scale_low;              // held: what scale_log2 lacks of that
    int32_t  causal, window;
    int32_t  held;                   // 1: a window with `sinks` first tokens that stay visible
    int32_t  sinks;
    int32_t  splits;
    int32_t  cluster;                // 1: a head's parts are CTAs of a cluster, which joins them
    int32_t  tc;                     // 1: on the tensor cores' kernel
    int32_t  row_tiles;              // of a CTA there
    int32_t  stay;                   // SMs that CTAs stay on, going over all pairs of row tiles; 0: a CTA to each
};

struct WeighJob {
    StepView step;
    RowsView q;
    const char* k_plane;
    const float* lse;
    float*   weights;
    int64_t  request_stride, head_stride;
    float    scale_log2, decay;
    int32_t  causal, window;
    int32_t  held, sinks;            // as in attention
    float    scale, scale_low;       // held: as given; what scale_log2 lacks
    int32_t  by_places;              // 1: of kvs_weigh_sinks, hidden tokens or not
};

struct EvictJob {
    StepView step;
    const void* const* planes;       // HOST array of 2L device addresses
    int32_t  layers;
    const float* weights;
    int64_t  layer_stride, request_stride, head_stride;
    const int32_t* dst_tables;
    int32_t  dst_stride, budget, sinks, recent;
    int32_t* kept;
    float*   new_weights;
    int32_t* new_lens;
};

// scale log2(e) as a binary32 number, cut towards zero: what it lacks (scale_rest) has its sign then, so that infinite scores
// times both stay what they are.
inline double scale_times_log2e(float scale) { return (double)scale * 1.4426950408889634; }
inline float scale_cut(float scale) {
    const double c = scale_times_log2e(scale);
    const float high = (float)c;
    return std::fabs((double)high) > std::fabs(c) ? std::nextafter(high, 0.0f) : high;
}
inline float scale_rest(float scale, float high) { return std::isfinite(high) ? (float)(scale_times_log2e(scale) - (double)high) : 0.0f; }

// Fills in the reciprocals of block_size and group.
void set_divisors(StepView& st);
// Each enqueues its kernels and returns how many (negative: a cudaError_t, negated).
int launch_append(const AppendJob& j, bool half, cudaStream_t s);
cudaError_t launch_append_axes(const AppendJob& j, bool half, cudaStream_t s);
int launch_attend(const AttendJob& j, bool half, cudaStream_t s);
int launch_weigh(const WeighJob& j, bool half, int sms, cudaStream_t s);
int launch_evict(const EvictJob& j, cudaStream_t s);
// Packed rows (token * group + head) of a 128-row tile: whole tokens, where a token's fit.
inline __host__ __device__ int32_t tile_rows_of(int32_t group) { return group <= 128 ? 128 / group * group : 128; }
// How attention goes about a step, by its bounds alone: the kernel, and the parts that a
// request's cached tokens are split into.
struct AttendPlan {
    int tc, splits, row_tiles, cluster;
};
constexpr int kCluster = 8;            // most parts that a cluster joins
constexpr int kClusterPairs = 4;       // ... of two row tiles
// Whether `ctas` CTAs, one to an SM, all run at once in clusters of n.  A cluster's lie on neighbouring SMs, of which
// some stay unused: what the occupancy calculator says of 152 SMs.
inline bool clusters_fit(int64_t ctas, int64_t n, int sms) {
    constexpr int room[kCluster + 1] = {0, 152, 152, 138, 144, 140, 138, 105, 120};
    return n <= kCluster && ctas * 152 <= (int64_t)room[n] * sms;
}
AttendPlan attend_plan(const StepView& st, int sms);
// A plane's TMA map (a CUtensorMap at `map`) in boxes of whole blocks, or of 128 tokens of one,
// of one head's 64 elements; false where blocks do not tile 128 tokens (kvs_attend_tc.cu).
bool plane_map(void* map, const StepView& st, const void* plane, bool half);
// The same of a step's rows, in boxes of one KV head's query heads by as many tokens as make
// at most 128 packed rows.
bool rows_map(void* map, const StepView& st, const RowsView& rows, bool half);
cudaError_t launch_attend_tc(const AttendJob& j, bool half, cudaStream_t s);
// Of a window with sinks, on CTAs that stay: pairs of row tiles that there may be at most, and the launch.
int64_t held_items(const StepView& st);
cudaError_t launch_attend_held(const AttendJob& j, bool half, int sms, cudaStream_t s);

// The current device's error word and number of SMs (kvs_api.cpp); allocates them at the first call,
// and takes no lock later.
int ops_device(int32_t** err, int* sms);
// Counts kernels for kvs_stat_launches.
void ops_launched(int n);
// kvs_check_errors' reading of the error word.
int ops_read_error(cudaStream_t s);

}  // namespace kvs
