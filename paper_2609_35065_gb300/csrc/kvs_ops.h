// kvs_ops.h -- what the C entries of the model operators (kvs_ops_api.cpp) hand to their
// kernels.  Not part of the public ABI.
#pragma once

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
};

struct AttendJob {
    StepView step;
    RowsView q, out;
    const char *k_plane, *v_plane;
    float*   lse;
    float*   partial;                // splits > 1: [splits][rows of total_q * heads][head_dim], then their (m, l) pairs
    float    scale_log2;             // scale * log2(e)
    int32_t  causal, window;
    int32_t  splits;
    int32_t  cluster;                // 1: a head's parts are CTAs of a cluster, which joins them
    int32_t  tc;                     // 1: on the tensor cores' kernel
    int32_t  row_tiles;              // of a CTA there
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

// Fills in the reciprocals of block_size and group.
void set_divisors(StepView& st);
// Each enqueues its kernels and returns how many (negative: a cudaError_t, negated).
int launch_append(const AppendJob& j, bool half, cudaStream_t s);
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
AttendPlan attend_plan(const StepView& st, int sms);
// A plane's TMA map (a CUtensorMap at `map`) in boxes of whole blocks, or of 128 tokens of one,
// of one head's 64 elements; false where blocks do not tile 128 tokens (kvs_attend_tc.cu).
bool plane_map(void* map, const StepView& st, const void* plane, bool half);
// The same of a step's rows, in boxes of one KV head's query heads by as many tokens as make
// at most 128 packed rows.
bool rows_map(void* map, const StepView& st, const RowsView& rows, bool half);
cudaError_t launch_attend_tc(const AttendJob& j, bool half, cudaStream_t s);

// The current device's error word and number of SMs (kvs_api.cpp); allocates them at the first call,
// and takes no lock later.
int ops_device(int32_t** err, int* sms);
// Counts kernels for kvs_stat_launches.
void ops_launched(int n);
// kvs_check_errors' reading of the error word.
int ops_read_error(cudaStream_t s);

}  // namespace kvs
