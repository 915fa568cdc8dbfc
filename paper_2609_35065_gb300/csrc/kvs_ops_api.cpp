// kvs_ops_api.cpp -- C entries of the model operators on the paged cache (kvs_append,
// kvs_attend, kvs_weigh, kvs_evict and the forms with axes and sinks): arguments are checked on the host before any CUDA
// call, and the kernels are enqueued on the caller's stream.  Nothing is allocated after
// the device's first call.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <new>
#include <vector>

#include "kvs.h"
#include "kvs_ops.h"

namespace kvs {
namespace {

int ops_fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

#define KVS_TRY(call)            \
    do {                         \
        const int rc_ = (call);  \
        if (rc_) return rc_;     \
    } while (0)

// No C++ exception leaves a C entry.
template <class F>
int entry(F&& f) {
    try {
        set_last_error("");
        return f();
    } catch (const std::bad_alloc&) {
        return KVS_ERR_NOMEM;
    } catch (const std::exception&) {
        return KVS_ERR_INVALID_ARG;
    }
}

// rowless: the call uses no row of the step, which may then have none.
int view_of(const kvs_geometry* g, const kvs_step* s, int32_t q_heads, StepView& v, bool rowless = false) {
    if (!g) return ops_fail(KVS_ERR_INVALID_ARG, "geometry is NULL");
    if (g->num_layers <= 0 || g->num_kv_heads <= 0 || g->head_dim <= 0)
        return ops_fail(KVS_ERR_INVALID_ARG, "layers, kv heads and head dim must be positive");
    if (g->num_layers > 32768) return ops_fail(KVS_ERR_INVALID_ARG, "too many layers");
    if (g->block_size <= 0) return ops_fail(KVS_ERR_INVALID_ARG, "block_size must be positive");
    if (g->elem_bytes != 2) return ops_fail(KVS_ERR_UNSUPPORTED, "elem_bytes must be 2 (got %d)", g->elem_bytes);
    if (g->head_dim % 8 || g->head_dim > 128)
        return ops_fail(KVS_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 up to 128 (got %d)", g->head_dim);
    if (g->num_kv_heads > 65535) return ops_fail(KVS_ERR_UNSUPPORTED, "at most 65535 kv heads");
    if (!s) return ops_fail(KVS_ERR_INVALID_ARG, "step is NULL");
    if (s->dtype != KVS_DTYPE_BF16 && s->dtype != KVS_DTYPE_F16)
        return ops_fail(KVS_ERR_INVALID_ARG, "dtype must be KVS_DTYPE_BF16 or KVS_DTYPE_F16 (got %d)", s->dtype);
    if (s->num_requests < 0 || s->total_q < 0 || s->max_q < 0 || s->max_kv < 0 || s->table_stride < 0)
        return ops_fail(KVS_ERR_INVALID_ARG, "a step's counts must not be negative");
    if (s->max_kv > 1 << 30) return ops_fail(KVS_ERR_UNSUPPORTED, "max_kv (%d) is above 2^30", s->max_kv);
    if (s->num_requests > 65535) return ops_fail(KVS_ERR_UNSUPPORTED, "at most 65535 requests in a step");
    if (s->num_requests > 0 && !s->kv_lens) return ops_fail(KVS_ERR_INVALID_ARG, "kv_lens is NULL");
    if (s->num_requests > 0 && s->max_kv > 0 && !s->block_tables) return ops_fail(KVS_ERR_INVALID_ARG, "block_tables is NULL");
    if ((int64_t)s->table_stride * g->block_size < s->max_kv)
        return ops_fail(KVS_ERR_BOUNDS, "tables of %d blocks of %d tokens do not hold max_kv = %d", s->table_stride, g->block_size, s->max_kv);
    const bool no_rows = rowless && s->total_q == 0 && s->max_q == 0;
    if (!s->q_starts && !no_rows && (s->total_q != s->num_requests || (s->num_requests > 0 && s->max_q < 1)))
        return ops_fail(KVS_ERR_INVALID_ARG, "without q_starts a step has one row per request");
    if (s->max_q > s->total_q) return ops_fail(KVS_ERR_INVALID_ARG, "max_q (%d) is above total_q (%d)", s->max_q, s->total_q);
    if (q_heads >= 0 && (q_heads == 0 || q_heads % g->num_kv_heads))
        return ops_fail(KVS_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of the %d kv heads", q_heads, g->num_kv_heads);
    v = StepView{};
    v.tables = s->block_tables;
    v.kv_lens = s->kv_lens;
    v.q_starts = s->q_starts;
    v.requests = s->num_requests;
    v.table_stride = s->table_stride;
    v.total_q = s->total_q;
    v.max_q = s->max_q;
    v.max_kv = s->max_kv;
    v.block_size = g->block_size;
    v.kv_heads = g->num_kv_heads;
    v.head_dim = g->head_dim;
    v.group = q_heads > 0 ? q_heads / g->num_kv_heads : 0;
    set_divisors(v);
    if ((int64_t)s->max_q * (v.group ? v.group : 1) > INT32_MAX / 2)
        return ops_fail(KVS_ERR_UNSUPPORTED, "max_q times the query heads of a KV head is above 2^30");
    return KVS_OK;
}

int cache_of(const kvs_geometry* g, const kvs_paged_cache* c, int32_t layer, int planes, StepView& v) {
    if (!c || !c->kv_planes) return ops_fail(KVS_ERR_INVALID_ARG, "cache or its plane array is NULL");
    if (c->num_blocks <= 0 || c->num_blocks > INT32_MAX) return ops_fail(KVS_ERR_INVALID_ARG, "num_blocks must be in [1, 2^31)");
    if (layer < 0 || layer >= g->num_layers) return ops_fail(KVS_ERR_INVALID_ARG, "layer %d of %d", layer, g->num_layers);
    for (int p = 2 * layer; p < 2 * layer + planes; ++p) {
        if (!c->kv_planes[p]) return ops_fail(KVS_ERR_INVALID_ARG, "plane %d is NULL", p);
        if ((uint64_t)c->kv_planes[p] % 16) return ops_fail(KVS_ERR_UNSUPPORTED, "plane %d is not 16-byte aligned", p);
    }
    v.num_blocks = (int32_t)c->num_blocks;
    return KVS_OK;
}

// The stride of a dimension of one entry means nothing.
int rows_of(const kvs_rows& r, int32_t rows, int32_t heads, const char* name, RowsView& v) {
    if (!r.base) return ops_fail(KVS_ERR_INVALID_ARG, "%s is NULL", name);
    v.base = (char*)r.base;
    v.row = rows > 1 ? r.row_stride : 0;
    v.head = heads > 1 ? r.head_stride : 0;
    if ((uint64_t)r.base % 16 || v.row % 8 || v.head % 8)
        return ops_fail(KVS_ERR_UNSUPPORTED, "%s: address and strides must be multiples of 16 bytes", name);
    if (v.row < 0 || v.head < 0) return ops_fail(KVS_ERR_INVALID_ARG, "%s: negative stride", name);
    return KVS_OK;
}

// Rows that a call writes lie apart: a head's, and a row's heads, behind one another.
int distinct_rows(const kvs_geometry* g, const kvs_rows& r, int32_t heads, int32_t rows, const char* name) {
    const bool heads_in_row = (heads <= 1 || r.head_stride >= g->head_dim) &&
                              (rows <= 1 || r.row_stride >= (int64_t)(heads - 1) * r.head_stride + g->head_dim);
    const bool rows_in_head = (rows <= 1 || r.row_stride >= g->head_dim) &&
                              (heads <= 1 || r.head_stride >= (int64_t)(rows - 1) * r.row_stride + g->head_dim);
    return heads_in_row || rows_in_head ? KVS_OK : ops_fail(KVS_ERR_ALIAS, "%s: rows overlap one another", name);
}

int flags_of(uint32_t flags) {
    return flags & ~KVS_F_VALIDATE ? ops_fail(KVS_ERR_INVALID_ARG, "the only flag is KVS_F_VALIDATE (got 0x%x)", flags) : KVS_OK;
}

// A window that no request's tokens fill hides nothing: 0 then, so that the kernels' sums of
// positions and windows stay in 32 bits.
int mask_of(float scale, int32_t window, const kvs_step* s, int32_t& out) {
    if (!std::isfinite(scale)) return ops_fail(KVS_ERR_INVALID_ARG, "scale is not finite");
    if (window < 0) return ops_fail(KVS_ERR_INVALID_ARG, "window is negative");
    out = window >= s->max_kv ? 0 : window;
    return KVS_OK;
}

// The same with sinks: where the last token of a request of max_kv sees them all, nothing is hidden.
int held_of(float scale, int32_t window, int32_t sinks, const kvs_step* s, int32_t& window_out, int32_t& held, int32_t& sinks_out) {
    KVS_TRY(mask_of(scale, window, s, window_out));
    if (sinks < 0) return ops_fail(KVS_ERR_INVALID_ARG, "sinks is negative");
    if ((int64_t)window + sinks >= s->max_kv) window_out = 0;
    held = window_out > 0;
    sinks_out = held ? sinks : 0;
    return KVS_OK;
}

// After a launcher: its status, its count, and the error word if the caller asked for it.
int done(int launched, cudaStream_t s, uint32_t flags) {
    if (launched < 0) return ops_fail(KVS_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString((cudaError_t)-launched));
    ops_launched(launched);
    return flags & KVS_F_VALIDATE ? ops_read_error(s) : KVS_OK;
}

constexpr float kLog2e = 1.4426950408889634f;

// axes NULL: positions are on one.
int append_call(const kvs_geometry* g, const kvs_paged_cache* c, const kvs_step* st, int32_t layer, const kvs_append_args* a, const kvs_axes* axes,
                cudaStream_t s, uint32_t flags) {
    if (!a) return ops_fail(KVS_ERR_INVALID_ARG, "args is NULL");
    AppendJob j{};
    KVS_TRY(view_of(g, st, a->q.base ? a->num_q_heads : -1, j.step));
    KVS_TRY(cache_of(g, c, layer, 2, j.step));
    KVS_TRY(flags_of(flags));
    if (a->rope) {
        const kvs_rope& r = *a->rope;
        if (r.rot_dim <= 0 || r.rot_dim % 2 || r.rot_dim > g->head_dim)
            return ops_fail(KVS_ERR_INVALID_ARG, "rot_dim must be even and in [2, head_dim] (got %d)", r.rot_dim);
        if (!r.turns) return ops_fail(KVS_ERR_INVALID_ARG, "rope's turns is NULL");
        if ((uint64_t)r.turns % 8) return ops_fail(KVS_ERR_UNSUPPORTED, "rope's turns is not 8-byte aligned");
        if (!std::isfinite(r.scale)) return ops_fail(KVS_ERR_INVALID_ARG, "rope's scale is not finite");
        j.turns = (const float2*)r.turns;
        j.rot_dim = r.rot_dim;
        j.interleaved = r.interleaved != 0;
        j.scale = r.scale;
    }
    if (axes) {
        if (!a->rope) return ops_fail(KVS_ERR_INVALID_ARG, "rope is NULL");
        if (axes->num_axes < 1 || axes->num_axes > KVS_MAX_AXES)
            return ops_fail(KVS_ERR_INVALID_ARG, "num_axes must be in [1, %d] (got %d)", KVS_MAX_AXES, axes->num_axes);
        if (2 * (int64_t)axes->pairs != a->rope->rot_dim)
            return ops_fail(KVS_ERR_INVALID_ARG, "axes of %d pairs, rot_dim is %d", axes->pairs, a->rope->rot_dim);
        if (!axes->axis) return ops_fail(KVS_ERR_INVALID_ARG, "axis is NULL");
        if (axes->num_axes > 1 && axes->stride < st->total_q)
            return ops_fail(KVS_ERR_INVALID_ARG, "axes' stride (%lld) is below total_q (%d)", (long long)axes->stride, st->total_q);
        j.axis = axes->axis;
        j.axes = axes->num_axes;
        j.axis_stride = axes->stride;
    }
    // without a request nothing is read of the step's arrays, which may have no entry
    if (st->total_q == 0 || st->num_requests == 0) return KVS_OK;
    if (axes && !a->positions) return ops_fail(KVS_ERR_INVALID_ARG, "positions is NULL");
    if (a->q.base) {
        KVS_TRY(rows_of(a->q, st->total_q, a->num_q_heads, "q", j.q));
        KVS_TRY(rows_of(a->q_out, st->total_q, a->num_q_heads, "q_out", j.q_out));
        KVS_TRY(distinct_rows(g, a->q_out, a->num_q_heads, st->total_q, "q_out"));
        if (a->q.base == a->q_out.base && (a->q.row_stride != a->q_out.row_stride || a->q.head_stride != a->q_out.head_stride))
            return ops_fail(KVS_ERR_ALIAS, "q_out is q with other strides");
        j.q_heads = a->num_q_heads;
    }
    KVS_TRY(rows_of(a->k, st->total_q, g->num_kv_heads, "k", j.k));
    KVS_TRY(rows_of(a->v, st->total_q, g->num_kv_heads, "v", j.v));
    j.k_plane = (char*)c->kv_planes[2 * layer];
    j.v_plane = (char*)c->kv_planes[2 * layer + 1];
    j.positions = a->positions;
    int sms;
    KVS_TRY(ops_device(&j.step.err, &sms));
    return done(launch_append(j, st->dtype == KVS_DTYPE_F16, s), s, flags);
}

// With sinks a plan goes by the tokens that a CTA's rows may see: the sinks and the window of its tiles'
// tokens, or of all of a request's where few rows share a CTA or nothing is hidden behind a token.
StepView held_view(StepView v, int32_t causal, int32_t window, int32_t sinks, int64_t tokens) {
    const int64_t most = (int64_t)window + sinks + (causal && v.max_q > tokens ? tokens : v.max_q);
    if (most < v.max_kv) v.max_kv = (int32_t)most;
    return v;
}

// Costs in us, fitted to measurements of some sixty steps (in a graph), most of them within a tenth: of a step of 128
// keys and of a CTA's start and end.  8 KV heads of 128 dims, 5 query heads each, a request of 293 new tokens: CTAs that stay and take two row
// tiles at a time 31.7 with a window of 2048, 14.5 with 512; a CTA to a row tile 30.5 and 16.7; two row tiles in
// two parts that their cluster joins 26.7 and 18.6, in three that a second kernel joins 27.9 and 21.6, with a window of 4096 36.6
// against 54.8 where they stay.  35 rows of 64 dims of 16 heads over 1000 tokens: parts of a cluster 8.7 in
// five, 10.1 in four, 16.6 in one.  Blocks of 1 or 12 tokens come by rows, and a step takes as long as those: 293 tokens as above 130 where CTAs stay, 145
// with a CTA to a row tile, 69 in three parts.
AttendPlan held_plan(const StepView& v, int32_t held, int32_t causal, int32_t window, int32_t sinks, int sms) {
    if (!held) return attend_plan(v, sms);
    const int64_t rows = (int64_t)v.max_q * v.group, units = (int64_t)v.kv_heads * v.requests, per = tile_rows_of(v.group);
    if (rows <= 16) {
        // attend_plan's costs of few rows, with what is known of clusters' room by now (four requests with a window of 4096 11.1 us for 12.8)
        const int64_t steps = ((int64_t)held_view(v, causal, window, sinks, v.max_q).max_kv + 127) / 128;
        AttendPlan best{0, 1, 1, 0};
        int64_t least = -1;
        for (int64_t n = 1; n <= 256 && n <= (steps + 1) / 2; ++n) {
            const bool cluster = n > 1 && clusters_fit(units * n, n, sms);
            const int64_t cost = (units * n + sms - 1) / sms * ((steps + n - 1) / n + 4) + (n == 1 ? 0 : cluster ? 1 : 5);
            if (least >= 0 && cost >= least) continue;
            least = cost;
            best = AttendPlan{0, (int)n, 1, cluster};
        }
        return best;
    }
    const bool narrow = v.head_dim <= 64, boxes = v.block_size % 8 == 0 && (128 % v.block_size == 0 || v.block_size % 128 == 0) && v.head_dim >= 64;
    const double step1 = boxes ? (narrow ? 0.95 : 1.17) : narrow ? 3.5 : 7.4, start1 = narrow ? (boxes ? 8.0 : 9.0) : boxes ? 9.0 : 0.5;
    const double step2 = boxes ? 1.43 : narrow ? 5.3 : 6.6, both = boxes && narrow ? 1.6 : step1;        // both: of two CTAs on an SM
    AttendPlan best{1, 1, 1, 0};
    double least = -1.0;
    auto offer = [&](int row_tiles, int64_t parts, int cluster, double cost) {
        if (least >= 0.0 && cost >= least) return;
        least = cost;
        best = AttendPlan{1, (int)parts, row_tiles, cluster};
    };
    for (int rt = 1; rt <= 2; ++rt) {
        const int64_t tiles = (rows + per * rt - 1) / (per * rt) * units, slots = rt == 1 && narrow ? 2 * sms : sms;
        // places of the last sink's block and of the window's first one may be nobody's
        const int64_t block = v.block_size < 128 ? v.block_size : 128;
        const int64_t steps = ((int64_t)held_view(v, causal, window, sinks, per * rt / v.group + 1).max_kv + 2 * block + 125) / 128;
        // one row tile is given to CTAs that stay, too: they start sooner (62 requests of 13 tokens, 2 x 2 heads of 96 dims, a window of
        // 167 9.7 us, 12.2 otherwise)
        const int64_t most = rt == 2 && rows <= per ? 1 : 256;
        for (int64_t n = 1; n <= most && n <= steps; ++n) {
            const int64_t ctas = tiles * n;
            const double each = (double)((steps + n - 1) / n), waves = (double)((ctas + slots - 1) / slots);
            const double alone = waves * ((ctas > sms ? both : step1) * each + start1);
            if (n == 1) offer(rt, 1, 0, rt == 2 ? 5.8 + step2 * each * waves + 3.0 * (waves - 1.0) : alone);
            else if (rt == 1 && clusters_fit(ctas, n, sms)) offer(1, n, 1, step1 * each + start1 + (narrow ? 1.0 : 2.4) * (rows < per ? (double)rows / per : 1.0));
            else if (rt == 1 && n <= kCluster && ctas <= slots - 5 * (n - 1)) offer(1, n, 1, boxes ? 1.1 * each + 11.5 : step1 * each + 2.0);
            else if (rt == 2 && n <= kClusterPairs && clusters_fit(ctas, n, sms)) offer(2, n, 1, step2 * each + 13.5);
            else if (n <= (steps + 1) / 2) offer(rt, n, 0, rt == 2 ? waves * (step2 * each + 7.0) + 12.0 : alone + 4.0 + 0.02 * n);
        }
    }
    return best;
}

int64_t pairs_of_tiles(const StepView& v) {
    const int64_t rows = 2 * tile_rows_of(v.group);
    return ((int64_t)v.max_q * v.group + rows - 1) / rows * v.kv_heads * v.requests;
}

int64_t workspace_bytes(const StepView& v, const AttendPlan& plan) {
    const int n = plan.splits;
    return n <= 1 || plan.cluster ? 0 : (int64_t)n * v.total_q * v.kv_heads * v.group * (v.head_dim + 2) * 4;
}

int attend_call(const kvs_geometry* g, const kvs_paged_cache* c, const kvs_step* st, int32_t layer, const kvs_attend_args* a, const int32_t* sinks,
                cudaStream_t s, uint32_t flags) {
    if (!a) return ops_fail(KVS_ERR_INVALID_ARG, "args is NULL");
    AttendJob j{};
    KVS_TRY(view_of(g, st, a->num_q_heads, j.step));
    KVS_TRY(cache_of(g, c, layer, 2, j.step));
    KVS_TRY(flags_of(flags));
    if (sinks) KVS_TRY(held_of(a->scale, a->window, *sinks, st, j.window, j.held, j.sinks));
    else KVS_TRY(mask_of(a->scale, a->window, st, j.window));
    if (st->total_q == 0 || st->num_requests == 0) return KVS_OK;
    KVS_TRY(rows_of(a->q, st->total_q, a->num_q_heads, "q", j.q));
    KVS_TRY(rows_of(a->out, st->total_q, a->num_q_heads, "out", j.out));
    KVS_TRY(distinct_rows(g, a->out, a->num_q_heads, st->total_q, "out"));
    j.k_plane = (const char*)c->kv_planes[2 * layer];
    j.v_plane = (const char*)c->kv_planes[2 * layer + 1];
    j.lse = a->lse;
    j.causal = a->causal != 0;
    int sms;
    KVS_TRY(ops_device(&j.step.err, &sms));
    const AttendPlan plan = held_plan(j.step, j.held, j.causal, j.window, j.sinks, sms);
    // With sinks lse is of the scale as given, as kvs_weigh_sinks takes it.  On the tensor cores' kernels what one binary32 number lacks is
    // added to the maximum at the end; the others multiply every score by both.
    j.scale_log2 = j.held && !plan.tc ? scale_cut(a->scale) : a->scale * kLog2e;
    if (j.held) j.scale_low = scale_rest(a->scale, j.scale_log2);
    j.tc = plan.tc;
    j.splits = plan.splits;
    j.cluster = plan.cluster;
    j.row_tiles = plan.row_tiles;
    j.stay = j.held && plan.tc && plan.splits == 1 && plan.row_tiles == 2 && pairs_of_tiles(j.step) <= INT32_MAX ? sms : 0;
    const int64_t need = workspace_bytes(j.step, plan);
    if (need > 0) {
        if (!a->workspace) return ops_fail(KVS_ERR_INVALID_ARG, "workspace is NULL, %lld bytes are needed", (long long)need);
        if (a->workspace_bytes < need)
            return ops_fail(KVS_ERR_BOUNDS, "workspace of %lld bytes, %lld are needed", (long long)a->workspace_bytes, (long long)need);
        if ((uint64_t)a->workspace % 16) return ops_fail(KVS_ERR_UNSUPPORTED, "workspace is not 16-byte aligned");
        j.partial = (float*)a->workspace;
    }
    return done(launch_attend(j, st->dtype == KVS_DTYPE_F16, s), s, flags);
}

int weigh_call(const kvs_geometry* g, const kvs_paged_cache* c, const kvs_step* st, int32_t layer, const kvs_weigh_args* a, const int32_t* sinks,
               cudaStream_t s, uint32_t flags) {
    if (!a) return ops_fail(KVS_ERR_INVALID_ARG, "args is NULL");
    WeighJob j{};
    KVS_TRY(view_of(g, st, a->num_q_heads, j.step));
    KVS_TRY(cache_of(g, c, layer, 1, j.step));
    KVS_TRY(flags_of(flags));
    if (sinks) KVS_TRY(held_of(a->scale, a->window, *sinks, st, j.window, j.held, j.sinks));
    else KVS_TRY(mask_of(a->scale, a->window, st, j.window));
    if (!std::isfinite(a->decay)) return ops_fail(KVS_ERR_INVALID_ARG, "decay is not finite");
    if (st->num_requests == 0 || st->max_kv == 0) return KVS_OK;
    if (!a->weights) return ops_fail(KVS_ERR_INVALID_ARG, "weights is NULL");
    if (st->total_q > 0) {
        if (!a->lse) return ops_fail(KVS_ERR_INVALID_ARG, "lse is NULL");
        KVS_TRY(rows_of(a->q, st->total_q, a->num_q_heads, "q", j.q));
    }
    const int64_t hs = a->head_stride, rs = a->request_stride, T = st->max_kv, H = g->num_kv_heads, R = st->num_requests;
    if (hs < 0 || rs < 0) return ops_fail(KVS_ERR_INVALID_ARG, "weights: negative stride");
    if (!(((H == 1 || hs >= T) && (R == 1 || rs >= (H - 1) * hs + T)) || ((R == 1 || rs >= T) && (H == 1 || hs >= (R - 1) * rs + T))))
        return ops_fail(KVS_ERR_ALIAS, "weights: rows of max_kv = %lld overlap one another", (long long)T);
    j.k_plane = (const char*)c->kv_planes[2 * layer];
    j.lse = a->lse;
    j.weights = a->weights;
    j.request_stride = rs;
    j.head_stride = hs;
    j.scale_log2 = a->scale * kLog2e;
    j.decay = a->decay;
    j.scale = a->scale;
    j.by_places = sinks != nullptr;
    j.causal = a->causal != 0;
    int sms;
    KVS_TRY(ops_device(&j.step.err, &sms));
    return done(launch_weigh(j, st->dtype == KVS_DTYPE_F16, sms, s), s, flags);
}

int evict_call(const kvs_geometry* g, const kvs_paged_cache* c, const kvs_step* st, const kvs_evict_args* a, cudaStream_t s, uint32_t flags) {
    if (!a) return ops_fail(KVS_ERR_INVALID_ARG, "args is NULL");
    EvictJob j{};
    KVS_TRY(view_of(g, st, -1, j.step, true));
    KVS_TRY(cache_of(g, c, 0, 2 * g->num_layers, j.step));
    KVS_TRY(flags_of(flags));
    if (a->budget < 1) return ops_fail(KVS_ERR_INVALID_ARG, "budget must be positive");
    if (a->budget > 1 << 30) return ops_fail(KVS_ERR_UNSUPPORTED, "budget (%d) is above 2^30", a->budget);
    if (a->sinks < 0 || a->recent < 0 || (int64_t)a->sinks + a->recent > a->budget)
        return ops_fail(KVS_ERR_INVALID_ARG, "sinks (%d) and recent (%d) must fit the budget (%d)", a->sinks, a->recent, a->budget);
    if (a->layer_stride < 0 || a->request_stride < 0 || a->head_stride < 0)
        return ops_fail(KVS_ERR_INVALID_ARG, "weights: negative stride");
    if (st->num_requests == 0) return KVS_OK;
    const int32_t most = st->max_kv < a->budget ? st->max_kv : a->budget;
    if (st->max_kv > 0 && !a->weights) return ops_fail(KVS_ERR_INVALID_ARG, "weights is NULL");
    if (!a->kept) return ops_fail(KVS_ERR_INVALID_ARG, "kept is NULL");
    if (most > 0 && !a->dst_tables) return ops_fail(KVS_ERR_INVALID_ARG, "dst_tables is NULL");
    if (a->dst_stride < 0 || (int64_t)a->dst_stride * g->block_size < most)
        return ops_fail(KVS_ERR_BOUNDS, "new tables of %d blocks of %d tokens do not hold %d", a->dst_stride, g->block_size, most);
    if (a->dst_tables == st->block_tables && most > 0) return ops_fail(KVS_ERR_ALIAS, "the new blocks are the old ones");
    if (a->new_lens == st->kv_lens) return ops_fail(KVS_ERR_ALIAS, "new_lens is kv_lens");
    if (a->new_weights && a->new_weights == a->weights) return ops_fail(KVS_ERR_ALIAS, "new_weights is weights");
    j.planes = c->kv_planes;
    j.layers = g->num_layers;
    j.weights = a->weights;
    j.layer_stride = a->layer_stride;
    j.request_stride = a->request_stride;
    j.head_stride = a->head_stride;
    j.dst_tables = a->dst_tables;
    j.dst_stride = a->dst_stride;
    j.budget = a->budget;
    j.sinks = a->sinks;
    j.recent = a->recent;
    j.kept = a->kept;
    j.new_weights = a->new_weights;
    j.new_lens = a->new_lens;
    int sms;
    KVS_TRY(ops_device(&j.step.err, &sms));
    return done(launch_evict(j, s), s, flags);
}

int rope_turns(const kvs_rope_spec* sp, float* out, float* scale) {
    if (!sp || !out || !scale) return ops_fail(KVS_ERR_INVALID_ARG, "spec, turns_out or scale_out is NULL");
    if (sp->rot_dim <= 0 || sp->rot_dim % 2) return ops_fail(KVS_ERR_INVALID_ARG, "rot_dim must be even and positive");
    if (sp->kind < KVS_ROPE_PLAIN || sp->kind > KVS_ROPE_YARN) return ops_fail(KVS_ERR_INVALID_ARG, "unknown kind %d", sp->kind);
    if (!(sp->base > 1.0) || !std::isfinite(sp->base)) return ops_fail(KVS_ERR_INVALID_ARG, "base must be above 1");
    if (sp->kind != KVS_ROPE_PLAIN && (!(sp->factor >= 1.0) || !std::isfinite(sp->factor)))
        return ops_fail(KVS_ERR_INVALID_ARG, "factor must be at least 1");
    const bool ranged = sp->kind == KVS_ROPE_BANDS || sp->kind == KVS_ROPE_YARN;
    if (ranged && !(sp->context > 0.0 && sp->low > 0.0 && sp->high > sp->low && std::isfinite(sp->high) && std::isfinite(sp->context)))
        return ops_fail(KVS_ERR_INVALID_ARG, "context must be positive and 0 < low < high");
    if (sp->kind == KVS_ROPE_NTK && sp->rot_dim == 2) return ops_fail(KVS_ERR_INVALID_ARG, "KVS_ROPE_NTK needs a rot_dim above 2");
    const double two_pi = 6.283185307179586476925286766559;
    const int n = sp->rot_dim / 2;
    const double rot = sp->rot_dim;
    const double base = sp->kind == KVS_ROPE_NTK ? sp->base * std::pow(sp->factor, rot / (rot - 2.0)) : sp->base;
    // Pair index (not whole) that turns `times` times within the context.
    auto index_of = [&](double times) { return rot * std::log(sp->context / (times * two_pi)) / (2.0 * std::log(base)); };
    double first = 0.0, last = 0.0;
    if (sp->kind == KVS_ROPE_YARN) {
        first = std::fmax(0.0, std::floor(index_of(sp->high)));
        last = std::fmin(rot - 1.0, std::ceil(index_of(sp->low)));
        if (last <= first) last = first + 0.001;
    }
    for (int k = 0; k < n; ++k) {
        double f = std::pow(base, -2.0 * k / rot);             // radians per position
        if (sp->kind == KVS_ROPE_LINEAR) f /= sp->factor;
        if (sp->kind == KVS_ROPE_BANDS) {
            const double ratio = sp->context * f / two_pi;     // context / wavelength
            const double mean = std::fmin(1.0, std::fmax(0.0, (ratio - sp->low) / (sp->high - sp->low)));
            f = (1.0 - mean) * f / sp->factor + mean * f;
        }
        if (sp->kind == KVS_ROPE_YARN) {
            const double ramp = std::fmin(1.0, std::fmax(0.0, (k - first) / (last - first)));
            f = ramp * f / sp->factor + (1.0 - ramp) * f;
        }
        f /= two_pi;
        out[2 * k] = (float)f;
        out[2 * k + 1] = (float)(f - (double)out[2 * k]);
    }
    *scale = sp->kind == KVS_ROPE_YARN ? (float)(0.1 * std::log(sp->factor) + 1.0) : 1.0f;
    return KVS_OK;
}

int rope_axes(const kvs_rope_spec* sp, const int32_t* parts, int32_t n, int32_t order, float* turns, uint8_t* axis, float* scale) {
    if (!sp || !parts || !turns || !axis || !scale) return ops_fail(KVS_ERR_INVALID_ARG, "spec, parts, turns_out, axis_out or scale_out is NULL");
    if (n < 1 || n > KVS_MAX_AXES) return ops_fail(KVS_ERR_INVALID_ARG, "num_axes must be in [1, %d] (got %d)", KVS_MAX_AXES, n);
    if (order & ~(KVS_AXES_CYCLE | KVS_AXES_RESTART)) return ops_fail(KVS_ERR_INVALID_ARG, "unknown order %d", order);
    int64_t pairs = 0;
    for (int a = 0; a < n; ++a) {
        if (parts[a] < 1) return ops_fail(KVS_ERR_INVALID_ARG, "axis %d has %d pairs", a, parts[a]);
        pairs += parts[a];
    }
    if (sp->rot_dim != 2 * pairs) return ops_fail(KVS_ERR_INVALID_ARG, "rot_dim (%d) is not twice the %lld pairs", sp->rot_dim, (long long)pairs);
    const bool cycle = order & KVS_AXES_CYCLE;
    for (int a = 1; cycle && a < n; ++a)
        if (a + (int64_t)n * (parts[a] - 1) >= pairs) return ops_fail(KVS_ERR_INVALID_ARG, "axis %d has no turn for %d pairs", a, parts[a]);
    KVS_TRY(rope_turns(sp, turns, scale));
    int64_t k = 0;
    for (int a = 0; a < n; ++a)
        for (int32_t m = 0; m < parts[a]; ++m) axis[k++] = cycle ? 0 : (uint8_t)a;
    for (int a = 1; cycle && a < n; ++a)
        for (int64_t m = 0; m < parts[a]; ++m) axis[a + n * m] = (uint8_t)a;
    if (!(order & KVS_AXES_RESTART)) return KVS_OK;
    // each axis's own table, of which its pairs take the entries in turn
    std::vector<float> own;
    for (int a = 0; a < n; ++a) {
        kvs_rope_spec one = *sp;
        one.rot_dim = 2 * parts[a];
        own.resize(2 * (size_t)parts[a]);
        KVS_TRY(rope_turns(&one, own.data(), scale));
        for (int64_t k = 0, at = 0; k < pairs; ++k) {
            if (axis[k] != a) continue;
            turns[2 * k] = own[2 * at];
            turns[2 * k + 1] = own[2 * at + 1];
            ++at;
        }
    }
    return KVS_OK;
}

}  // namespace
}  // namespace kvs

using namespace kvs;

extern "C" {

int kvs_rope_turns(const kvs_rope_spec* spec, float* turns_out, float* scale_out) {
    return entry([&] { return rope_turns(spec, turns_out, scale_out); });
}

int kvs_rope_axes(const kvs_rope_spec* spec, const int32_t* parts, int32_t num_axes, int32_t order, float* turns_out,
                  uint8_t* axis_out, float* scale_out) {
    return entry([&] { return rope_axes(spec, parts, num_axes, order, turns_out, axis_out, scale_out); });
}

int kvs_append(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
               const kvs_append_args* args, void* cuda_stream, uint32_t flags) {
    return entry([&] { return append_call(geom, cache, step, layer, args, nullptr, (cudaStream_t)cuda_stream, flags); });
}

int kvs_append_axes(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
                    const kvs_append_args* args, const kvs_axes* axes, void* cuda_stream, uint32_t flags) {
    return entry([&] {
        if (!axes) return ops_fail(KVS_ERR_INVALID_ARG, "axes is NULL");
        return append_call(geom, cache, step, layer, args, axes, (cudaStream_t)cuda_stream, flags);
    });
}

int kvs_attend(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
               const kvs_attend_args* args, void* cuda_stream, uint32_t flags) {
    return entry([&] { return attend_call(geom, cache, step, layer, args, nullptr, (cudaStream_t)cuda_stream, flags); });
}

int kvs_attend_sinks(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
                     const kvs_attend_args* args, int32_t sinks, void* cuda_stream, uint32_t flags) {
    return entry([&] { return attend_call(geom, cache, step, layer, args, &sinks, (cudaStream_t)cuda_stream, flags); });
}

int64_t kvs_attend_workspace(const kvs_geometry* geom, const kvs_step* step, int32_t num_q_heads) {
    int64_t bytes = 0;
    const int rc = entry([&] {
        StepView v;
        KVS_TRY(view_of(geom, step, num_q_heads, v));
        int32_t* err;
        int sms;
        KVS_TRY(ops_device(&err, &sms));
        bytes = workspace_bytes(v, attend_plan(v, sms));
        return (int)KVS_OK;
    });
    return rc ? rc : bytes;
}

int64_t kvs_attend_sinks_workspace(const kvs_geometry* geom, const kvs_step* step, int32_t num_q_heads, int32_t causal,
                                   int32_t window, int32_t sinks) {
    int64_t bytes = 0;
    const int rc = entry([&] {
        StepView v;
        int32_t held = 0;
        KVS_TRY(view_of(geom, step, num_q_heads, v));
        KVS_TRY(held_of(1.0f, window, sinks, step, window, held, sinks));
        int32_t* err;
        int sms;
        KVS_TRY(ops_device(&err, &sms));
        bytes = workspace_bytes(v, held_plan(v, held, causal, window, sinks, sms));
        return (int)KVS_OK;
    });
    return rc ? rc : bytes;
}

int kvs_weigh(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
              const kvs_weigh_args* args, void* cuda_stream, uint32_t flags) {
    return entry([&] { return weigh_call(geom, cache, step, layer, args, nullptr, (cudaStream_t)cuda_stream, flags); });
}

int kvs_weigh_sinks(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step, int32_t layer,
                    const kvs_weigh_args* args, int32_t sinks, void* cuda_stream, uint32_t flags) {
    return entry([&] { return weigh_call(geom, cache, step, layer, args, &sinks, (cudaStream_t)cuda_stream, flags); });
}

int kvs_evict(const kvs_geometry* geom, const kvs_paged_cache* cache, const kvs_step* step,
              const kvs_evict_args* args, void* cuda_stream, uint32_t flags) {
    return entry([&] { return evict_call(geom, cache, step, args, (cudaStream_t)cuda_stream, flags); });
}

}  // extern "C"
