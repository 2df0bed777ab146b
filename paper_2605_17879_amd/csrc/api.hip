// Host side of the C ABI declared in guard.h: configuration checks, the layout
// of the caller's state buffer, argument validation and the kernel launches.
// No device memory is allocated here and no call synchronises.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>
#include <string>

#include "../../include/guard.h"
#include "gd_internal.h"
#include "gd_operators.h"

struct gd_handle_s {
    gd_config cfg;
    uint32_t N, RW, NW;
    gd_state_layout lay;
    uint8_t* d_state;
    uint32_t split_steps;
    const float* hint_med;
    const float* hint_mad;
    gd_ledger_config lcfg;
    gd_ledger_layout llay;
    uint8_t* d_led;
    uint32_t led_max_T;
    std::string err;
};

namespace {

std::string g_create_error;

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

gd_state_layout make_layout(uint32_t R, uint32_t N, uint32_t W) {
    const size_t RW = (R + 63) / 64, NW = (N + 63) / 64;
    gd_state_layout l;
    size_t o = 0;
    l.rank_ring = o;   o = align256(o + (size_t)W * RW * 8);
    l.node_ring = o;   o = align256(o + (size_t)W * NW * 8);
    l.rank_count = o;  o = align256(o + (size_t)R * 2);
    l.node_count = o;  o = align256(o + (size_t)N * 2);
    l.rank_first = o;  o = align256(o + (size_t)R * 4);
    l.node_first = o;  o = align256(o + (size_t)N * 4);
    l.node_z_last = o; o = align256(o + (size_t)N * 4);
    l.total = o;
    return l;
}

gd_ledger_layout make_ledger_layout(uint32_t R, uint32_t N, uint32_t W, uint32_t max_T) {
    const size_t NW = (N + 63) / 64;
    gd_ledger_layout l;
    size_t o = 0;
    l.head = o;        o = align256(o + 32);
    l.rank_ring = o;   o = align256(o + (size_t)W * R);
    l.node_ring = o;   o = align256(o + (size_t)W * N);
    l.rank_cnt = o;    o = align256(o + (size_t)R * 16);
    l.node_cnt = o;    o = align256(o + (size_t)N * 16);
    l.node_ccnt = o;   o = align256(o + (size_t)N * 2);
    l.counts_bytes = o - l.rank_cnt;
    l.counts_new = o;  o += l.counts_bytes;
    l.rank_first = o;  o = align256(o + (size_t)R * 4);
    l.node_first = o;  o = align256(o + (size_t)N * 4);
    l.node_qring = o;  o = align256(o + (size_t)W * N * 2);
    l.node_qsum = o;   o = align256(o + (size_t)N * 4);
    l.node_starts = o; o = align256(o + (size_t)N * 32);
    l.node_term = o;   o = align256(o + (size_t)N * 4);
    l.rise = o;        o = align256(o + (size_t)max_T * NW * 8);
    l.total = o;
    return l;
}

gd_status fail(gd_handle h, gd_status st, const std::string& msg) {
    if (h) h->err = msg; else g_create_error = msg;
    return st;
}

gd_status hip_fail(gd_handle h, hipError_t e, const char* what) {
    return fail(h, GD_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// ---- arguments of the operators of a training step ----

// Rows are addressed by 32-bit byte offsets from a tile's first one.
constexpr uint64_t MAX_STRIDE = 1u << 22;

uint32_t bytes_of(uint32_t type) { return type == GD_F32 || type == GD_I32 ? 4 : type == GD_I64 ? 8 : type == GD_E4M3 ? 1 : 2; }
bool is_float(uint32_t type) { return type == GD_F32 || type == GD_BF16 || type == GD_F16; }

// What is wrong with a matrix of rows x cols elements, or null.
const char* bad_matrix(const gd_matrix* m, uint64_t rows, uint64_t cols) {
    if (!m) return "null matrix";
    if (m->reserved != 0) return "reserved field of a matrix is not 0";
    if (m->rows != rows || m->cols != cols) return "sizes of the matrices do not fit each other";
    if (rows == 0 || cols == 0) return nullptr;
    if (!m->d_data) return "null pointer of a matrix";
    if (m->stride < cols) return "stride below the row's length";
    if (m->stride > MAX_STRIDE && cols > 1) return "stride above 2^22 elements";
    if (m->stride > (1ull << 40)) return "stride above 2^40 elements";
    if ((uintptr_t)m->d_data % bytes_of(m->dtype)) return "pointer of a matrix not aligned to its element";
    return nullptr;
}

// The same for a list of tokens or targets.
const char* bad_tokens(const gd_matrix* m) {
    if (!m) return "null matrix";
    if (m->dtype != GD_I32 && m->dtype != GD_I64) return "tokens must be i32 or i64";
    if (m->cols != 1) return "tokens must have one column";
    if (m->rows > GD_MAX_TOKENS) return "more than 2^24 tokens";
    return bad_matrix(m, m->rows, 1);
}

gd_token_list tokens_of(const gd_matrix* m) {
    return gd_token_list{m->d_data, m->stride, (uint32_t)m->rows, m->dtype == GD_I64 ? 1u : 0u};
}

gd_status invalid(gd_handle h, const char* call, const char* what) {
    return fail(h, GD_ERR_INVALID_ARG, std::string(call) + ": " + what);
}

// The work area of a call that needs one.
gd_status bad_work(gd_handle h, const char* call, const void* d_work, size_t have, size_t need) {
    if (need && !d_work) return invalid(h, call, "null work area");
    if ((uintptr_t)d_work & 255) return invalid(h, call, "work area not 256-byte aligned");
    if (have < need) return fail(h, GD_ERR_BUFFER_TOO_SMALL, std::string(call) + ": work area too small");
    return GD_OK;
}

// Sizes and types of a projection onto a vocabulary, or what is wrong with them.
const char* bad_projection(const gd_matrix* hidden, const gd_matrix* weight, const gd_matrix* targets) {
    if (const char* e = bad_tokens(targets)) return e;
    if (!hidden || !weight) return "null matrix";
    if (hidden->dtype != weight->dtype) return "hidden and weight differ in type";
    if (weight->rows == 0 || weight->cols == 0) return "weight has no elements";
    if (weight->rows > GD_MAX_VOCAB) return "vocabulary above 2^24 rows";
    if (weight->cols > GD_MAX_WIDTH) return "width above 65536";
    if (const char* e = bad_matrix(weight, weight->rows, weight->cols)) return e;
    return bad_matrix(hidden, targets->rows, weight->cols);
}

// What is wrong with one tensor of an update, or null.
const char* bad_tensor(const gd_adamw_tensor& t) {
    if (!is_float(t.param_type) || !is_float(t.grad_type)) return "param and grad must be f32, bf16 or f16";
    if (t.state_type != GD_F32 && t.state_type != GD_E4M3) return "states must be f32 or e4m3";
    if (t.d_copy && t.copy_type != GD_BF16 && t.copy_type != GD_F16) return "a copy must be bf16 or f16";
    if (!(isfinite(t.lr_scale) && isfinite(t.weight_decay))) return "lr_scale and weight_decay must be finite";
    if (t.n > (1ull << 42)) return "tensor of more than 2^42 elements";
    if (t.n == 0) return nullptr;
    if (!t.d_param || !t.d_grad || !t.d_m || !t.d_v) return "null pointer of a tensor";
    if (t.state_type == GD_E4M3 && (!t.d_m_exp || !t.d_v_exp)) return "8-bit states need their exponents";
    const uint32_t state = bytes_of(t.state_type);
    if ((uintptr_t)t.d_param % bytes_of(t.param_type) || (uintptr_t)t.d_grad % bytes_of(t.grad_type) ||
        (uintptr_t)t.d_m % state || (uintptr_t)t.d_v % state || (uintptr_t)t.d_copy % 2)
        return "pointer of a tensor not aligned to its element";
    return nullptr;
}

const char* bad_tensors(const gd_adamw_tensor* t, uint32_t n) {
    if (n && !t) return "null list of tensors";
    for (uint32_t i = 0; i < n; ++i)
        if (const char* e = bad_tensor(t[i])) return e;
    return nullptr;
}

}  // namespace

extern "C" {

void gd_default_config(gd_config* c, uint32_t n_ranks, uint32_t n_metrics, uint32_t window,
                       uint32_t persist_k) {
    if (!c) return;
    memset(c, 0, sizeof(*c));
    c->struct_size = (uint32_t)sizeof(gd_config);
    c->n_ranks = n_ranks;
    c->gpus_per_node = 8;
    c->n_metrics = n_metrics;
    c->primary_metric = 0;
    c->min_signals = n_metrics < 2 ? n_metrics : 2;
    c->window = window;
    c->persist_k = persist_k;
    const uint32_t N = n_ranks / 8;
    c->topk = N < 64 ? N : 64;
    c->node_agg = GD_NODE_SUM_SCALED;
    c->z_threshold = 3.5f;
    c->node_scale = 0.35355338f;   // 1/sqrt(8)
    c->rel_floor = 1e-6f;
    c->abs_floor = 1e-30f;
    for (int i = 0; i < GD_MAX_METRICS; ++i) c->direction[i] = 1;
}

gd_status gd_create(const gd_config* c, gd_handle* out) {
    if (out) *out = nullptr;
    if (!c || !out) return fail(nullptr, GD_ERR_INVALID_ARG, "gd_create: null argument");
    if (c->struct_size != sizeof(gd_config))
        return fail(nullptr, GD_ERR_BAD_CONFIG, "struct_size does not match this library's gd_config");
    if (c->gpus_per_node != 8)
        return fail(nullptr, GD_ERR_UNSUPPORTED, "only gpus_per_node = 8 is built");
    if (c->n_ranks < 8 || c->n_ranks % 8 != 0)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "n_ranks must be a positive multiple of gpus_per_node");
    if (c->n_ranks > GD_MAX_RANKS)
        return fail(nullptr, GD_ERR_UNSUPPORTED, "n_ranks above 65536 is not built");
    if (c->n_metrics < 1 || c->n_metrics > GD_MAX_METRICS)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "n_metrics must be 1..8");
    if (c->primary_metric >= c->n_metrics)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "primary_metric out of range");
    if (c->min_signals < 1 || c->min_signals > c->n_metrics)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "min_signals must be 1..n_metrics");
    if (c->window < 1 || c->window > GD_MAX_WINDOW)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "window must be 1..1024");
    if (c->persist_k < 1 || c->persist_k > c->window)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "persist_k must be 1..window");
    const uint32_t N = c->n_ranks / 8;
    if (c->topk > N) return fail(nullptr, GD_ERR_BAD_CONFIG, "topk exceeds the number of nodes");
    if (c->node_agg != GD_NODE_SUM_SCALED && c->node_agg != GD_NODE_MAX)
        return fail(nullptr, GD_ERR_BAD_CONFIG, "unknown node_agg");
    if (!isfinite(c->z_threshold) || !isfinite(c->node_scale) || !(c->rel_floor >= 0.0f) ||
        !(c->abs_floor > 0.0f) || !isfinite(c->rel_floor) || !isfinite(c->abs_floor))
        return fail(nullptr, GD_ERR_BAD_CONFIG,
                    "threshold and node_scale must be finite, rel_floor >= 0, abs_floor > 0");
    for (uint32_t m = 0; m < c->n_metrics; ++m)
        if (c->direction[m] < -1 || c->direction[m] > 1)
            return fail(nullptr, GD_ERR_BAD_CONFIG, "direction must be -1, 0 or +1");
    gd_handle h = new (std::nothrow) gd_handle_s();
    if (!h) return fail(nullptr, GD_ERR_INVALID_ARG, "out of host memory");
    h->cfg = *c;
    h->N = N;
    h->RW = (c->n_ranks + 63) / 64;
    h->NW = (N + 63) / 64;
    h->lay = make_layout(c->n_ranks, N, c->window);
    h->d_state = nullptr;
    h->split_steps = GD_DEFAULT_STREAMING_STEPS;
    h->hint_med = nullptr;
    h->hint_mad = nullptr;
    h->d_led = nullptr;
    h->led_max_T = 0;
    *out = h;
    return GD_OK;
}

gd_status gd_destroy(gd_handle h) {
    delete h;
    return GD_OK;
}

gd_status gd_set_streaming_steps(gd_handle h, uint32_t max_steps) {
    if (!h) return GD_ERR_INVALID_ARG;
    h->split_steps = max_steps;
    return GD_OK;
}

gd_status gd_set_streaming_hints(gd_handle h, const float* d_med, const float* d_mad) {
    if (!h) return GD_ERR_INVALID_ARG;
    if ((d_med == nullptr) != (d_mad == nullptr))
        return fail(h, GD_ERR_INVALID_ARG, "gd_set_streaming_hints: give both arrays or neither");
    if (((uintptr_t)d_med & 3) || ((uintptr_t)d_mad & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_set_streaming_hints: misaligned pointer");
    h->hint_med = d_med;
    h->hint_mad = d_mad;
    return GD_OK;
}

size_t gd_state_bytes(gd_handle h) { return h ? h->lay.total : 0; }

gd_status gd_bind_state(gd_handle h, void* d_state, size_t state_bytes) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!d_state) return fail(h, GD_ERR_INVALID_ARG, "gd_bind_state: null state");
    if (((uintptr_t)d_state & 255) != 0)
        return fail(h, GD_ERR_INVALID_ARG, "gd_bind_state: state must be 256-byte aligned");
    if (state_bytes < h->lay.total)
        return fail(h, GD_ERR_BUFFER_TOO_SMALL, "gd_bind_state: buffer smaller than gd_state_bytes");
    h->d_state = static_cast<uint8_t*>(d_state);
    return GD_OK;
}

gd_status gd_score_batch(gd_handle h, const float* d_x, uint32_t T, float* d_med, float* d_mad,
                         float* d_z, uint8_t* d_exceed_mask, uint64_t* d_rank_anom,
                         float* d_node_z, uint8_t* d_node_mask, uint64_t* d_node_anom,
                         void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (T == 0) return GD_OK;
    if (!d_x || !d_med || !d_mad || !d_exceed_mask || !d_rank_anom || !d_node_z || !d_node_mask ||
        !d_node_anom)
        return fail(h, GD_ERR_INVALID_ARG, "gd_score_batch: a required pointer is null");
    if (((uintptr_t)d_x & 15) || ((uintptr_t)d_z & 15) || ((uintptr_t)d_exceed_mask & 3) ||
        ((uintptr_t)d_rank_anom & 7) || ((uintptr_t)d_node_anom & 7) || ((uintptr_t)d_node_z & 3) ||
        ((uintptr_t)d_med & 3) || ((uintptr_t)d_mad & 3))
        return fail(h, GD_ERR_INVALID_ARG,
                    "gd_score_batch: x and z must be 16-byte aligned, the other arrays naturally aligned");
    gd_score_args a;
    a.x = d_x; a.med = d_med; a.mad = d_mad; a.z = d_z;
    a.exceed_mask = d_exceed_mask; a.rank_anom = d_rank_anom;
    a.node_z = d_node_z; a.node_mask = d_node_mask; a.node_anom = d_node_anom;
    a.T = T; a.R = h->cfg.n_ranks; a.M = h->cfg.n_metrics; a.N = h->N;
    a.primary = h->cfg.primary_metric; a.min_signals = h->cfg.min_signals;
    a.node_agg = h->cfg.node_agg;
    a.split_steps = h->split_steps;
    a.hint_med = h->hint_med; a.hint_mad = h->hint_mad;
    // (a threshold of -0 is one of +0: the kernels tell "greater" by the sign of thr less the score)
    a.thr = h->cfg.z_threshold + 0.0f; a.node_scale = h->cfg.node_scale;
    a.rel_floor = h->cfg.rel_floor; a.abs_floor = h->cfg.abs_floor;
    memcpy(a.dir, h->cfg.direction, 8);
    hipError_t e = gd_launch_score(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_score_batch");
    return GD_OK;
}

gd_status gd_update_window(gd_handle h, const uint64_t* d_rank_anom, const uint64_t* d_node_anom,
                           const float* d_node_z, uint32_t T, uint64_t first_step_index,
                           void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_state) return fail(h, GD_ERR_INVALID_ARG, "gd_update_window: no state bound");
    if (T == 0) return GD_OK;
    if (!d_rank_anom || !d_node_anom || !d_node_z)
        return fail(h, GD_ERR_INVALID_ARG, "gd_update_window: a required pointer is null");
    if (((uintptr_t)d_rank_anom & 7) || ((uintptr_t)d_node_anom & 7) || ((uintptr_t)d_node_z & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_update_window: misaligned pointer");
    if (first_step_index + (uint64_t)T > 0x7FFFFFFFull)
        return fail(h, GD_ERR_INVALID_ARG, "gd_update_window: step index beyond 2^31 - 1");
    gd_window_args a;
    a.state = h->d_state; a.lay = h->lay;
    a.rank_anom = d_rank_anom; a.node_anom = d_node_anom; a.node_z = d_node_z;
    a.T = T; a.R = h->cfg.n_ranks; a.N = h->N; a.W = h->cfg.window; a.K = h->cfg.persist_k;
    a.first_step = first_step_index;
    hipError_t e = gd_launch_window(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_update_window");
    return GD_OK;
}

gd_status gd_flags(gd_handle h, uint8_t* d_rank_flag, uint16_t* d_rank_count,
                   int32_t* d_rank_first, uint8_t* d_node_flag, uint16_t* d_node_count,
                   int32_t* d_node_first, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_state) return fail(h, GD_ERR_INVALID_ARG, "gd_flags: no state bound");
    if (((uintptr_t)d_rank_count & 1) || ((uintptr_t)d_node_count & 1) ||
        ((uintptr_t)d_rank_first & 3) || ((uintptr_t)d_node_first & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_flags: misaligned pointer");
    gd_flags_args a;
    a.state = h->d_state; a.lay = h->lay;
    a.rank_flag = d_rank_flag; a.rank_count = d_rank_count; a.rank_first = d_rank_first;
    a.node_flag = d_node_flag; a.node_count = d_node_count; a.node_first = d_node_first;
    a.R = h->cfg.n_ranks; a.N = h->N; a.K = h->cfg.persist_k;
    hipError_t e = gd_launch_flags(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_flags");
    return GD_OK;
}

gd_status gd_topk_nodes(gd_handle h, uint32_t k, int32_t* d_idx, uint64_t* d_key, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_state) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes: no state bound");
    if (k == 0) k = h->cfg.topk;
    if (k == 0) return GD_OK;
    if (k > h->N) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes: k exceeds the number of nodes");
    if (!d_idx) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes: null index output");
    if (((uintptr_t)d_idx & 3) || ((uintptr_t)d_key & 7))
        return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes: misaligned pointer");
    gd_topk_args a;
    a.count = reinterpret_cast<const uint16_t*>(h->d_state + h->lay.node_count);
    a.z_last = reinterpret_cast<const float*>(h->d_state + h->lay.node_z_last);
    a.score_sum = nullptr;
    a.idx = d_idx; a.key = d_key; a.N = h->N; a.k = k;
    hipError_t e = gd_launch_topk(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_topk_nodes");
    return GD_OK;
}

gd_status gd_apply_membership(gd_handle h, float* d_x, uint32_t T, const uint64_t* d_active, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (T == 0) return GD_OK;
    if (!d_x || !d_active) return fail(h, GD_ERR_INVALID_ARG, "gd_apply_membership: null pointer");
    if (((uintptr_t)d_x & 15) || ((uintptr_t)d_active & 7))
        return fail(h, GD_ERR_INVALID_ARG, "gd_apply_membership: misaligned pointer");
    if (T > 65535u) return fail(h, GD_ERR_INVALID_ARG, "gd_apply_membership: more than 65535 steps in one call");
    hipError_t e = gd_launch_membership(d_x, d_active, T, h->cfg.n_ranks, h->cfg.n_metrics,
                                        static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_apply_membership");
    return GD_OK;
}

gd_status gd_severity(gd_handle h, const float* d_x, uint32_t T, const float* d_med, float moderate,
                      float severe, float* d_node_slowdown, uint8_t* d_node_tier, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_state) return fail(h, GD_ERR_INVALID_ARG, "gd_severity: no state bound");
    if (!d_node_slowdown || !d_node_tier)
        return fail(h, GD_ERR_INVALID_ARG, "gd_severity: null output");
    if (T > 0 && (!d_x || !d_med)) return fail(h, GD_ERR_INVALID_ARG, "gd_severity: null input");
    if (((uintptr_t)d_x & 3) || ((uintptr_t)d_med & 3) || ((uintptr_t)d_node_slowdown & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_severity: misaligned pointer");
    if (!(moderate <= severe)) return fail(h, GD_ERR_INVALID_ARG, "gd_severity: moderate must not exceed severe");
    gd_severity_args a;
    a.state = h->d_state; a.lay = h->lay; a.x = d_x; a.med = d_med;
    a.slowdown = d_node_slowdown; a.tier = d_node_tier;
    a.T = T; a.R = h->cfg.n_ranks; a.M = h->cfg.n_metrics; a.N = h->N;
    a.W = h->cfg.window; a.K = h->cfg.persist_k; a.primary = h->cfg.primary_metric;
    a.dir = h->cfg.direction[h->cfg.primary_metric];
    a.moderate = moderate; a.severe = severe;
    hipError_t e = gd_launch_severity(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_severity");
    return GD_OK;
}

gd_status gd_sweep_score(gd_handle h, const float* d_flops, const float* d_bw, uint32_t n_nodes,
                         float tol_compute, float tol_sym, float tol_bw, float* d_gpu_shortfall,
                         uint8_t* d_gpu_mask, uint32_t* d_link_mask, uint8_t* d_verdict, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (n_nodes == 0) return GD_OK;
    if (!d_flops || !d_bw || !d_gpu_shortfall || !d_gpu_mask || !d_link_mask || !d_verdict)
        return fail(h, GD_ERR_INVALID_ARG, "gd_sweep_score: null pointer");
    if (((uintptr_t)d_flops & 3) || ((uintptr_t)d_bw & 3) || ((uintptr_t)d_gpu_shortfall & 3) ||
        ((uintptr_t)d_link_mask & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_sweep_score: misaligned pointer");
    gd_sweep_args a;
    a.flops = d_flops; a.bw = d_bw; a.shortfall = d_gpu_shortfall; a.gpu_mask = d_gpu_mask;
    a.link_mask = d_link_mask; a.verdict = d_verdict; a.n_nodes = n_nodes;
    a.tol_compute = tol_compute; a.tol_sym = tol_sym; a.tol_bw = tol_bw;
    hipError_t e = gd_launch_sweep(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_sweep_score");
    return GD_OK;
}

void gd_default_ledger_config(gd_ledger_config* c) {
    if (!c) return;
    memset(c, 0, sizeof(*c));
    c->struct_size = (uint32_t)sizeof(gd_ledger_config);
    c->score_quant = 64.0f;
    c->recur_limit = 3;
    c->recur_horizon = 604800;
}

size_t gd_ledger_bytes(gd_handle h, uint32_t max_T) {
    return h ? make_ledger_layout(h->cfg.n_ranks, h->N, h->cfg.window, max_T).total : 0;
}

gd_status gd_bind_ledger(gd_handle h, const gd_ledger_config* cfg, void* d_ledger, size_t bytes,
                         uint32_t max_T) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!cfg || !d_ledger) return fail(h, GD_ERR_INVALID_ARG, "gd_bind_ledger: null argument");
    if (cfg->struct_size != sizeof(gd_ledger_config))
        return fail(h, GD_ERR_BAD_CONFIG, "struct_size does not match this library's gd_ledger_config");
    if (!isfinite(cfg->score_quant) || !(cfg->score_quant > 0.0f))
        return fail(h, GD_ERR_BAD_CONFIG, "score_quant must be finite and positive");
    if (cfg->recur_limit < 1 || cfg->recur_limit > 8)
        return fail(h, GD_ERR_BAD_CONFIG, "recur_limit must be 1..8");
    if (cfg->recur_horizon < 1 || cfg->recur_horizon > (1ull << 62))
        return fail(h, GD_ERR_BAD_CONFIG, "recur_horizon must be 1..2^62 steps");
    if (max_T < 1) return fail(h, GD_ERR_INVALID_ARG, "gd_bind_ledger: max_T must be at least 1");
    if (((uintptr_t)d_ledger & 255) != 0)
        return fail(h, GD_ERR_INVALID_ARG, "gd_bind_ledger: ledger must be 256-byte aligned");
    const gd_ledger_layout l = make_ledger_layout(h->cfg.n_ranks, h->N, h->cfg.window, max_T);
    if (bytes < l.total)
        return fail(h, GD_ERR_BUFFER_TOO_SMALL, "gd_bind_ledger: buffer smaller than gd_ledger_bytes");
    h->lcfg = *cfg;
    h->llay = l;
    h->d_led = static_cast<uint8_t*>(d_ledger);
    h->led_max_T = max_T;
    return GD_OK;
}

namespace {

// Checks and arguments shared by the two entry points that take a batch into the ledger.
gd_status ledger_update_args(gd_handle h, const char* who, const uint8_t* d_exceed_mask,
                             const uint8_t* d_node_mask, const float* d_node_z, uint32_t T,
                             uint64_t first_step_index, gd_ledger_args* out) {
    const std::string name(who);
    if (!d_exceed_mask || !d_node_mask || !d_node_z)
        return fail(h, GD_ERR_INVALID_ARG, name + ": a required pointer is null");
    if (((uintptr_t)d_exceed_mask & 3) || ((uintptr_t)d_node_z & 3))
        return fail(h, GD_ERR_INVALID_ARG, name + ": misaligned pointer");
    if (first_step_index + (uint64_t)T > 0x7FFFFFFFull)
        return fail(h, GD_ERR_INVALID_ARG, name + ": step index beyond 2^31 - 1");
    gd_ledger_args& a = *out;
    a.led = h->d_led; a.lay = h->llay;
    a.rise = reinterpret_cast<uint64_t*>(h->d_led + h->llay.rise);
    a.exceed_mask = d_exceed_mask; a.node_mask = d_node_mask; a.node_z = d_node_z;
    a.T = T; a.R = h->cfg.n_ranks; a.N = h->N; a.W = h->cfg.window; a.K = h->cfg.persist_k;
    a.primary = h->cfg.primary_metric; a.min_signals = h->cfg.min_signals;
    a.limit = h->lcfg.recur_limit;
    a.quant = h->lcfg.score_quant;
    a.first_step = first_step_index; a.horizon = h->lcfg.recur_horizon;
    return GD_OK;
}

}  // namespace

gd_status gd_update_ledger(gd_handle h, const uint8_t* d_exceed_mask, const uint8_t* d_node_mask,
                           const float* d_node_z, uint32_t T, uint64_t first_step_index,
                           void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_led) return fail(h, GD_ERR_INVALID_ARG, "gd_update_ledger: no ledger bound");
    if (T == 0) return GD_OK;
    if (T > h->led_max_T)
        return fail(h, GD_ERR_INVALID_ARG, "gd_update_ledger: T exceeds the max_T the ledger was bound with");
    gd_ledger_args a;
    const gd_status st = ledger_update_args(h, "gd_update_ledger", d_exceed_mask, d_node_mask, d_node_z, T,
                                            first_step_index, &a);
    if (st != GD_OK) return st;
    hipError_t e = gd_launch_ledger(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_update_ledger");
    return GD_OK;
}

size_t gd_ledger_static_scratch_bytes(void) { return gd_ledger_static_bytes(); }

gd_status gd_update_ledger_static(gd_handle h, const uint8_t* d_exceed_mask, const uint8_t* d_node_mask,
                                  const float* d_node_z, uint32_t T, uint64_t first_step_index,
                                  void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_led) return fail(h, GD_ERR_INVALID_ARG, "gd_update_ledger_static: no ledger bound");
    if (T == 0) return GD_OK;
    gd_ledger_args a;
    const gd_status st = ledger_update_args(h, "gd_update_ledger_static", d_exceed_mask, d_node_mask,
                                            d_node_z, T, first_step_index, &a);
    if (st != GD_OK) return st;
    bool fits = true;
    hipError_t e = gd_launch_ledger_static(a, static_cast<hipStream_t>(stream), &fits);
    if (!fits) {
        char msg[200];
        snprintf(msg, sizeof msg,
                 "gd_update_ledger_static: %u steps of %u nodes need more than the %zu bytes of the "
                 "library's static work area; send shorter batches",
                 T, h->N, gd_ledger_static_bytes());
        return fail(h, GD_ERR_INVALID_ARG, msg);
    }
    if (e != hipSuccess) return hip_fail(h, e, "gd_update_ledger_static");
    return GD_OK;
}

gd_status gd_ledger_flags(gd_handle h, uint8_t* d_rank_pmask, uint8_t* d_rank_pflag,
                          int32_t* d_rank_pfirst, uint8_t* d_node_pmask, uint8_t* d_node_pflag,
                          int32_t* d_node_pfirst, int32_t* d_node_score_sum,
                          uint8_t* d_node_episodes, int32_t* d_node_terminal_first, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_led) return fail(h, GD_ERR_INVALID_ARG, "gd_ledger_flags: no ledger bound");
    if (((uintptr_t)d_rank_pfirst & 3) || ((uintptr_t)d_node_pfirst & 3) ||
        ((uintptr_t)d_node_score_sum & 3) || ((uintptr_t)d_node_terminal_first & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_ledger_flags: misaligned pointer");
    gd_ledger_flags_args a;
    a.led = h->d_led; a.lay = h->llay;
    a.rank_pmask = d_rank_pmask; a.rank_pflag = d_rank_pflag; a.rank_pfirst = d_rank_pfirst;
    a.node_pmask = d_node_pmask; a.node_pflag = d_node_pflag; a.node_pfirst = d_node_pfirst;
    a.node_score_sum = d_node_score_sum; a.node_episodes = d_node_episodes;
    a.node_terminal_first = d_node_terminal_first;
    a.R = h->cfg.n_ranks; a.N = h->N; a.K = h->cfg.persist_k;
    a.primary = h->cfg.primary_metric; a.min_signals = h->cfg.min_signals;
    a.limit = h->lcfg.recur_limit; a.horizon = h->lcfg.recur_horizon;
    hipError_t e = gd_launch_ledger_flags(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_ledger_flags");
    return GD_OK;
}

gd_status gd_topk_nodes_mean(gd_handle h, uint32_t k, int32_t* d_idx, uint64_t* d_key, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!h->d_led) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes_mean: no ledger bound");
    if (k == 0) k = h->cfg.topk;
    if (k == 0) return GD_OK;
    if (k > h->N) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes_mean: k exceeds the number of nodes");
    if (!d_idx) return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes_mean: null index output");
    if (((uintptr_t)d_idx & 3) || ((uintptr_t)d_key & 7))
        return fail(h, GD_ERR_INVALID_ARG, "gd_topk_nodes_mean: misaligned pointer");
    gd_topk_args a;
    a.count = reinterpret_cast<const uint16_t*>(h->d_led + h->llay.node_ccnt);
    a.z_last = nullptr;
    a.score_sum = reinterpret_cast<const int32_t*>(h->d_led + h->llay.node_qsum);
    a.idx = d_idx; a.key = d_key; a.N = h->N; a.k = k;
    hipError_t e = gd_launch_topk(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_topk_nodes_mean");
    return GD_OK;
}

gd_status gd_probe_read(gd_handle h, const float* d_x, uint64_t n_bytes, uint32_t* d_sink,
                        void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!d_x || !d_sink) return fail(h, GD_ERR_INVALID_ARG, "gd_probe_read: null pointer");
    if (((uintptr_t)d_x & 15) || ((uintptr_t)d_sink & 3))
        return fail(h, GD_ERR_INVALID_ARG, "gd_probe_read: misaligned pointer");
    hipError_t e = gd_launch_read_probe(d_x, n_bytes, d_sink, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_probe_read");
    return GD_OK;
}

gd_status gd_embed(gd_handle h, const gd_matrix* weight, const gd_matrix* tokens, float scale, const gd_matrix* out, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (const char* e = bad_tokens(tokens)) return invalid(h, "gd_embed", e);
    if (!weight || !out) return invalid(h, "gd_embed", "null matrix");
    if (!is_float(weight->dtype)) return fail(h, GD_ERR_UNSUPPORTED, "gd_embed: weight must be f32, bf16 or f16");
    if (out->dtype != weight->dtype) return invalid(h, "gd_embed", "out and weight differ in type");
    if (weight->rows > GD_MAX_VOCAB) return invalid(h, "gd_embed", "vocabulary above 2^24 rows");
    if (weight->cols > GD_MAX_WIDTH) return invalid(h, "gd_embed", "width above 65536");
    if (const char* e = bad_matrix(weight, weight->rows, weight->cols)) return invalid(h, "gd_embed", e);
    if (const char* e = bad_matrix(out, tokens->rows, weight->cols)) return invalid(h, "gd_embed", e);
    gd_embed_args a;
    a.weight = weight->d_data; a.weight_stride = weight->stride;
    a.out = out->d_data; a.out_stride = out->stride;
    a.tokens = tokens_of(tokens);
    a.vocab = (uint32_t)weight->rows; a.width = (uint32_t)weight->cols; a.dtype = weight->dtype; a.scale = scale;
    hipError_t e = gd_launch_embed(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_embed");
    return GD_OK;
}

size_t gd_embed_grad_work_bytes(uint64_t n, uint64_t vocab, uint64_t width) {
    if (n > GD_MAX_TOKENS || vocab > GD_MAX_VOCAB || width > GD_MAX_WIDTH) return 0;
    return gd_embed_grad_work(n, width);
}

gd_status gd_embed_grad(gd_handle h, const gd_matrix* out_grad, const gd_matrix* tokens, float scale, int32_t accumulate,
                        const gd_matrix* weight_grad, void* d_work, size_t work_bytes, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (const char* e = bad_tokens(tokens)) return invalid(h, "gd_embed_grad", e);
    if (!out_grad || !weight_grad) return invalid(h, "gd_embed_grad", "null matrix");
    if (!is_float(out_grad->dtype)) return fail(h, GD_ERR_UNSUPPORTED, "gd_embed_grad: gradients must be f32, bf16 or f16");
    if (out_grad->dtype != weight_grad->dtype) return invalid(h, "gd_embed_grad", "the gradients differ in type");
    if (weight_grad->rows > GD_MAX_VOCAB) return invalid(h, "gd_embed_grad", "vocabulary above 2^24 rows");
    if (weight_grad->cols > GD_MAX_WIDTH) return invalid(h, "gd_embed_grad", "width above 65536");
    if (const char* e = bad_matrix(weight_grad, weight_grad->rows, weight_grad->cols)) return invalid(h, "gd_embed_grad", e);
    if (const char* e = bad_matrix(out_grad, tokens->rows, weight_grad->cols)) return invalid(h, "gd_embed_grad", e);
    if (gd_status st = bad_work(h, "gd_embed_grad", d_work, work_bytes, gd_embed_grad_work(tokens->rows, weight_grad->cols))) return st;
    gd_embed_grad_args a;
    a.out_grad = out_grad->d_data; a.out_grad_stride = out_grad->stride;
    a.weight_grad = weight_grad->d_data; a.weight_grad_stride = weight_grad->stride;
    a.tokens = tokens_of(tokens);
    a.vocab = (uint32_t)weight_grad->rows; a.width = (uint32_t)weight_grad->cols; a.dtype = out_grad->dtype;
    a.accumulate = accumulate != 0; a.scale = scale;
    a.work = static_cast<uint8_t*>(d_work);
    hipError_t e = gd_launch_embed_grad(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_embed_grad");
    return GD_OK;
}

size_t gd_vocab_loss_work_bytes(uint64_t n, uint64_t vocab, uint64_t width, int32_t with_grad) {
    if (n > GD_MAX_TOKENS || vocab < 1 || vocab > GD_MAX_VOCAB || width < 1 || width > GD_MAX_WIDTH) return 0;
    return gd_vocab_loss_work(n, vocab, width, with_grad != 0);
}

gd_status gd_vocab_loss(gd_handle h, const gd_matrix* hidden, const gd_matrix* weight, const gd_matrix* targets, float logit_scale,
                        float* d_loss, float* d_lse, float* d_mean, void* d_work, size_t work_bytes, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (const char* e = bad_projection(hidden, weight, targets)) return invalid(h, "gd_vocab_loss", e);
    if (hidden->dtype != GD_BF16 && hidden->dtype != GD_F16)
        return fail(h, GD_ERR_UNSUPPORTED, "gd_vocab_loss: hidden and weight must be bf16 or f16");
    const uint64_t n = targets->rows;
    if (!d_mean || (n && (!d_loss || !d_lse))) return invalid(h, "gd_vocab_loss", "null output");
    if (((uintptr_t)d_loss & 3) || ((uintptr_t)d_lse & 3) || ((uintptr_t)d_mean & 3)) return invalid(h, "gd_vocab_loss", "misaligned output");
    if (gd_status st = bad_work(h, "gd_vocab_loss", d_work, work_bytes, gd_vocab_loss_work(n, weight->rows, weight->cols, false))) return st;
    gd_vocab_loss_args a;
    a.hidden = hidden->d_data; a.hidden_stride = hidden->stride;
    a.weight = weight->d_data; a.weight_stride = weight->stride;
    a.targets = tokens_of(targets);
    a.vocab = (uint32_t)weight->rows; a.width = (uint32_t)weight->cols; a.dtype = hidden->dtype; a.scale = logit_scale;
    a.loss = d_loss; a.lse = d_lse; a.mean = d_mean;
    a.work = static_cast<uint8_t*>(d_work);
    hipError_t e = gd_launch_vocab_loss(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_vocab_loss");
    return GD_OK;
}

gd_status gd_vocab_loss_grad(gd_handle h, const gd_matrix* hidden, const gd_matrix* weight, const gd_matrix* targets,
                             float logit_scale, const float* d_lse, const float* d_mean, const float* d_grad_mean,
                             const float* d_grad_rows, const gd_matrix* hidden_grad, const gd_matrix* weight_grad, void* d_work,
                             size_t work_bytes, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    const char* call = "gd_vocab_loss_grad";
    if (const char* e = bad_projection(hidden, weight, targets)) return invalid(h, call, e);
    if (hidden->dtype != GD_BF16 && hidden->dtype != GD_F16)
        return fail(h, GD_ERR_UNSUPPORTED, "gd_vocab_loss_grad: hidden and weight must be bf16 or f16");
    const uint64_t n = targets->rows;
    if (!d_grad_mean && !d_grad_rows) return invalid(h, call, "no gradient of the loss");
    if ((n && !d_lse) || (d_grad_mean && !d_mean)) return invalid(h, call, "null result of the loss");
    if (((uintptr_t)d_lse & 3) || ((uintptr_t)d_mean & 3) || ((uintptr_t)d_grad_mean & 3) || ((uintptr_t)d_grad_rows & 3))
        return invalid(h, call, "misaligned pointer");
    if (hidden_grad) {
        if (const char* e = bad_matrix(hidden_grad, n, weight->cols)) return invalid(h, call, e);
        if (hidden_grad->dtype != hidden->dtype) return invalid(h, call, "the gradients must have the type of hidden");
    }
    if (weight_grad) {
        if (const char* e = bad_matrix(weight_grad, weight->rows, weight->cols)) return invalid(h, call, e);
        if (weight_grad->dtype != hidden->dtype) return invalid(h, call, "the gradients must have the type of hidden");
    }
    if (!hidden_grad && !weight_grad) return GD_OK;
    if (gd_status st = bad_work(h, call, d_work, work_bytes, gd_vocab_loss_work(n, weight->rows, weight->cols, true))) return st;
    gd_vocab_grad_args a;
    a.hidden = hidden->d_data; a.hidden_stride = hidden->stride;
    a.weight = weight->d_data; a.weight_stride = weight->stride;
    a.targets = tokens_of(targets);
    a.vocab = (uint32_t)weight->rows; a.width = (uint32_t)weight->cols; a.dtype = hidden->dtype; a.scale = logit_scale;
    a.lse = d_lse; a.mean = d_mean; a.grad_mean = d_grad_mean; a.grad_rows = d_grad_rows;
    a.hidden_grad = hidden_grad ? hidden_grad->d_data : nullptr; a.hidden_grad_stride = hidden_grad ? hidden_grad->stride : 0;
    a.weight_grad = weight_grad ? weight_grad->d_data : nullptr; a.weight_grad_stride = weight_grad ? weight_grad->stride : 0;
    a.work = static_cast<uint8_t*>(d_work);
    hipError_t e = gd_launch_vocab_grad(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, call);
    return GD_OK;
}

size_t gd_adamw_table_bytes(gd_handle h, const gd_adamw_tensor* tensors, uint32_t n_tensors) {
    if (!h) return 0;
    if (const char* e = bad_tensors(tensors, n_tensors)) { invalid(h, "gd_adamw_table_bytes", e); return 0; }
    const size_t bytes = gd_adamw_table(tensors, n_tensors, nullptr);
    if (!bytes) invalid(h, "gd_adamw_table_bytes", "too many elements");
    return bytes;
}

gd_status gd_adamw_fill_table(gd_handle h, const gd_adamw_tensor* tensors, uint32_t n_tensors, void* host_table, size_t bytes) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (const char* e = bad_tensors(tensors, n_tensors)) return invalid(h, "gd_adamw_fill_table", e);
    const size_t need = gd_adamw_table(tensors, n_tensors, nullptr);
    if (!need) return invalid(h, "gd_adamw_fill_table", "too many elements");
    if (!host_table || ((uintptr_t)host_table & 7)) return invalid(h, "gd_adamw_fill_table", "null or misaligned table");
    if (bytes != need) return fail(h, GD_ERR_BUFFER_TOO_SMALL, "gd_adamw_fill_table: not gd_adamw_table_bytes bytes");
    gd_adamw_table(tensors, n_tensors, host_table);
    return GD_OK;
}

gd_status gd_adamw(gd_handle h, const void* d_table, size_t table_bytes, const gd_adamw_config* c, const float* d_grad_scale, void* stream) {
    if (!h) return GD_ERR_INVALID_ARG;
    if (!d_table || !c) return invalid(h, "gd_adamw", "null argument");
    if (c->struct_size != sizeof(gd_adamw_config))
        return fail(h, GD_ERR_BAD_CONFIG, "gd_adamw: struct_size does not match this library's gd_adamw_config");
    if (((uintptr_t)d_table & 255) || ((uintptr_t)d_grad_scale & 3)) return invalid(h, "gd_adamw", "misaligned pointer");
    if (table_bytes < 256 || (table_bytes & 255)) return invalid(h, "gd_adamw", "table_bytes is no table's size");
    if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0))
        return fail(h, GD_ERR_BAD_CONFIG, "gd_adamw: beta1 and beta2 must be in [0, 1)");
    if (!(isfinite(c->lr) && c->eps >= 0.0 && isfinite(c->eps))) return fail(h, GD_ERR_BAD_CONFIG, "gd_adamw: lr must be finite, eps finite and not negative");
    if (c->step < 1) return fail(h, GD_ERR_BAD_CONFIG, "gd_adamw: step counts from 1");
    gd_adamw_args a;
    a.table = static_cast<const uint8_t*>(d_table); a.table_bytes = table_bytes; a.grad_scale = d_grad_scale;
    a.lr = c->lr;
    a.fbeta1 = (float)c->beta1; a.fbeta2 = (float)c->beta2;
    a.one_beta1 = (float)(1.0 - c->beta1); a.one_beta2 = (float)(1.0 - c->beta2);
    a.c1 = 1.0 - pow(c->beta1, (double)c->step);
    a.inv_root_c2 = (float)(1.0 / sqrt(1.0 - pow(c->beta2, (double)c->step)));
    a.eps = (float)c->eps; a.seed = c->seed;
    hipError_t e = gd_launch_adamw(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(h, e, "gd_adamw");
    return GD_OK;
}

const char* gd_last_error(gd_handle h) { return h ? h->err.c_str() : g_create_error.c_str(); }

}  // extern "C"
