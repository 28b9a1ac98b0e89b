// C ABI of the library: argument checks, workspace carving, status text.  All arithmetic lives in the
// kernel translation units; nothing here allocates device memory or synchronises.
#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <utility>
#include <vector>

#include "common.cuh"
#include "kernels.h"
#include "vec_io.cuh"

namespace vardrop {

static thread_local char g_last_error[512] = "";

int fail(int status, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return status;
}

int check_cuda(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return VARDROP_OK;
    return fail(VARDROP_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

static int check_ptr(const void* p, const char* name, bool required) {
    if (!p) return required ? fail(VARDROP_ERR_INVALID_ARG, "%s is NULL", name) : VARDROP_OK;
    if (!aligned16(p)) return fail(VARDROP_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return VARDROP_OK;
}

static int check_ws(const void* ws, size_t have, size_t need) {
    if (int st = check_ptr(ws, "ws", true)) return st;
    if (have < need) return fail(VARDROP_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", have, need);
    return VARDROP_OK;
}

// ---- launch counter and optional per-kernel event timer ---------------------------------------------------
namespace {
std::mutex g_prof_mutex;
std::atomic<bool> g_prof_on{false};                                        // read on every launch, so without the lock
std::atomic<long long> g_launches{0};
std::vector<std::pair<cudaEvent_t, cudaEvent_t>> g_prof_events[K_COUNT];   // pairs recorded since the timer was armed
std::vector<std::pair<cudaEvent_t, cudaEvent_t>> g_prof_free;              // pairs ready for reuse
const char* const g_kernel_names[K_COUNT] = {"hash_kernel", "select_small_kernel", "select_count_kernel", "select_group_kernel", "select_sample_kernel",
                                             "attn_fwd_kernel", "bwd_prep_kernel", "attn_bwd_kernel", "bwd_convert_kernel", "pearson_normalize_kernel",
                                             "pearson_max_kernel", "gather_rows_kernel", "select_place_kernel", "select_cluster_kernel", "packed_plan_kernel",
                                             "attn_packed_fwd_kernel", "attn_packed_tile_kernel", "packed_short_kernel", "packed_prep_kernel", "attn_packed_bwd_kernel", "packed_convert_kernel", "norm_fwd_kernel", "norm_bwd_kernel", "norm_params_kernel", "grad_norm_kernel", "grad_scale_kernel",
                                             "embed_fwd_kernel", "embed_count_kernel", "embed_sort_kernel", "embed_sum_kernel", "embed_join_kernel", "embed_scan_kernel", "embed_place_kernel", "act_fwd_kernel", "act_bwd_kernel",
                                             "loss_count_kernel", "loss_rows_kernel", "loss_stats_kernel", "loss_join_kernel", "loss_grad_kernel", "loss_back_kernel", "loss_rest_kernel"};
}  // namespace

LaunchScope::LaunchScope(int id, cudaStream_t stream) : id_(id), stream_(stream), stop_(nullptr) {
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (!g_prof_on.load(std::memory_order_relaxed)) return;
    std::lock_guard<std::mutex> lock(g_prof_mutex);
    if (!g_prof_on.load(std::memory_order_relaxed)) return;                // disarmed in between
    std::pair<cudaEvent_t, cudaEvent_t> ev;
    if (!g_prof_free.empty()) {
        ev = g_prof_free.back();
        g_prof_free.pop_back();
    } else if (cudaEventCreate(&ev.first) != cudaSuccess || cudaEventCreate(&ev.second) != cudaSuccess) {
        return;
    }
    cudaEventRecord(ev.first, stream);
    g_prof_events[id].push_back(ev);
    stop_ = ev.second;
}

LaunchScope::~LaunchScope() {
    if (stop_) cudaEventRecord(static_cast<cudaEvent_t>(stop_), stream_);
}

// A wait that nothing ever completes: one warp polls a fresh barrier with the library's bounded wait and a caller-chosen limit,
// then reports the way every kernel of the library does (status word, normal exit).
__global__ void bounded_wait_probe_kernel(int* status, unsigned long long limit_ns) {
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        mbar_fence_init();
    }
    __syncthreads();
    chain_wait();
    chain_release();
    const bool done = mbar_wait(&bar, 0, limit_ns);
    if (!__all_sync(0xffffffffu, done) && threadIdx.x == 0) set_status(status, VARDROP_ERR_TIMEOUT);
}

}  // namespace vardrop

using namespace vardrop;

#define VD_CHECK(expr) do { if (int st_ = (expr)) return st_; } while (0)

extern "C" {

const char* vardrop_status_string(int status) {
    switch (status) {
        case VARDROP_OK: return "ok";
        case VARDROP_ERR_INVALID_ARG: return "invalid argument";
        case VARDROP_ERR_UNSUPPORTED: return "unsupported shape";
        case VARDROP_ERR_WORKSPACE: return "workspace too small";
        case VARDROP_ERR_CUDA: return "CUDA error";
        case VARDROP_ERR_TIMEOUT: return "bounded device wait timed out";
        case VARDROP_ERR_NONFINITE: return "non-finite amplitude";
        default: return "unknown status";
    }
}

const char* vardrop_last_error(void) { return g_last_error; }
const char* vardrop_version(void) { return "0.1"; }

int vardrop_ws_status(const void* ws, void* stream) {
    if (!ws) return fail(VARDROP_ERR_INVALID_ARG, "ws is NULL");
    int word = 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (int st = check_cuda(cudaMemcpyAsync(&word, ws, sizeof(int), cudaMemcpyDeviceToHost, s), "ws_status: copy")) return st;
    if (int st = check_cuda(cudaStreamSynchronize(s), "ws_status: synchronize")) return st;
    return word;
}

int vardrop_probe_bounded_wait(void* ws, size_t ws_bytes, unsigned int limit_us, void* stream) {
    VD_CHECK(check_ws(ws, ws_bytes, kWsHeaderBytes));
    if (limit_us < 1 || limit_us > 100000) return fail(VARDROP_ERR_INVALID_ARG, "probe: limit of %u us outside 1..100000", limit_us);
    const cudaError_t err = launch_chained(bounded_wait_probe_kernel, dim3(1), dim3(32), 0, static_cast<cudaStream_t>(stream), static_cast<int*>(ws),
                                           static_cast<unsigned long long>(limit_us) * 1000ull);
    return check_cuda(err, "probe: launch");
}

long long vardrop_launch_count(void) {
    return g_launches.load(std::memory_order_relaxed);
}

int vardrop_profile_kernels(void) { return K_COUNT; }

const char* vardrop_profile_kernel_name(int id) { return id >= 0 && id < K_COUNT ? g_kernel_names[id] : ""; }

int vardrop_profile_enable(int on) {
    std::lock_guard<std::mutex> lock(g_prof_mutex);
    for (int id = 0; id < K_COUNT; ++id) {
        for (auto& ev : g_prof_events[id]) g_prof_free.push_back(ev);
        g_prof_events[id].clear();
    }
    g_prof_on = on != 0;
    return VARDROP_OK;
}

int vardrop_profile_read(int id, double* total_ms, long long* launches) {
    if (id < 0 || id >= K_COUNT || !total_ms || !launches) return fail(VARDROP_ERR_INVALID_ARG, "profile_read: bad argument");
    std::lock_guard<std::mutex> lock(g_prof_mutex);
    double sum = 0.0;
    for (auto& ev : g_prof_events[id]) {
        if (int st = check_cuda(cudaEventSynchronize(ev.second), "profile_read: event synchronize")) return st;
        float ms = 0.f;
        if (int st = check_cuda(cudaEventElapsedTime(&ms, ev.first, ev.second), "profile_read: elapsed time")) return st;
        sum += ms;
    }
    *total_ms = sum;
    *launches = static_cast<long long>(g_prof_events[id].size());
    return VARDROP_OK;
}

size_t vardrop_hash_workspace_bytes(const vardrop_hash_cfg* cfg) { return cfg ? hash_workspace_bytes(*cfg) : 0; }

int vardrop_hash(const float* x, const vardrop_hash_cfg* cfg, uint64_t* keys, int32_t* freqs, float* amp_dbg, void* ws,
                 size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    int f_lo, f_hi;
    VD_CHECK(hash_validate(*cfg, &f_lo, &f_hi));
    VD_CHECK(check_ptr(x, "x", true));
    VD_CHECK(check_ptr(keys, "keys", true));
    VD_CHECK(check_ptr(freqs, "freqs", false));
    VD_CHECK(check_ptr(amp_dbg, "amp_dbg", false));
    VD_CHECK(check_ws(ws, ws_bytes, hash_workspace_bytes(*cfg)));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return hash_launch(x, *cfg, keys, freqs, amp_dbg, static_cast<int*>(ws), s);
}

size_t vardrop_select_workspace_bytes(const vardrop_select_cfg* cfg) {
    if (!cfg || select_validate(*cfg) != VARDROP_OK) return 0;
    return select_workspace_bytes(*cfg);
}

int vardrop_select(const uint64_t* keys, const vardrop_select_cfg* cfg, int32_t* group_id, int32_t* group_offsets,
                   int32_t* members, int32_t* n_groups, int32_t* sel_idx, int32_t* n_sel, int32_t* inv_idx, void* ws,
                   size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(select_validate(*cfg));
    VD_CHECK(check_ptr(keys, "keys", true));
    VD_CHECK(check_ptr(group_id, "group_id", true));
    VD_CHECK(check_ptr(group_offsets, "group_offsets", true));
    VD_CHECK(check_ptr(members, "members", true));
    VD_CHECK(check_ptr(n_groups, "n_groups", true));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", true));
    VD_CHECK(check_ptr(n_sel, "n_sel", true));
    VD_CHECK(check_ptr(inv_idx, "inv_idx", true));
    VD_CHECK(check_ws(ws, ws_bytes, select_workspace_bytes(*cfg)));
    return select_launch(keys, *cfg, group_id, group_offsets, members, n_groups, sel_idx, n_sel, inv_idx, ws,
                         static_cast<cudaStream_t>(stream));
}

int vardrop_select_static(const uint64_t* keys, const vardrop_select_cfg* cfg, int32_t* group_id, int32_t* group_offsets,
                          int32_t* members, int32_t* n_groups, int32_t* sel_idx, int32_t* n_sel, int32_t* inv_idx, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(select_validate(*cfg));
    VD_CHECK(check_ptr(keys, "keys", true));
    VD_CHECK(check_ptr(group_id, "group_id", true));
    VD_CHECK(check_ptr(group_offsets, "group_offsets", true));
    VD_CHECK(check_ptr(members, "members", true));
    VD_CHECK(check_ptr(n_groups, "n_groups", true));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", true));
    VD_CHECK(check_ptr(n_sel, "n_sel", true));
    VD_CHECK(check_ptr(inv_idx, "inv_idx", true));
    return select_static_launch(keys, *cfg, group_id, group_offsets, members, n_groups, sel_idx, n_sel, inv_idx,
                                static_cast<cudaStream_t>(stream));
}

int vardrop_gather_rows(const float* x, const int32_t* sel_idx, const int32_t* n_sel, const vardrop_gather_cfg* cfg, float* x_sel, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(gather_rows_validate(*cfg));
    VD_CHECK(check_ptr(x, "x", true));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", true));
    VD_CHECK(check_ptr(n_sel, "n_sel", true));
    VD_CHECK(check_ptr(x_sel, "x_sel", true));
    return gather_rows_launch(x, sel_idx, n_sel, *cfg, x_sel, static_cast<cudaStream_t>(stream));
}

size_t vardrop_attn_workspace_bytes(const vardrop_attn_cfg* cfg) {
    if (!cfg || attn_validate(*cfg) != VARDROP_OK) return 0;
    return attn_workspace_bytes(*cfg);
}

int vardrop_attn_fwd(const void* q, const void* k, const void* v, const int32_t* sel_idx, const int32_t* n_sel,
                     const vardrop_attn_cfg* cfg, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(attn_validate(*cfg));
    VD_CHECK(check_ptr(q, "q", true));
    VD_CHECK(check_ptr(k, "k", true));
    VD_CHECK(check_ptr(v, "v", true));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", false));
    if (sel_idx) VD_CHECK(check_ptr(n_sel, "n_sel", true));
    VD_CHECK(check_ptr(o, "o", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ws(ws, ws_bytes, attn_workspace_bytes(*cfg)));
    return attn_fwd_launch(q, k, v, sel_idx, n_sel, *cfg, o, lse, ws, static_cast<cudaStream_t>(stream));
}

int vardrop_attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o,
                     const int32_t* sel_idx, const int32_t* n_sel, const int32_t* inv_idx, const vardrop_attn_cfg* cfg,
                     void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(attn_validate(*cfg));
    VD_CHECK(check_ptr(q, "q", true));
    VD_CHECK(check_ptr(k, "k", true));
    VD_CHECK(check_ptr(v, "v", true));
    VD_CHECK(check_ptr(o, "o", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ptr(d_o, "d_o", true));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", false));
    if (sel_idx) {
        VD_CHECK(check_ptr(n_sel, "n_sel", true));
        VD_CHECK(check_ptr(inv_idx, "inv_idx", true));
    }
    VD_CHECK(check_ptr(dq, "dq", true));
    VD_CHECK(check_ptr(dk, "dk", true));
    VD_CHECK(check_ptr(dv, "dv", true));
    VD_CHECK(check_ws(ws, ws_bytes, attn_workspace_bytes(*cfg)));
    return attn_bwd_launch(q, k, v, o, lse, d_o, sel_idx, n_sel, inv_idx, *cfg, dq, dk, dv, ws, static_cast<cudaStream_t>(stream));
}

size_t vardrop_pearson_workspace_bytes(const vardrop_pearson_cfg* cfg) {
    if (!cfg || pearson_validate(*cfg) != VARDROP_OK) return 0;
    return pearson_workspace_bytes(*cfg);
}

int vardrop_pearson_max(const float* x, const vardrop_pearson_cfg* cfg, float* max_rho, int32_t* n_above, void* ws, size_t ws_bytes,
                        void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(pearson_validate(*cfg));
    VD_CHECK(check_ptr(x, "x", true));
    VD_CHECK(check_ptr(max_rho, "max_rho", true));
    VD_CHECK(check_ptr(n_above, "n_above", true));
    VD_CHECK(check_ws(ws, ws_bytes, pearson_workspace_bytes(*cfg)));
    return pearson_launch(x, *cfg, max_rho, n_above, ws, static_cast<cudaStream_t>(stream));
}

size_t vardrop_packed_plan_bytes(const vardrop_packed_cfg* cfg) {
    if (!cfg || packed_validate(*cfg) != VARDROP_OK) return 0;
    return packed_plan_bytes(*cfg);
}

size_t vardrop_attn_packed_workspace_bytes(const vardrop_packed_cfg* cfg) {
    if (!cfg || packed_validate(*cfg) != VARDROP_OK) return 0;
    return attn_packed_workspace_bytes(*cfg);
}

static int check_plan(const void* plan, size_t have, const vardrop_packed_cfg& cfg) {
    if (int st = check_ptr(plan, "plan", true)) return st;
    if (have < packed_plan_bytes(cfg)) return fail(VARDROP_ERR_WORKSPACE, "plan of %zu bytes given, %zu needed", have, packed_plan_bytes(cfg));
    return VARDROP_OK;
}

int vardrop_packed_plan(const int32_t* cu_seqlens, const vardrop_packed_cfg* cfg, void* plan, size_t plan_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(packed_validate(*cfg));
    VD_CHECK(check_ptr(cu_seqlens, "cu_seqlens", true));
    VD_CHECK(check_plan(plan, plan_bytes, *cfg));
    return packed_plan_launch(cu_seqlens, *cfg, plan, static_cast<cudaStream_t>(stream));
}

int vardrop_attn_packed_fwd(const void* q, const void* k, const void* v, const void* plan, size_t plan_bytes, const vardrop_packed_cfg* cfg, void* o, float* lse, void* ws,
                            size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(packed_validate(*cfg));
    VD_CHECK(check_ptr(q, "q", true));
    VD_CHECK(check_ptr(k, "k", true));
    VD_CHECK(check_ptr(v, "v", true));
    VD_CHECK(check_plan(plan, plan_bytes, *cfg));
    VD_CHECK(check_ptr(o, "o", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ws(ws, ws_bytes, kWsHeaderBytes));
    return attn_packed_fwd_launch(q, k, v, plan, *cfg, o, lse, ws, static_cast<cudaStream_t>(stream));
}

int vardrop_attn_packed_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o, const void* plan, size_t plan_bytes,
                            const vardrop_packed_cfg* cfg, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(packed_validate(*cfg));
    VD_CHECK(check_ptr(q, "q", true));
    VD_CHECK(check_ptr(k, "k", true));
    VD_CHECK(check_ptr(v, "v", true));
    VD_CHECK(check_ptr(o, "o", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ptr(d_o, "d_o", true));
    VD_CHECK(check_plan(plan, plan_bytes, *cfg));
    VD_CHECK(check_ptr(dq, "dq", true));
    VD_CHECK(check_ptr(dk, "dk", true));
    VD_CHECK(check_ptr(dv, "dv", true));
    VD_CHECK(check_ws(ws, ws_bytes, attn_packed_workspace_bytes(*cfg)));
    return attn_packed_bwd_launch(q, k, v, o, lse, d_o, plan, *cfg, dq, dk, dv, ws, static_cast<cudaStream_t>(stream));
}

// parameters and gradients that a configuration has no use for are refused, not ignored
static int norm_params_check(const vardrop_norm_cfg& c, const void* y, const void* gate, const void* w_post, const void* b_post, const void* w_pre, const void* b_pre) {
    if (!y && (c.post || c.gate_rows)) return fail(VARDROP_ERR_INVALID_ARG, "norm: y is NULL, but post=%d gate_rows=%d", c.post, c.gate_rows);
    if ((gate != nullptr) != (c.gate_rows != 0)) return fail(VARDROP_ERR_INVALID_ARG, "norm: gate_rows=%d and gate %s", c.gate_rows, gate ? "given" : "NULL");
    if ((w_post && c.post == 0) || (b_post && c.post != 2)) return fail(VARDROP_ERR_INVALID_ARG, "norm: post=%d has no such parameter", c.post);
    if ((w_pre && c.pre == 0) || (b_pre && c.pre != 2)) return fail(VARDROP_ERR_INVALID_ARG, "norm: pre=%d has no such parameter", c.pre);
    VD_CHECK(check_ptr(gate, "gate", false));
    VD_CHECK(check_ptr(w_post, "w_post", false));
    VD_CHECK(check_ptr(b_post, "b_post", false));
    VD_CHECK(check_ptr(w_pre, "w_pre", false));
    return check_ptr(b_pre, "b_pre", false);
}

// Buffers of a norm call that overlap.  An output that begins where an input of the same rows does is written by the threads that have read them; with a selection x and dx hold other rows than the
// rest.  Anything else would be read, or written, twice.
struct NormBuffer {
    const void* p;
    size_t bytes;
    enum Rows { kNone, kOwn, kAll } rows;    // of its own layout; of the kept tokens (all, without a selection); of all tokens
    const char* name;
};
static int norm_overlap_check(const NormBuffer* ins, int n_ins, const NormBuffer* outs, int n_outs) {
    const auto overlap = [](const NormBuffer& a, const NormBuffer& b) {
        const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
        return a.p && b.p && a.bytes && b.bytes && pa < pb + b.bytes && pb < pa + a.bytes;
    };
    for (int o = 0; o < n_outs; ++o) {
        for (int i = 0; i < n_ins; ++i)
            if (overlap(outs[o], ins[i]) && !(outs[o].p == ins[i].p && outs[o].rows == ins[i].rows && outs[o].rows != NormBuffer::kNone))
                return fail(VARDROP_ERR_INVALID_ARG, "norm: %s and %s overlap", outs[o].name, ins[i].name);
        for (int i = 0; i < o; ++i)
            if (overlap(outs[o], outs[i])) return fail(VARDROP_ERR_INVALID_ARG, "norm: %s and %s overlap", outs[o].name, outs[i].name);
    }
    return VARDROP_OK;
}

int vardrop_norm_fwd(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const float* b_pre,
                     const int32_t* sel_idx, const int32_t* n_sel, const vardrop_norm_cfg* cfg, void* h, void* u, float* stats, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(norm_validate(*cfg));
    VD_CHECK(check_ptr(x, "x", true));
    VD_CHECK(check_ptr(y, "y", false));
    VD_CHECK(norm_params_check(*cfg, y, gate, w_post, b_post, w_pre, b_pre));
    VD_CHECK(check_ptr(sel_idx, "sel_idx", false));
    if (sel_idx) VD_CHECK(check_ptr(n_sel, "n_sel", true));
    VD_CHECK(check_ptr(h, "h", false));
    if ((u != nullptr) != (cfg->pre != 0)) return fail(VARDROP_ERR_INVALID_ARG, "norm: pre=%d and u %s", cfg->pre, u ? "given" : "NULL");
    VD_CHECK(check_ptr(u, "u", false));
    VD_CHECK(check_ptr(stats, "stats", false));
    const size_t tokens = static_cast<size_t>(cfg->B) * cfg->N, rows = tokens * cfg->C * (cfg->dtype == 2 ? 4 : 2), row = sizeof(float) * cfg->C, S = sel_idx && cfg->S > 1 ? cfg->S : 1;
    const NormBuffer ins[] = {{x, rows, sel_idx ? NormBuffer::kAll : NormBuffer::kOwn, "x"}, {y, rows, NormBuffer::kOwn, "y"}, {gate, row * cfg->gate_rows, NormBuffer::kNone, "gate"},
                              {w_post, row, NormBuffer::kNone, "w_post"}, {b_post, row, NormBuffer::kNone, "b_post"}, {w_pre, row, NormBuffer::kNone, "w_pre"}, {b_pre, row, NormBuffer::kNone, "b_pre"},
                              {sel_idx, S * cfg->N * sizeof(int32_t), NormBuffer::kNone, "sel_idx"}, {sel_idx ? n_sel : nullptr, S * sizeof(int32_t), NormBuffer::kNone, "n_sel"}};
    const NormBuffer outs[] = {{h, rows, NormBuffer::kOwn, "h"}, {u, rows, NormBuffer::kOwn, "u"}, {stats, tokens * 16, NormBuffer::kNone, "stats"}};
    VD_CHECK(norm_overlap_check(ins, 9, outs, 3));
    return norm_fwd_launch(x, y, gate, w_post, b_post, w_pre, b_pre, sel_idx, n_sel, *cfg, h, u, stats, static_cast<cudaStream_t>(stream));
}

size_t vardrop_norm_workspace_bytes(const vardrop_norm_cfg* cfg) {
    if (!cfg || norm_validate(*cfg) != VARDROP_OK) return 0;
    return norm_workspace_bytes(*cfg);
}

int vardrop_norm_bwd(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const int32_t* sel_idx,
                     const int32_t* n_sel, const int32_t* inv_idx, const float* stats, const void* d_h, const void* d_u, const vardrop_norm_cfg* cfg, void* dx, void* dy,
                     float* d_gate, float* d_w_post, float* d_b_post, float* d_w_pre, float* d_b_pre, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(norm_validate(*cfg));
    VD_CHECK(check_ptr(x, "x", true));
    VD_CHECK(check_ptr(y, "y", false));
    VD_CHECK(norm_params_check(*cfg, y, gate, w_post, b_post, w_pre, nullptr));
    if ((d_gate && !cfg->gate_rows) || (d_w_post && !cfg->post) || (d_b_post && cfg->post != 2) || (d_w_pre && !cfg->pre) || (d_b_pre && cfg->pre != 2))
        return fail(VARDROP_ERR_INVALID_ARG, "norm: gradient of a parameter that pre=%d post=%d gate_rows=%d does not have", cfg->pre, cfg->post, cfg->gate_rows);
    VD_CHECK(check_ptr(sel_idx, "sel_idx", false));
    if (sel_idx) {
        VD_CHECK(check_ptr(n_sel, "n_sel", true));
        VD_CHECK(check_ptr(inv_idx, "inv_idx", true));
    }
    VD_CHECK(check_ptr(stats, "stats", true));
    VD_CHECK(check_ptr(d_h, "d_h", false));
    if ((d_u != nullptr) != (cfg->pre != 0)) return fail(VARDROP_ERR_INVALID_ARG, "norm: pre=%d and d_u %s", cfg->pre, d_u ? "given" : "NULL");
    VD_CHECK(check_ptr(d_u, "d_u", false));
    VD_CHECK(check_ptr(dx, "dx", true));
    if ((dy != nullptr) != (y != nullptr)) return fail(VARDROP_ERR_INVALID_ARG, "norm: y and dy have to be given, or NULL, together");
    VD_CHECK(check_ptr(dy, "dy", false));
    VD_CHECK(check_ptr(d_gate, "d_gate", false));
    VD_CHECK(check_ptr(d_w_post, "d_w_post", false));
    VD_CHECK(check_ptr(d_b_post, "d_b_post", false));
    VD_CHECK(check_ptr(d_w_pre, "d_w_pre", false));
    VD_CHECK(check_ptr(d_b_pre, "d_b_pre", false));
    VD_CHECK(check_ws(ws, ws_bytes, norm_workspace_bytes(*cfg)));
    const size_t tokens = static_cast<size_t>(cfg->B) * cfg->N, rows = tokens * cfg->C * (cfg->dtype == 2 ? 4 : 2), row = sizeof(float) * cfg->C, S = sel_idx && cfg->S > 1 ? cfg->S : 1;
    const size_t index = sel_idx ? S * cfg->N * sizeof(int32_t) : 0;
    const NormBuffer::Rows of_x = sel_idx ? NormBuffer::kAll : NormBuffer::kOwn;
    const NormBuffer ins[] = {{x, rows, of_x, "x"}, {y, rows, NormBuffer::kOwn, "y"}, {d_h, rows, NormBuffer::kOwn, "d_h"}, {d_u, rows, NormBuffer::kOwn, "d_u"}, {stats, tokens * 16, NormBuffer::kNone, "stats"},
                              {gate, row * cfg->gate_rows, NormBuffer::kNone, "gate"}, {w_post, row, NormBuffer::kNone, "w_post"}, {b_post, row, NormBuffer::kNone, "b_post"},
                              {w_pre, row, NormBuffer::kNone, "w_pre"}, {sel_idx, index, NormBuffer::kNone, "sel_idx"}, {inv_idx, index, NormBuffer::kNone, "inv_idx"},
                              {n_sel, sel_idx ? S * sizeof(int32_t) : 0, NormBuffer::kNone, "n_sel"}};
    const NormBuffer outs[] = {{dx, rows, of_x, "dx"}, {dy, rows, NormBuffer::kOwn, "dy"}, {d_gate, row * cfg->gate_rows, NormBuffer::kNone, "d_gate"}, {d_w_post, row, NormBuffer::kNone, "d_w_post"},
                               {d_b_post, row, NormBuffer::kNone, "d_b_post"}, {d_w_pre, row, NormBuffer::kNone, "d_w_pre"}, {d_b_pre, row, NormBuffer::kNone, "d_b_pre"}};
    VD_CHECK(norm_overlap_check(ins, 12, outs, 7));
    return norm_bwd_launch(x, y, gate, w_post, b_post, w_pre, sel_idx, n_sel, inv_idx, stats, d_h, d_u, *cfg, dx, dy, d_gate, d_w_post, d_b_post, d_w_pre, d_b_pre, ws,
                           static_cast<cudaStream_t>(stream));
}

size_t vardrop_grad_clip_workspace_bytes(void) { return grad_clip_workspace_bytes(); }

int vardrop_grad_clip(const vardrop_tensor* tensors, int32_t count, const vardrop_clip_cfg* cfg, float* norm, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(grad_clip_validate(tensors, count, *cfg));
    VD_CHECK(check_ptr(norm, "norm", true));
    VD_CHECK(check_ws(ws, ws_bytes, grad_clip_workspace_bytes()));
    return grad_clip_launch(tensors, count, *cfg, norm, ws, static_cast<cudaStream_t>(stream));
}

// Buffers of a call that overlap: rows of `cols` elements, `stride` apart.  Views of one tensor whose rows lie between each other's do not.
struct Rows {
    const void* p;
    size_t rows, cols, stride, size;            // size: of an element
    const char* name;
};
static Rows flat(const void* p, size_t n, size_t size, const char* name) { return Rows{p, 1, n, n, size, name}; }
static bool rows_overlap(const Rows& x, const Rows& y) {
    if (!x.p || !y.p || x.rows * x.cols == 0 || y.rows * y.cols == 0) return false;
    const uintptr_t px = reinterpret_cast<uintptr_t>(x.p), py = reinterpret_cast<uintptr_t>(y.p);
    const size_t nx = ((x.rows - 1) * x.stride + x.cols) * x.size, ny = ((y.rows - 1) * y.stride + y.cols) * y.size;
    if (px >= py + ny || py >= px + nx) return false;
    if (x.stride != y.stride || x.size != y.size) return true;
    const size_t step = x.stride * x.size, r = (px < py ? py - px : px - py) % step, first = px < py ? x.cols : y.cols, second = px < py ? y.cols : x.cols;
    return !(r >= first * x.size && r + second * x.size <= step);
}
// An output may begin where an input of the same rows does where `same` says so: it is written by the threads that have read it.
static int overlap_check(const char* call, const Rows* ins, int n_ins, const Rows* outs, int n_outs, bool same) {
    for (int o = 0; o < n_outs; ++o) {
        for (int i = 0; i < n_ins; ++i)
            if (rows_overlap(outs[o], ins[i]) &&
                !(same && outs[o].p == ins[i].p && outs[o].rows == ins[i].rows && outs[o].cols == ins[i].cols && outs[o].stride == ins[i].stride && outs[o].size == ins[i].size))
                return fail(VARDROP_ERR_INVALID_ARG, "%s: %s and %s overlap", call, outs[o].name, ins[i].name);
        for (int i = 0; i < o; ++i)
            if (rows_overlap(outs[o], outs[i])) return fail(VARDROP_ERR_INVALID_ARG, "%s: %s and %s overlap", call, outs[o].name, outs[i].name);
    }
    return VARDROP_OK;
}

size_t vardrop_embed_workspace_bytes(const vardrop_embed_cfg* cfg) {
    if (!cfg || embed_validate(*cfg) != VARDROP_OK) return 0;
    return embed_workspace_bytes(*cfg);
}

int vardrop_embed_fwd(const void* table, const int32_t* idx, const vardrop_embed_cfg* cfg, void* out, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(embed_validate(*cfg));
    VD_CHECK(check_ptr(table, "table", true));
    VD_CHECK(check_ptr(idx, "idx", true));
    VD_CHECK(check_ptr(out, "out", true));
    VD_CHECK(check_ws(ws, ws_bytes, kWsHeaderBytes));
    const size_t C = cfg->C;
    const Rows ins[] = {flat(table, cfg->V * C, dtype_bytes(cfg->dtype), "table"), flat(idx, cfg->T, 4, "idx"), flat(ws, kWsHeaderBytes, 1, "ws")};
    const Rows outs[] = {flat(out, cfg->T * C, dtype_bytes(cfg->out_dtype), "out")};
    VD_CHECK(overlap_check("embed", ins, 3, outs, 1, false));
    return embed_fwd_launch(table, idx, *cfg, out, ws, static_cast<cudaStream_t>(stream));
}

int vardrop_embed_bwd(const void* d_out, const int32_t* idx, const vardrop_embed_cfg* cfg, void* d_table, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(embed_validate(*cfg));
    VD_CHECK(check_ptr(d_out, "d_out", true));
    VD_CHECK(check_ptr(idx, "idx", true));
    VD_CHECK(check_ptr(d_table, "d_table", true));
    VD_CHECK(check_ws(ws, ws_bytes, embed_workspace_bytes(*cfg)));
    const size_t C = cfg->C;
    const Rows ins[] = {flat(d_out, cfg->T * C, dtype_bytes(cfg->out_dtype), "d_out"), flat(idx, cfg->T, 4, "idx")};
    const Rows outs[] = {flat(d_table, cfg->V * C, dtype_bytes(cfg->dtype), "d_table"), flat(ws, embed_workspace_bytes(*cfg), 1, "ws")};
    VD_CHECK(overlap_check("embed", ins, 2, outs, 2, false));
    return embed_bwd_launch(d_out, idx, *cfg, d_table, ws, static_cast<cudaStream_t>(stream));
}

size_t vardrop_act_ckpt_bytes(const vardrop_act_cfg* cfg) {
    if (!cfg || act_validate(*cfg) != VARDROP_OK) return 0;
    return act_ckpt_bytes(*cfg);
}

static int check_ckpt(const void* ckpt, size_t have, const vardrop_act_cfg& cfg) {
    if (int st = check_ptr(ckpt, "ckpt", true)) return st;
    if (have < act_ckpt_bytes(cfg)) return fail(VARDROP_ERR_WORKSPACE, "checkpoint of %zu bytes given, %zu needed", have, act_ckpt_bytes(cfg));
    return VARDROP_OK;
}

int vardrop_act_fwd(const void* a, const void* b, const int32_t* n_sel, const vardrop_act_cfg* cfg, void* y, void* ckpt, size_t ckpt_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(act_validate(*cfg));
    VD_CHECK(check_ptr(a, "a", true));
    if ((b != nullptr) != (cfg->gated != 0)) return fail(VARDROP_ERR_INVALID_ARG, "act: gated=%d and b %s", cfg->gated, b ? "given" : "NULL");
    VD_CHECK(check_ptr(b, "b", false));
    VD_CHECK(check_ptr(n_sel, "n_sel", false));
    VD_CHECK(check_ptr(y, "y", true));
    if (ckpt) VD_CHECK(check_ckpt(ckpt, ckpt_bytes, *cfg));
    const size_t rows = static_cast<size_t>(cfg->B) * cfg->N, C = cfg->C, stride = cfg->stride ? cfg->stride : C, size = dtype_bytes(cfg->dtype);
    const Rows ins[] = {{a, rows, C, stride, size, "a"}, {b, rows, C, stride, size, "b"}, flat(n_sel, cfg->S > 1 ? cfg->S : 1, 4, "n_sel")};
    const Rows outs[] = {{y, rows, C, C, size, "y"}, flat(ckpt, ckpt ? act_ckpt_bytes(*cfg) : 0, 1, "ckpt")};
    VD_CHECK(overlap_check("act", ins, 3, outs, 2, true));
    return act_fwd_launch(a, b, n_sel, *cfg, y, ckpt, static_cast<cudaStream_t>(stream));
}

int vardrop_act_bwd(const void* d_y, const void* ckpt, size_t ckpt_bytes, const int32_t* n_sel, const vardrop_act_cfg* cfg, void* d_a, void* d_b, void* y, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(act_validate(*cfg));
    VD_CHECK(check_ptr(d_y, "d_y", true));
    VD_CHECK(check_ckpt(ckpt, ckpt_bytes, *cfg));
    VD_CHECK(check_ptr(n_sel, "n_sel", false));
    VD_CHECK(check_ptr(d_a, "d_a", true));
    if ((d_b != nullptr) != (cfg->gated != 0)) return fail(VARDROP_ERR_INVALID_ARG, "act: gated=%d and d_b %s", cfg->gated, d_b ? "given" : "NULL");
    VD_CHECK(check_ptr(d_b, "d_b", false));
    VD_CHECK(check_ptr(y, "y", false));
    const size_t rows = static_cast<size_t>(cfg->B) * cfg->N, C = cfg->C, stride = cfg->stride ? cfg->stride : C, size = dtype_bytes(cfg->dtype);
    const Rows ins[] = {{d_y, rows, C, C, size, "d_y"}, flat(ckpt, act_ckpt_bytes(*cfg), 1, "ckpt"), flat(n_sel, cfg->S > 1 ? cfg->S : 1, 4, "n_sel")};
    const Rows outs[] = {{d_a, rows, C, stride, size, "d_a"}, {d_b, rows, C, stride, size, "d_b"}, {y, rows, C, C, size, "y"}};
    VD_CHECK(overlap_check("act", ins, 3, outs, 3, true));
    return act_bwd_launch(d_y, ckpt, n_sel, *cfg, d_a, d_b, y, static_cast<cudaStream_t>(stream));
}

size_t vardrop_loss_workspace_bytes(const vardrop_loss_cfg* cfg) {
    if (!cfg || loss_validate(*cfg) != VARDROP_OK) return 0;
    return loss_workspace_bytes(*cfg);
}

int vardrop_loss_fwd(const void* h, const void* w, const int32_t* labels, const vardrop_loss_cfg* cfg, float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(loss_validate(*cfg));
    VD_CHECK(check_ptr(h, "h", true));
    VD_CHECK(check_ptr(w, "w", true));
    VD_CHECK(check_ptr(labels, "labels", true));
    VD_CHECK(check_ptr(loss, "loss", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ws(ws, ws_bytes, loss_workspace_bytes(*cfg)));
    const size_t T = cfg->T, V = cfg->V, C = cfg->C;
    const Rows ins[] = {flat(h, T * C, 2, "h"), flat(w, V * C, 2, "w"), flat(labels, T, 4, "labels")};
    const Rows outs[] = {flat(loss, T, 4, "loss"), flat(lse, T, 4, "lse"), flat(ws, loss_workspace_bytes(*cfg), 1, "ws")};
    VD_CHECK(overlap_check("loss", ins, 3, outs, 3, false));
    return loss_fwd_launch(h, w, labels, *cfg, loss, lse, ws, static_cast<cudaStream_t>(stream));
}

int vardrop_loss_bwd(const void* h, const void* w, const int32_t* labels, const float* lse, const float* d_loss, const vardrop_loss_cfg* cfg, void* d_h, void* d_w, void* ws, size_t ws_bytes,
                     void* stream) {
    if (!cfg) return fail(VARDROP_ERR_INVALID_ARG, "cfg is NULL");
    VD_CHECK(loss_validate(*cfg));
    VD_CHECK(check_ptr(h, "h", true));
    VD_CHECK(check_ptr(w, "w", true));
    VD_CHECK(check_ptr(labels, "labels", true));
    VD_CHECK(check_ptr(lse, "lse", true));
    VD_CHECK(check_ptr(d_loss, "d_loss", true));
    if (!d_h && !d_w) return fail(VARDROP_ERR_INVALID_ARG, "loss: d_h and d_w are both NULL");
    VD_CHECK(check_ptr(d_h, "d_h", false));
    VD_CHECK(check_ptr(d_w, "d_w", false));
    VD_CHECK(check_ws(ws, ws_bytes, loss_workspace_bytes(*cfg)));
    const size_t T = cfg->T, V = cfg->V, C = cfg->C;
    const Rows ins[] = {flat(h, T * C, 2, "h"), flat(w, V * C, 2, "w"), flat(labels, T, 4, "labels"), flat(lse, T, 4, "lse"), flat(d_loss, T, 4, "d_loss")};
    const Rows outs[] = {flat(d_h, T * C, 2, "d_h"), flat(d_w, V * C, 2, "d_w"), flat(ws, loss_workspace_bytes(*cfg), 1, "ws")};
    VD_CHECK(overlap_check("loss", ins, 5, outs, 3, false));
    return loss_bwd_launch(h, w, labels, lse, d_loss, *cfg, d_h, d_w, ws, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
