// C ABI glue: argument checks, then the kernel launchers.  No compute happens on the host.
#include <string>

#include "tc_internal.h"

namespace {

bool misaligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

tc_status fail(tc_status s, const std::string &msg) {
    tc::set_error(msg);
    return s;
}

tc_status device_result(int err, const char *what) {
    if (!err) return TC_OK;
    return fail(TC_ERR_DEVICE, std::string(what) + ": " + tc::hip_error_text(err));
}

tc_status check_runnable(const tc_plan *plan, const tc_kv_pool *pool) {
    tc_status st = tc::check_pool_matches(plan, pool, true);
    if (st != TC_OK) return st;
    if (!plan->dev) return fail(TC_ERR_ARG, "plan was built host-only (tc_plan_create_host) and cannot be launched");
    return TC_OK;
}

tc_status check_plan_device(const tc_plan *plan) {  // last, so that a plan without a device copy shows every other mistake
    if (!plan->dev) return fail(TC_ERR_ARG, "plan was built host-only (tc_plan_create_host) and cannot be launched");
    int device = -1;
    if (int err = tc::current_device(&device)) return device_result(err, "current device");
    if (device != plan->device) return fail(TC_ERR_DEVICE, "the current device is not the one the plan was made on");
    return TC_OK;
}

tc_status attention(const tc_plan *plan, const tc_kv_pool *pool, const void *q, const void *k_new, const void *v_new, void *out,
                    float scale, void *workspace, size_t workspace_bytes, int launches, void *stream, const char *what) {
    tc_status st = check_runnable(plan, pool);
    if (st != TC_OK) return st;
    if (plan->T == 0) return TC_OK;
    if (!out || (!q && (launches & (tc::kLaunchAttention | tc::kLaunchFused)))) return fail(TC_ERR_NULL, "q or out is NULL");
    const size_t need = plan->workspace_bytes();
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(TC_ERR_WORKSPACE, "workspace missing or too small");
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(TC_ERR_ARG, "scale must be positive and finite");
    return device_result(tc::launch_attention(plan, pool, q, k_new, v_new, out, scale, need ? workspace : nullptr, launches, stream), what);
}

}  // namespace

extern "C" {

tc_status tc_kv_append(const tc_plan *plan, const tc_kv_pool *pool, const void *k_new, const void *v_new, void *stream) {
    tc_status st = check_runnable(plan, pool);
    if (st != TC_OK) return st;
    if (plan->T == 0) return TC_OK;
    if (!k_new || !v_new) return fail(TC_ERR_NULL, "k_new or v_new is NULL");
    return device_result(tc::launch_kv_append(plan, pool, k_new, v_new, false, stream), "tc_kv_append launch");
}

tc_status tc_mixed_attention(const tc_plan *plan, const tc_kv_pool *pool, const void *q, void *out, float scale,
                             void *workspace, size_t workspace_bytes, void *stream) {
    return attention(plan, pool, q, nullptr, nullptr, out, scale, workspace, workspace_bytes, tc::kLaunchFused, stream,
                     "tc_mixed_attention launch");
}

tc_status tc_mixed_attention_append(const tc_plan *plan, const tc_kv_pool *pool, const void *q, const void *k_new,
                                    const void *v_new, void *out, float scale, void *workspace, size_t workspace_bytes,
                                    void *stream) {
    tc_status st = check_runnable(plan, pool);
    if (st != TC_OK) return st;
    if (plan->T == 0) return TC_OK;
    if (!k_new || !v_new) return fail(TC_ERR_NULL, "k_new or v_new is NULL");
    if (!out || !q) return fail(TC_ERR_NULL, "q or out is NULL");
    const size_t need = plan->workspace_bytes();
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(TC_ERR_WORKSPACE, "workspace missing or too small");
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(TC_ERR_ARG, "scale must be positive and finite");
    // A batch with a prefill chunk: the chunk's rows are read by many workgroups of the attention kernel, which may not
    // wait for one another, so all rows are stored first, by the append kernel (the two calls in one).  So they are where a decode attends
    // over a block that another's row goes into.  Other batches of decodes: one launch, whose last workgroups store the rows while the grid drains.
    if (plan->append_apart) {
        st = device_result(tc::launch_kv_append(plan, pool, k_new, v_new, false, stream), "tc_mixed_attention_append launch");
        if (st != TC_OK) return st;
    }
    const bool apart = plan->append_apart;
    return device_result(tc::launch_attention(plan, pool, q, apart ? nullptr : k_new, apart ? nullptr : v_new, out, scale, need ? workspace : nullptr, tc::kLaunchFused, stream),
                         "tc_mixed_attention_append launch");
}

tc_status tc_mixed_attention_static(const tc_plan *plan, const tc_kv_pool *pool, const void *q, void *out, float scale, void *stream) {
    tc_status st = check_runnable(plan, pool);
    if (st != TC_OK) return st;
    if (plan->T == 0) return TC_OK;
    void *scratch = nullptr;
    size_t scratch_bytes = 0;
    if (int err = tc::static_scratch(plan->device, &scratch, &scratch_bytes)) return device_result(err, "static scratch of this GPU");
    if (plan->workspace_bytes() > scratch_bytes)
        return fail(TC_ERR_WORKSPACE, "this batch needs more scratch than the static array holds (64 MiB): use tc_mixed_attention with a workspace");
    return attention(plan, pool, q, nullptr, nullptr, out, scale, scratch, scratch_bytes, tc::kLaunchFused, stream,
                     "tc_mixed_attention_static launch");
}

tc_status tc_attention_partials(const tc_plan *plan, const tc_kv_pool *pool, const void *q, void *out, float scale,
                                void *workspace, size_t workspace_bytes, void *stream) {
    return attention(plan, pool, q, nullptr, nullptr, out, scale, workspace, workspace_bytes, tc::kLaunchAttention, stream,
                     "tc_attention_partials launch");
}

tc_status tc_split_merge(const tc_plan *plan, const tc_kv_pool *pool, void *out, void *workspace, size_t workspace_bytes,
                         void *stream) {
    return attention(plan, pool, nullptr, nullptr, nullptr, out, 1.f, workspace, workspace_bytes, tc::kLaunchMerge, stream,
                     "tc_split_merge launch");
}

tc_status tc_probe_mfma_loop(int32_t iters, void *sink, size_t sink_bytes, void *stream) {
    if (!sink) return fail(TC_ERR_NULL, "sink is NULL");
    if (iters < 1 || sink_bytes < (size_t)tc::kNumCu * 512 * sizeof(float)) return fail(TC_ERR_ARG, "iters < 1 or sink smaller than 512 KiB");
    return device_result(tc::launch_probe_mfma(iters, sink, stream), "tc_probe_mfma_loop launch");
}

tc_status tc_probe_stream_read(const void *src, size_t bytes, void *sink, void *stream) {
    if (!src || !sink) return fail(TC_ERR_NULL, "src or sink is NULL");
    if (bytes < 16) return fail(TC_ERR_ARG, "nothing to read");
    return device_result(tc::launch_probe_stream(src, bytes, sink, stream), "tc_probe_stream_read launch");
}

tc_status tc_probe_stream_copy(const void *src, void *dst, size_t bytes, void *stream) {
    if (!src || !dst) return fail(TC_ERR_NULL, "src or dst is NULL");
    if (bytes < 16) return fail(TC_ERR_ARG, "nothing to copy");
    return device_result(tc::launch_probe_copy(src, dst, bytes, stream), "tc_probe_stream_copy launch");
}

tc_status tc_kv_gather(const tc_plan *plan, const tc_kv_pool *pool, int32_t seq, void *k_out, void *v_out, void *stream) {
    tc_status st = check_runnable(plan, pool);
    if (st != TC_OK) return st;
    if (seq < 0 || seq >= plan->S) return fail(TC_ERR_ARG, "sequence index out of range");
    if (!k_out || !v_out) return fail(TC_ERR_NULL, "k_out or v_out is NULL");
    return device_result(tc::launch_kv_gather(plan, pool, seq, k_out, v_out, stream), "tc_kv_gather launch");
}

}  // extern "C"

namespace {

// Pages [page0, page0 + n) of the plan that `seq` selects (-1 = every sequence).
bool selection(const tc_plan *plan, int32_t seq, int *page0, int *n) {
    if (seq == -1) { *page0 = 0; *n = (int)plan->total_pages; return true; }
    if (seq < 0 || seq >= plan->S) return false;
    *page0 = plan->page_off[seq];
    *n = plan->page_off[seq + 1] - plan->page_off[seq];
    return true;
}

tc_status migrate(const tc_plan *plan, const tc_kv_pool *pool, int32_t seq, int32_t num_layers, void *const *k_pools,
                  void *const *v_pools, void *buffer, void *stream, bool import) {
    tc_status st = tc::check_pool_matches(plan, pool, false);
    if (st != TC_OK) return st;
    if (!plan->dev) return fail(TC_ERR_ARG, "plan was built host-only (tc_plan_create_host) and cannot be launched");
    int page0 = 0, n = 0;
    if (!selection(plan, seq, &page0, &n)) return fail(TC_ERR_ARG, "sequence index out of range");
    if (num_layers < 1 || num_layers > tc::kMaxLayers) return fail(TC_ERR_ARG, "num_layers must be in [1, 4096]");
    if (n == 0) return TC_OK;
    if (!k_pools || !v_pools || !buffer) return fail(TC_ERR_NULL, "k_pools, v_pools or buffer is NULL");
    for (int l = 0; l < num_layers; l++)
        if (!k_pools[l] || !v_pools[l]) return fail(TC_ERR_NULL, "a layer's pool pointer is NULL");
    return device_result(tc::launch_kv_migrate(plan, import, page0, n, num_layers, k_pools, v_pools, buffer, stream),
                         import ? "tc_kv_import launch" : "tc_kv_export launch");
}

}  // namespace

extern "C" {

size_t tc_kv_transfer_bytes(const tc_plan *plan, int32_t seq, int32_t num_layers) {
    int page0 = 0, n = 0;
    if (!plan || plan->kvq || num_layers < 1 || num_layers > tc::kMaxLayers || !selection(plan, seq, &page0, &n)) return 0;
    return (size_t)num_layers * (size_t)n * 2 * (size_t)plan->Hkv * tc::kBlock * (size_t)plan->D * sizeof(uint16_t);
}

tc_status tc_kv_export(const tc_plan *plan, const tc_kv_pool *pool, int32_t seq, int32_t num_layers,
                       const void *const *k_pools, const void *const *v_pools, void *buffer, void *stream) {
    return migrate(plan, pool, seq, num_layers, (void *const *)k_pools, (void *const *)v_pools, buffer, stream, false);
}

tc_status tc_kv_import(const tc_plan *plan, const tc_kv_pool *pool, int32_t seq, int32_t num_layers,
                       void *const *k_pools, void *const *v_pools, const void *buffer, void *stream) {
    return migrate(plan, pool, seq, num_layers, k_pools, v_pools, (void *)buffer, stream, true);
}

}  // extern "C"

// ---- the KV cache in 8 bits

namespace {

tc_status check_kvq(const tc_plan *plan, const tc_kvq_pool *pool) {
    if (!plan || !pool) return fail(TC_ERR_NULL, "plan or pool is NULL");
    tc_status st = tc::check_pool_matches(plan, &pool->base, true, true);
    if (st != TC_OK) return st;
    if (!pool->scales) return fail(TC_ERR_NULL, "scales is NULL");
    if (misaligned(pool->base.k_pool, 16) || misaligned(pool->base.v_pool, 16) || misaligned(pool->scales, 2))
        return fail(TC_ERR_ARG, "k_pool and v_pool must be 16-byte aligned, scales 2-byte");
    return TC_OK;
}

tc_status check_kvq_rows(const tc_plan *plan, const void *k_new, const void *v_new) {
    if (plan->append_shared) return fail(TC_ERR_BLOCK, "a block gets rows from more than one place of the block table");
    if (!k_new || !v_new) return fail(TC_ERR_NULL, "k_new or v_new is NULL");
    if (misaligned(k_new, 16) || misaligned(v_new, 16)) return fail(TC_ERR_ARG, "k_new and v_new must be 16-byte aligned");
    return TC_OK;
}

tc_status check_kvq_attention(const tc_plan *plan, const void *q, const void *out, float scale, const void *workspace, size_t workspace_bytes) {
    if (!q || !out) return fail(TC_ERR_NULL, "q or out is NULL");
    if (misaligned(q, 16) || misaligned(out, 16)) return fail(TC_ERR_ARG, "q and out must be 16-byte aligned");
    const size_t need = plan->workspace_bytes();
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(TC_ERR_WORKSPACE, "workspace missing or too small");
    if (need > 0 && misaligned(workspace, 16)) return fail(TC_ERR_ARG, "workspace must be 16-byte aligned");
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(TC_ERR_ARG, "scale must be positive and finite");
    return TC_OK;
}

}  // namespace

extern "C" {

tc_status tc_kvq_append(const tc_plan *plan, const tc_kvq_pool *pool, const void *k_new, const void *v_new, void *stream) {
    tc_status st = check_kvq(plan, pool);
    if (st != TC_OK || plan->T == 0) return st;
    if ((st = check_kvq_rows(plan, k_new, v_new)) != TC_OK || (st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_kvq_append(plan, pool, k_new, v_new, stream), "tc_kvq_append launch");
}

tc_status tc_kvq_read(const tc_plan *plan, const tc_kvq_pool *pool, int32_t seq, void *k_out, void *v_out, void *stream) {
    tc_status st = check_kvq(plan, pool);
    if (st != TC_OK) return st;
    int page0 = 0, n = 0;
    if (!selection(plan, seq, &page0, &n)) return fail(TC_ERR_ARG, "sequence index out of range");
    if (n == 0) return TC_OK;
    if (!k_out || !v_out) return fail(TC_ERR_NULL, "k_out or v_out is NULL");
    if (misaligned(k_out, 16) || misaligned(v_out, 16)) return fail(TC_ERR_ARG, "k_out and v_out must be 16-byte aligned");
    if (seq == -1) {
        int64_t tokens = plan->T;
        for (int s = 0; s < plan->S; s++) tokens += plan->ctx_len[s];
        if (tokens >= (int64_t)1 << 31) return fail(TC_ERR_ARG, "2^31 tokens or more: read the sequences one by one");
    }
    if ((st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_kvq_read(plan, pool, page0, n, k_out, v_out, stream), "tc_kvq_read launch");
}

tc_status tc_kvq_mixed_attention(const tc_plan *plan, const tc_kvq_pool *pool, const void *q, void *out, float scale, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    tc_status st = check_kvq(plan, pool);
    if (st != TC_OK || plan->T == 0) return st;
    if ((st = check_kvq_attention(plan, q, out, scale, workspace, workspace_bytes)) != TC_OK || (st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_kvq_attention(plan, pool, q, nullptr, nullptr, out, scale, workspace, stream), "tc_kvq_mixed_attention launch");
}

tc_status tc_kvq_mixed_attention_append(const tc_plan *plan, const tc_kvq_pool *pool, const void *q, const void *k_new, const void *v_new,
                                        void *out, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    tc_status st = check_kvq(plan, pool);
    if (st != TC_OK || plan->T == 0) return st;
    if ((st = check_kvq_rows(plan, k_new, v_new)) != TC_OK) return st;
    if ((st = check_kvq_attention(plan, q, out, scale, workspace, workspace_bytes)) != TC_OK || (st = check_plan_device(plan)) != TC_OK) return st;
    const bool apart = plan->append_apart;
    if (apart) {
        st = device_result(tc::launch_kvq_append(plan, pool, k_new, v_new, stream), "tc_kvq_mixed_attention_append launch");
        if (st != TC_OK) return st;
    }
    return device_result(tc::launch_kvq_attention(plan, pool, q, apart ? nullptr : k_new, apart ? nullptr : v_new, out, scale, workspace, stream),
                         "tc_kvq_mixed_attention_append launch");
}

}  // extern "C"

// ---- norm and rotation of the rows

namespace {

// Rows that are their own output lie as it does: a token would be written over the heads of another that are yet to be read.
tc_status check_own_output(const tc_plan *plan, const void *in, const void *out, int64_t stride, int heads) {
    if (in == out && plan->T > 1 && stride != (int64_t)heads * plan->D) return fail(TC_ERR_ARG, "rows that are their own output must be packed");
    return TC_OK;
}

tc_status check_rows(const tc_plan *plan, const tc_qkv_rows *rows, bool needs_v) {
    if (rows->rotary_dim < 0 || rows->rotary_dim > plan->D || rows->rotary_dim % 8)
        return fail(TC_ERR_SHAPE, "rotary_dim must be a multiple of 8 from 0 to head_dim");
    if (!rows->q || !rows->k || (needs_v && !rows->v)) return fail(TC_ERR_NULL, "q, k or v is NULL");
    if (rows->rotary_dim > 0 && !rows->freq) return fail(TC_ERR_NULL, "freq is NULL");
    if (misaligned(rows->q, 16) || misaligned(rows->k, 16) || (needs_v && misaligned(rows->v, 16)))
        return fail(TC_ERR_ARG, "q, k and v must be 16-byte aligned");
    if (misaligned(rows->q_weight, 16) || misaligned(rows->k_weight, 16) || misaligned(rows->freq, 8) || misaligned(rows->positions, 4))
        return fail(TC_ERR_ARG, "weights must be 16-byte aligned, freq 8-byte, positions 4-byte");
    const int64_t q_row = (int64_t)plan->Hq * plan->D, kv_row = (int64_t)plan->Hkv * plan->D;
    if (rows->q_stride < q_row || rows->k_stride < kv_row || (needs_v && rows->v_stride < kv_row))
        return fail(TC_ERR_ARG, "a stride is smaller than a token's heads");
    if (rows->q_stride % 8 || rows->k_stride % 8 || (needs_v && rows->v_stride % 8)) return fail(TC_ERR_ARG, "strides must be multiples of 8 elements");
    if ((rows->q_weight || rows->k_weight) && (!(rows->eps > 0.f) || rows->eps > 3.0e38f)) return fail(TC_ERR_ARG, "eps must be positive and finite");
    return TC_OK;
}

}  // namespace

extern "C" {

tc_status tc_qk_norm_rotate(const tc_plan *plan, const tc_qkv_rows *rows, void *q_out, void *k_out, void *stream) {
    if (!plan || !rows) return fail(TC_ERR_NULL, "plan or rows is NULL");
    if (plan->T == 0) return TC_OK;
    tc_status st = check_rows(plan, rows, false);
    if (st != TC_OK) return st;
    if (!q_out || !k_out) return fail(TC_ERR_NULL, "q_out or k_out is NULL");
    if (misaligned(q_out, 16) || misaligned(k_out, 16)) return fail(TC_ERR_ARG, "q_out and k_out must be 16-byte aligned");
    if ((st = check_own_output(plan, rows->q, q_out, rows->q_stride, plan->Hq)) != TC_OK || (st = check_own_output(plan, rows->k, k_out, rows->k_stride, plan->Hkv)) != TC_OK) return st;
    if ((st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_rows(plan, nullptr, rows, q_out, k_out, stream), "tc_qk_norm_rotate launch");
}

tc_status tc_qk_norm_rotate_append(const tc_plan *plan, const tc_kv_pool *pool, const tc_qkv_rows *rows, void *q_out, void *stream) {
    if (!rows) return fail(TC_ERR_NULL, "rows is NULL");
    tc_status st = tc::check_pool_matches(plan, pool, true);
    if (st != TC_OK || plan->T == 0) return st;
    if ((st = check_rows(plan, rows, true)) != TC_OK) return st;
    if (!q_out) return fail(TC_ERR_NULL, "q_out is NULL");
    if (misaligned(q_out, 16)) return fail(TC_ERR_ARG, "q_out must be 16-byte aligned");
    if ((st = check_own_output(plan, rows->q, q_out, rows->q_stride, plan->Hq)) != TC_OK) return st;
    if (misaligned(pool->k_pool, 16) || misaligned(pool->v_pool, 16)) return fail(TC_ERR_ARG, "k_pool and v_pool must be 16-byte aligned");
    if ((st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_rows(plan, pool, rows, q_out, nullptr, stream), "tc_qk_norm_rotate_append launch");
}

}  // extern "C"

// ---- attention over spans

namespace {

tc_status span_attention(const tc_plan *plan, const tc::SpanList &list, const tc_kv_pool *pool, const void *q, void *out, float scale, void *workspace, size_t workspace_bytes,
                         void *stream, const char *no_list, const char *what) {
    tc_status st = tc::check_pool_matches(plan, pool, true);
    if (st != TC_OK || plan->T == 0) return st;
    if (!list.ready) return fail(TC_ERR_ARG, no_list);
    if (!q || !out) return fail(TC_ERR_NULL, "q or out is NULL");
    if (misaligned(q, 16) || misaligned(out, 16)) return fail(TC_ERR_ARG, "q and out must be 16-byte aligned");
    if (misaligned(pool->k_pool, 16) || misaligned(pool->v_pool, 16)) return fail(TC_ERR_ARG, "k_pool and v_pool must be 16-byte aligned");
    const size_t need = plan->span_workspace_bytes(list);
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(TC_ERR_WORKSPACE, "workspace missing or too small");
    if (need > 0 && misaligned(workspace, 16)) return fail(TC_ERR_ARG, "workspace must be 16-byte aligned");
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(TC_ERR_ARG, "scale must be positive and finite");
    if ((st = check_plan_device(plan)) != TC_OK) return st;
    return device_result(tc::launch_span(plan, list, pool, q, out, scale, workspace, stream), what);
}

}  // namespace

extern "C" {

tc_status tc_window_attention(const tc_plan *plan, const tc_kv_pool *pool, const void *q, void *out, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    if (!plan) return fail(TC_ERR_NULL, "plan is NULL");
    return span_attention(plan, plan->window, pool, q, out, scale, workspace, workspace_bytes, stream, "the plan has no window for its batch: tc_plan_set_window first",
                          "tc_window_attention launch");
}

tc_status tc_shared_attention(const tc_plan *plan, const tc_kv_pool *pool, const void *q, void *out, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    if (!plan) return fail(TC_ERR_NULL, "plan is NULL");
    return span_attention(plan, plan->shared, pool, q, out, scale, workspace, workspace_bytes, stream, "the plan has no groups for its batch: tc_plan_set_shared first",
                          "tc_shared_attention launch");
}

}  // extern "C"
