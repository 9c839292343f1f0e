// C ABI of the paged key/value cache (declared in include/sim_kv.h): argument checks and launches.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "sim.h"
#include "sim_kv.h"
#include "sim_kv_internal.h"

namespace simgb {
void set_global_error(const char *msg);
}

namespace {

int fail(int code, const char *fmt, ...) noexcept {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    try {
        simgb::set_global_error(buf);
    } catch (...) {  // no memory for the message
    }
    return code;
}

int done(cudaError_t e, const char *what) {
    if (e == cudaSuccess) return SIM_OK;
    cudaGetLastError();  // reported here, not again by the next launch
    return fail(SIM_E_CUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

bool aligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Null, or what is wrong with the sizes.
const char *bad_sizes(const sim_kv *kv) {
    if (!kv) return "NULL cache";
    if (kv->dtype != SIM_KV_BF16 && kv->dtype != SIM_KV_F16) return "dtype must be SIM_KV_BF16 or SIM_KV_F16";
    if (kv->n_pages < 1 || kv->n_pages > 1 << 28) return "n_pages outside [1, 2^28]";
    if (kv->n_layers < 1 || kv->n_layers > 1 << 16 || kv->n_kv_heads < 1 || kv->n_kv_heads > 1 << 16) return "n_layers and n_kv_heads must be in [1, 2^16]";
    if (kv->page_size != 16 && kv->page_size != 32 && kv->page_size != 64 && kv->page_size != 128) return "page_size must be 16, 32, 64 or 128";
    if (kv->head_dim < 8 || kv->head_dim > 128 || kv->head_dim % 8) return "head_dim must be a multiple of 8 in [8, 128]";
    if (kv->max_seqs < 1 || kv->max_seqs > simgb::kKvMaxSeqs) return "max_seqs outside [1, 2^17]";
    if (kv->max_pages < 1 || int64_t(kv->max_pages) * kv->page_size >= 1 << 30) return "max_pages < 1 or max_pages * page_size >= 2^30";
    if (int64_t(kv->max_pages) * kv->page_size * kv->n_kv_heads >= int64_t(1) << 37) return "max_pages * page_size * n_kv_heads >= 2^37";
    if (simgb::kv_page_bytes(*kv) >= int64_t(1) << 40) return "a page of 2^40 bytes or more";
    return nullptr;
}

const char *bad_cache(const sim_kv *kv) {
    if (const char *m = bad_sizes(kv)) return m;
    if (!kv->pool || !kv->table || !kv->length || !kv->ref || !kv->status || !kv->scratch) return "NULL array in the cache";
    if (!aligned(kv->pool, 16) || !aligned(kv->ref, 16) || !aligned(kv->scratch, 16)) return "pool, ref and scratch must be 16-byte aligned";
    return nullptr;
}

const char *bad_batch_sizes(const sim_kv *kv, const sim_kv_batch *b) {
    if (const char *m = bad_sizes(kv)) return m;
    if (!b) return "NULL batch";
    if (b->n < 0 || b->n > simgb::kKvMaxSeqs || b->n_groups < 0 || b->n_groups > b->n) return "n outside [0, 2^17] or n_groups outside [0, n]";
    if (b->q_heads < 1 || b->q_heads % kv->n_kv_heads) return "q_heads must be a positive multiple of n_kv_heads";
    if (int64_t(b->n) * kv->n_kv_heads > 1 << 26) return "n * n_kv_heads > 2^26";
    if (b->n_q < 0 || int64_t(b->n_q) * b->q_heads > 1 << 30) return "n_q < 0 or n_q * q_heads > 2^30";
    return nullptr;
}

const char *bad_batch(const sim_kv *kv, const sim_kv_batch *b) {
    if (const char *m = bad_cache(kv)) return m;
    if (const char *m = bad_batch_sizes(kv, b)) return m;
    if (!b->cu_q || (b->n > 0 && !b->seqs) || (b->n_groups > 0 && !b->cu_group)) return "NULL array in the batch";
    if (!b->plan || !b->workspace || !aligned(b->plan, 16) || !aligned(b->workspace, 16)) return "plan and workspace must be 16-byte aligned and not NULL";
    return nullptr;
}

const char *bad_entries(const sim_kv *kv, int32_t n, const void *a, const void *b) {
    if (const char *m = bad_cache(kv)) return m;
    if (n < 0 || n > kv->max_seqs) return "n outside [0, max_seqs]";
    if (n > 0 && (!a || !b)) return "NULL list of entries";
    return nullptr;
}

}  // namespace

extern "C" {

int64_t sim_kv_scratch_bytes(const sim_kv *kv) { return bad_sizes(kv) ? 0 : simgb::kv_scratch_ints(*kv) * 4; }

int sim_kv_extend(const sim_kv *kv, int32_t n, const int32_t *seqs, const int32_t *cu_new, int32_t n_new, int64_t *slots,
                  void *cuda_stream) {
    if (const char *m = bad_entries(kv, n, seqs, cu_new)) return fail(SIM_E_INVAL, "sim_kv_extend: %s", m);
    if (n_new < 0 || (n_new > 0 && !slots)) return fail(SIM_E_INVAL, "sim_kv_extend: n_new < 0 or NULL slots");
    if (n == 0 && n_new == 0) return SIM_OK;
    if (!cu_new) return fail(SIM_E_INVAL, "sim_kv_extend: NULL offsets");
    return done(simgb::launch_kv_extend(*kv, n, seqs, cu_new, n_new, slots, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_extend");
}

int sim_kv_write(const sim_kv *kv, int32_t layer, int32_t n_new, const int64_t *slots, const void *k, int64_t k_token_stride,
                 int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, void *cuda_stream) {
    if (const char *m = bad_cache(kv)) return fail(SIM_E_INVAL, "sim_kv_write: %s", m);
    if (layer < 0 || layer >= kv->n_layers || n_new < 0) return fail(SIM_E_INVAL, "sim_kv_write: layer outside the cache or n_new < 0");
    if (n_new == 0) return SIM_OK;
    if (!slots || !k || !v || !aligned(k, 2) || !aligned(v, 2)) return fail(SIM_E_INVAL, "sim_kv_write: NULL or odd pointer");
    const simgb::KvWrite w = {k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots, layer, n_new};
    return done(simgb::launch_kv_write(*kv, w, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_write");
}

int sim_kv_fork(const sim_kv *kv, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *tokens, void *cuda_stream) {
    if (const char *m = bad_entries(kv, n, src, dst)) return fail(SIM_E_INVAL, "sim_kv_fork: %s", m);
    if (n == 0) return SIM_OK;
    return done(simgb::launch_kv_fork(*kv, n, src, dst, tokens, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_fork");
}

int sim_kv_copy(const sim_kv *kv, int32_t n, const int32_t *src, const int32_t *dst, void *cuda_stream) {
    if (const char *m = bad_entries(kv, n, src, dst)) return fail(SIM_E_INVAL, "sim_kv_copy: %s", m);
    if (n == 0) return SIM_OK;
    return done(simgb::launch_kv_copy(*kv, n, src, dst, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_copy");
}

int sim_kv_free(const sim_kv *kv, int32_t n, const int32_t *seqs, const int32_t *keep, void *cuda_stream) {
    if (const char *m = bad_entries(kv, n, seqs, seqs)) return fail(SIM_E_INVAL, "sim_kv_free: %s", m);
    if (n == 0) return SIM_OK;
    return done(simgb::launch_kv_free(*kv, n, seqs, keep, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_free");
}

int sim_kv_compact(const sim_kv *kv, int32_t *to, void *cuda_stream) {
    if (const char *m = bad_cache(kv)) return fail(SIM_E_INVAL, "sim_kv_compact: %s", m);
    if (!to) return fail(SIM_E_INVAL, "sim_kv_compact: NULL list");
    return done(simgb::launch_kv_compact(*kv, to, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_compact");
}

int64_t sim_kv_plan_bytes(const sim_kv *kv, const sim_kv_batch *b) { return bad_batch_sizes(kv, b) ? 0 : (simgb::kv_plan(*kv, *b).bytes + 15) / 16 * 16; }

int64_t sim_kv_workspace_bytes(const sim_kv *kv, const sim_kv_batch *b) {
    return bad_batch_sizes(kv, b) ? 0 : simgb::kv_partial_rows(*b, simgb::kv_sm_count()) * (kv->head_dim + 1) * 4;
}

int sim_kv_plan(const sim_kv *kv, const sim_kv_batch *b, void *cuda_stream) {
    if (const char *m = bad_batch(kv, b)) return fail(SIM_E_INVAL, "sim_kv_plan: %s", m);
    return done(simgb::launch_kv_plan(*kv, *b, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_plan");
}

int sim_kv_attend(const sim_kv *kv, const sim_kv_batch *b, int32_t layer, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                  float scale, void *out, int64_t out_token_stride, int64_t out_head_stride, float *lse, void *cuda_stream) {
    if (const char *m = bad_batch(kv, b)) return fail(SIM_E_INVAL, "sim_kv_attend: %s", m);
    if (layer < 0 || layer >= kv->n_layers) return fail(SIM_E_INVAL, "sim_kv_attend: layer %d outside [0, %d)", layer, kv->n_layers);
    if (!(scale > 0.f) || !std::isfinite(scale * 1.44269504088896341f)) return fail(SIM_E_INVAL, "sim_kv_attend: scale must be positive and finite");
    if (b->n_q == 0) return SIM_OK;
    if (!q || !out || !aligned(q, 2)) return fail(SIM_E_INVAL, "sim_kv_attend: NULL or odd pointer");
    if (!aligned(out, 16) || out_token_stride % 8 || out_head_stride % 8)
        return fail(SIM_E_INVAL, "sim_kv_attend: out must be 16-byte aligned with strides that are multiples of 8");
    simgb::KvAttend a = {};
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.sms = simgb::kv_sm_count();
    a.group = simgb::FastDiv(uint32_t(b->q_heads / kv->n_kv_heads));
    a.part = static_cast<float *>(b->workspace);
    a.part_lse = a.part + simgb::kv_partial_rows(*b, a.sms) * kv->head_dim;
    a.qt = q_token_stride;
    a.qh = q_head_stride;
    a.ot = out_token_stride;
    a.oh = out_head_stride;
    a.scale_log2 = scale * 1.44269504088896341f;
    a.layer = layer;
    a.q_vec = aligned(q, 16) && q_token_stride % 8 == 0 && q_head_stride % 8 == 0;
    return done(simgb::launch_kv_attend(*kv, *b, a, static_cast<cudaStream_t>(cuda_stream)), "sim_kv_attend");
}

}  // extern "C"
