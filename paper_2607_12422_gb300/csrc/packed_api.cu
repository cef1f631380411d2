// packed_api.cu -- C entry points (include/pbd_ops.h) of the operators that bring prompts and drafted trees into a caller's
// paged cache: argument checks, workspaces and launches.
#include <cuda_runtime.h>

#include <algorithm>

#include "kv_checks.h"
#include "packed_ops.h"

using namespace pbd;
using namespace pbd::checks;

namespace {

// What is wrong with packed rows of queries, keys and values, or null.
const char *bad_rows_of(int T, int batch, int hq, int hkv, int D, int64_t q_stride, int64_t kv_stride) {
    if (T < 1 || T > (1 << 30)) return "T must be 1 to 2^30";
    if (batch < 1 || batch > KV_MAX_BATCH) return "batch must be 1 to 1024";
    if (hkv < 1 || hkv > 256) return "n_kv_heads must be 1 to 256";
    if (hq < hkv || hq % hkv || hq > 4096) return "n_q_heads must be a multiple of n_kv_heads, at most 4096";
    if (D != 64 && D != 128 && D != 256) return "head_dim must be 64, 128 or 256";
    if (q_stride < (int64_t)hq * D || q_stride % 8 || kv_stride < (int64_t)hkv * D || kv_stride % 8)
        return "row strides must be multiples of 8 values and hold a row";
    // (tensor maps hold strides below 2^40 bytes)
    if (q_stride >= (1ll << 38) || kv_stride >= (1ll << 38)) return "row strides must be below 2^38 values";
    if (!addressable(T, q_stride) || !addressable(T, kv_stride)) return "rows reach further than 2^60 values";
    return nullptr;
}

long long rows_span(int T, int64_t stride, int heads, int D) { return 2 * ((T - 1) * stride + (long long)heads * D); }

}  // namespace

extern "C" {

size_t pbd_op_assign_pages_workspace_bytes(int32_t batch) { return batch < 1 || batch > KV_MAX_BATCH ? 0 : 1024; }

pbd_status pbd_op_assign_pages(int32_t batch, int32_t max_pages, int32_t page_size, int32_t n_pages, const int32_t *d_lens,
                               const int32_t *d_n_new, int32_t *d_page_table, int32_t *d_held, int32_t *d_free,
                               int32_t *d_n_free, int32_t max_new, int32_t *d_starts, int64_t *d_slots,
                               int32_t *d_positions_opt, void *d_ws, size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_assign_pages";
    if (batch < 1 || batch > KV_MAX_BATCH) return fail(PBD_ERR_INVALID_ARG, who, "batch must be 1 to 1024");
    if (n_pages < 1 || page_size < 1 || max_pages < 1) return fail(PBD_ERR_INVALID_ARG, who, "n_pages, page_size and max_pages must be positive");
    if ((long long)max_pages * page_size > (1ll << 30)) return fail(PBD_ERR_INVALID_ARG, who, "a sequence holds at most 2^30 slots");
    if (max_new < 0 || max_new > (1 << 30)) return fail(PBD_ERR_INVALID_ARG, who, "max_new must be 0 to 2^30");
    if (!d_lens || !d_n_new || !d_page_table || !d_held || !d_free || !d_n_free || !d_starts || (max_new && !d_slots))
        return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!aligned(d_lens, 4) || !aligned(d_n_new, 4) || !aligned(d_page_table, 4) || !aligned(d_held, 4) || !aligned(d_free, 4) ||
        !aligned(d_n_free, 4) || !aligned(d_starts, 4) || !aligned(d_positions_opt, 4))
        return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    if (!aligned(d_slots, 8)) return fail(PBD_ERR_INVALID_ARG, who, "the slots must be 8-byte aligned");
    if (const char *w = bad_workspace(d_ws, ws_bytes, 1024)) return fail(PBD_ERR_WORKSPACE, who, w);
    Ranges mem;
    mem.add("the lengths", d_lens, 4ll * batch, false);
    mem.add("the new tokens' numbers", d_n_new, 4ll * batch, false);
    mem.add("the page table", d_page_table, 4ll * batch * max_pages, true);
    mem.add("the held pages' numbers", d_held, 4ll * batch, true);
    mem.add("the free pages", d_free, 4ll * n_pages, true);
    mem.add("the free pages' number", d_n_free, 4, true);
    mem.add("the starts", d_starts, 4ll * (batch + 1), true);
    mem.add("the slots", max_new ? d_slots : nullptr, 8ll * max_new, true);
    mem.add("the positions", max_new ? d_positions_opt : nullptr, 4ll * max_new, true);
    mem.add("the workspace", d_ws, 1024, true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    AssignArgs a{};
    a.lens = d_lens;
    a.n_new = d_n_new;
    a.table = d_page_table;
    a.held = d_held;
    a.free_list = d_free;
    a.n_free = d_n_free;
    a.B = batch;
    a.max_pages = max_pages;
    a.page_size = page_size;
    a.n_pages = n_pages;
    a.max_new = max_new;
    a.cap = (long long)max_pages * page_size;
    a.starts = d_starts;
    a.slots = reinterpret_cast<long long *>(d_slots);
    a.positions = d_positions_opt;
    a.status = static_cast<int *>(d_ws);
    const cudaError_t e = launch_assign_pages(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

size_t pbd_op_prompt_attention_workspace_bytes(int32_t T, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t head_dim) {
    if (bad_rows_of(T, batch, n_q_heads, n_kv_heads, head_dim, (int64_t)n_q_heads * head_dim, (int64_t)n_kv_heads * head_dim)) return 0;
    return 1024;
}

pbd_status pbd_op_prompt_attention(int32_t T, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                   int32_t dtype, float scale, const void *d_q, int64_t q_stride, const void *d_k,
                                   const void *d_v, int64_t kv_stride, const int32_t *d_starts, const pbd_kv_pages *kv_opt,
                                   const int64_t *d_slots_opt, void *d_out, float *d_lse_opt, void *d_ws, size_t ws_bytes,
                                   void *d_stream) {
    const char *who = "pbd_op_prompt_attention";
    if (const char *w = bad_rows_of(T, batch, n_q_heads, n_kv_heads, head_dim, q_stride, kv_stride)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (dtype != PBD_BF16 && dtype != PBD_FP16) return fail(PBD_ERR_INVALID_ARG, who, "the type must be PBD_BF16 or PBD_FP16");
    if (!usable_factor(scale)) return fail(PBD_ERR_INVALID_ARG, who, "scale must be positive and finite");
    if (!d_q || !d_k || !d_v || !d_starts || !d_out) return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_out, 16))
        return fail(PBD_ERR_INVALID_ARG, who, "q, k, v and out must be 16-byte aligned");
    if (!aligned(d_starts, 4) || !aligned(d_lse_opt, 4)) return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    if (!kv_opt != !d_slots_opt) return fail(PBD_ERR_INVALID_ARG, who, "a cache and slots come together");
    if (kv_opt) {
        if (const char *w = bad_cache(kv_opt)) return fail(PBD_ERR_INVALID_ARG, who, w);
        if (kv_opt->dtype != dtype || kv_opt->head_dim != head_dim || kv_opt->n_kv_heads != n_kv_heads)
            return fail(PBD_ERR_INVALID_ARG, who, "the cache's type, head_dim or n_kv_heads are not k's and v's");
        if (const char *w = bad_rows(kv_opt)) return fail(PBD_ERR_INVALID_ARG, who, w);
        if (!aligned(d_slots_opt, 8)) return fail(PBD_ERR_INVALID_ARG, who, "the slots must be 8-byte aligned");
    }
    const size_t need = pbd_op_prompt_attention_workspace_bytes(T, batch, n_q_heads, n_kv_heads, head_dim);
    if (const char *w = bad_workspace(d_ws, ws_bytes, need)) return fail(PBD_ERR_WORKSPACE, who, w);
    if (const char *w = kv_opt ? k_over_v(kv_opt) : nullptr) return fail(PBD_ERR_INVALID_ARG, who, w);
    Ranges mem;
    if (kv_opt) mem.cache(kv_opt, true);
    mem.add("the slots", d_slots_opt, 8ll * T, false);
    mem.add("q", d_q, rows_span(T, q_stride, n_q_heads, head_dim), false);
    mem.add("k", d_k, rows_span(T, kv_stride, n_kv_heads, head_dim), false);
    mem.add("v", d_v, rows_span(T, kv_stride, n_kv_heads, head_dim), false);
    mem.add("the starts", d_starts, 4ll * (batch + 1), false);
    mem.add("out", d_out, 2ll * T * n_q_heads * head_dim, true);
    mem.add("lse", d_lse_opt, 4ll * T * n_q_heads, true);
    mem.add("the workspace", d_ws, (long long)need, true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    PackedArgs a{};
    if (kv_opt) a.kv = view(*kv_opt);
    a.T = T;
    a.B = batch;
    a.hq = n_q_heads;
    a.hkv = n_kv_heads;
    a.group = n_q_heads / n_kv_heads;
    a.d = head_dim;
    a.fp16 = dtype == PBD_FP16;
    a.scale = scale;
    a.q = static_cast<const uint16_t *>(d_q);
    a.k = static_cast<const uint16_t *>(d_k);
    a.v = static_cast<const uint16_t *>(d_v);
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.starts = d_starts;
    a.slots = reinterpret_cast<const long long *>(d_slots_opt);
    a.out = static_cast<uint16_t *>(d_out);
    a.lse = d_lse_opt;
    a.status = static_cast<int *>(d_ws);
    const cudaError_t e = launch_prompt_attention(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

size_t pbd_op_tree_attention_workspace_bytes(const pbd_kv_pages *kv, int32_t T, int32_t n_q_heads) {
    TreePlan p;
    if (bad_sizes(kv) || bad_heads(kv, n_q_heads) || T < 1 || T > (1 << 30) || !tree_plan(view(*kv), T, n_q_heads, &p)) return 0;
    return p.total;
}

pbd_status pbd_op_tree_attention(const pbd_kv_pages *kv, int32_t T, int32_t n_q_heads, float scale, const void *d_q,
                                 int64_t q_stride, const void *d_k_new, const void *d_v_new, int64_t new_stride,
                                 const int32_t *d_starts, const int32_t *d_parents_opt, const int32_t *d_new_positions_opt,
                                 void *d_out, float *d_lse_opt, void *d_ws, size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_tree_attention";
    if (const char *w = bad_cache(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (const char *w = bad_rows(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    const int D = kv->head_dim, B = kv->batch, hkv = kv->n_kv_heads;
    if (const char *w = bad_rows_of(T, B, n_q_heads, hkv, D, q_stride, new_stride)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (!usable_factor(scale)) return fail(PBD_ERR_INVALID_ARG, who, "scale must be positive and finite");
    if (!d_q || !d_k_new || !d_v_new || !d_starts || !d_out) return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!aligned(d_q, 16) || !aligned(d_k_new, 16) || !aligned(d_v_new, 16) || !aligned(d_out, 16))
        return fail(PBD_ERR_INVALID_ARG, who, "q, k_new, v_new and out must be 16-byte aligned");
    if (!aligned(d_starts, 4) || !aligned(d_parents_opt, 4) || !aligned(d_new_positions_opt, 4) || !aligned(d_lse_opt, 4))
        return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    TreePlan p;
    const KvView v = view(*kv);
    if (!tree_plan(v, T, n_q_heads, &p)) return fail(PBD_ERR_CAPACITY, who, "the table has room for more places than the list holds (2^31 - 2; pbd_ops.h)");
    const size_t need = p.total;
    if (const char *w = bad_workspace(d_ws, ws_bytes, need)) return fail(PBD_ERR_WORKSPACE, who, w);
    if (const char *w = k_over_v(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    Ranges mem;
    mem.cache(kv, true);
    mem.add("q", d_q, rows_span(T, q_stride, n_q_heads, D), false);
    mem.add("k_new", d_k_new, rows_span(T, new_stride, hkv, D), false);
    mem.add("v_new", d_v_new, rows_span(T, new_stride, hkv, D), false);
    mem.add("the starts", d_starts, 4ll * (B + 1), false);
    mem.add("the parents", d_parents_opt, 4ll * T, false);
    if (d_new_positions_opt) {
        mem.add("new_positions", d_new_positions_opt, 4ll * T, false);
        mem.add("the positions", kv->d_positions, 4ll * B * hkv * v.cap, true);
    }
    mem.add("out", d_out, 2ll * T * n_q_heads * D, true);
    mem.add("lse", d_lse_opt, 4ll * T * n_q_heads, true);
    mem.add("the workspace", d_ws, (long long)need, true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    PackedArgs a{};
    a.kv = v;
    a.T = T;
    a.B = B;
    a.hq = n_q_heads;
    a.hkv = hkv;
    a.group = n_q_heads / hkv;
    a.d = D;
    a.fp16 = kv->dtype == PBD_FP16;
    a.scale = scale;
    a.q = static_cast<const uint16_t *>(d_q);
    a.k = static_cast<const uint16_t *>(d_k_new);
    a.v = static_cast<const uint16_t *>(d_v_new);
    a.q_stride = q_stride;
    a.kv_stride = new_stride;
    a.starts = d_starts;
    a.parents = d_parents_opt;
    a.new_pos = d_new_positions_opt;
    a.out = static_cast<uint16_t *>(d_out);
    a.lse = d_lse_opt;
    uint8_t *ws = static_cast<uint8_t *>(d_ws);
    a.status = reinterpret_cast<int *>(ws);
    a.part_rows = p.rows;
    a.worker_code = reinterpret_cast<int *>(ws + p.codes);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o);
    const cudaError_t e = launch_tree_attention(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

size_t pbd_op_commit_path_workspace_bytes(const pbd_kv_pages *kv, int32_t max_path) {
    return bad_sizes(kv) || max_path < 1 || max_path > TREE_NODES ? 0 : 1024;
}

pbd_status pbd_op_commit_path(const pbd_kv_pages *kv, const int32_t *d_path, int32_t max_path, const int32_t *d_n_accepted,
                              void *d_ws, size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_commit_path";
    if (const char *w = bad_cache(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (const char *w = bad_rows(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (max_path < 1 || max_path > TREE_NODES) return fail(PBD_ERR_INVALID_ARG, who, "max_path must be 1 to 64");
    if (!d_path || !d_n_accepted) return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!aligned(d_path, 4) || !aligned(d_n_accepted, 4)) return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    if (const char *w = bad_workspace(d_ws, ws_bytes, 1024)) return fail(PBD_ERR_WORKSPACE, who, w);
    if (const char *w = k_over_v(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    const KvView v = view(*kv);
    const long long slots = 4ll * v.B * v.hkv * v.cap;
    Ranges mem;
    mem.cache(kv, true);
    mem.add("the weights", kv->d_weights, slots, true);
    mem.add("the positions", kv->d_positions, slots, true);
    mem.add("the path", d_path, 4ll * v.B * max_path, false);
    mem.add("the accepted numbers", d_n_accepted, 4ll * v.B, false);
    mem.add("the workspace", d_ws, 1024, true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    CommitArgs a{};
    a.kv = v;
    a.path = d_path;
    a.n_accepted = d_n_accepted;
    a.max_path = max_path;
    a.status = static_cast<int *>(d_ws);
    const cudaError_t e = launch_commit_path(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

}  // extern "C"
