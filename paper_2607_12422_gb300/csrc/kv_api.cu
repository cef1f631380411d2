// kv_api.cu -- C entry points (include/pbd_ops.h) of the operators on a caller's paged cache and on logits: argument
// checks, workspace plans and launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "../../include/pbd_ops.h"
#include "kv_ops.h"

using namespace pbd;

namespace {

pbd_status fail(pbd_status s, const char *who, const char *what, cudaError_t e = cudaSuccess) {
    char b[256];
    snprintf(b, sizeof b, "%s: %s%s%s", who, what, e != cudaSuccess ? ": " : "", e != cudaSuccess ? cudaGetErrorString(e) : "");
    op_record_error(b);
    return s;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The exponents' factor, which kernels hold with log2 e in it, is finite too.
bool usable_factor(float f) { return f > 0.f && !std::isinf(f * 1.4426950408889634f); }

bool overlap(const void *a, long long na, const void *b, long long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Whether `n` rows `stride` values apart can be addressed: byte offsets and spans stay below 2^63.
bool addressable(long long n, long long stride) { return n <= 1 || stride <= (1ll << 60) / (n - 1); }

// What is wrong with a cache's sizes and strides, or null.  Pointers are looked at by the entry points: workspace sizes
// are asked for before there are any.
const char *bad_sizes(const pbd_kv_pages *kv) {
    if (!kv) return "null cache";
    if (kv->dtype != PBD_BF16 && kv->dtype != PBD_FP16) return "the cache's type must be PBD_BF16 or PBD_FP16";
    if (kv->batch < 1 || kv->batch > KV_MAX_BATCH) return "batch must be 1 to 1024";
    if (kv->n_kv_heads < 1 || kv->n_kv_heads > 256) return "n_kv_heads must be 1 to 256";
    if (kv->head_dim != 64 && kv->head_dim != 128 && kv->head_dim != 256) return "head_dim must be 64, 128 or 256";
    if (kv->n_pages < 1 || kv->page_size < 1 || kv->max_pages < 1) return "n_pages, page_size and max_pages must be positive";
    if ((long long)kv->max_pages * kv->page_size > (1ll << 30)) return "a sequence holds at most 2^30 slots";
    if (kv->stride_page < 0 || kv->stride_head < 0 || kv->stride_slot < 0 || kv->stride_page % 8 || kv->stride_head % 8 ||
        kv->stride_slot % 8)
        return "strides must be multiples of 8 values and not negative";
    if (!addressable(kv->n_pages, kv->stride_page) || !addressable(kv->n_kv_heads, kv->stride_head) || !addressable(kv->page_size, kv->stride_slot))
        return "strides reach further than 2^60 values";
    return nullptr;
}

const char *bad_cache(const pbd_kv_pages *kv) {
    if (const char *w = bad_sizes(kv)) return w;
    if (!kv->d_k || !kv->d_v || !kv->d_page_table || !kv->d_lens) return "null pointer in the cache";
    if (!aligned(kv->d_k, 16) || !aligned(kv->d_v, 16)) return "K and V must be 16-byte aligned";
    if (!aligned(kv->d_page_table, 4) || !aligned(kv->d_lens, 4) || !aligned(kv->d_weights, 4) || !aligned(kv->d_positions, 4))
        return "the cache's 32-bit arrays must be 4-byte aligned";
    return nullptr;
}

// The dimensions of K or V with more than one place, the smallest stride first; below[i]: what a place of it spans.
struct Places {
    int n = 0;
    long long extent[3], stride[3], below[4];
    explicit Places(const pbd_kv_pages *kv) {
        const long long all[3][2] = {{kv->n_pages, kv->stride_page}, {kv->n_kv_heads, kv->stride_head}, {kv->page_size, kv->stride_slot}};
        for (const auto &x : all) {
            if (x[0] < 2) continue;
            int i = n++;
            for (; i > 0 && stride[i - 1] > x[1]; --i) extent[i] = extent[i - 1], stride[i] = stride[i - 1];
            extent[i] = x[0];
            stride[i] = x[1];
        }
        below[0] = kv->head_dim;
        for (int i = 0; i < n; ++i) below[i + 1] = below[i] + (extent[i] - 1) * stride[i];
    }
    // whether rows lie apart by strides alone: each stride is at least what the dimensions below it span
    bool apart() const {
        for (int i = 0; i < n; ++i)
            if (stride[i] < below[i]) return false;
        return true;
    }
    // whether a row and one of the same rows moved by `off` values meet (rows lie apart): only the two multiples of a stride
    // next to `off` can bring it within what lies below
    bool meet(long long off, int dims) const {
        if (dims == 0) return off > -below[0] && off < below[0];
        const long long s = stride[dims - 1], q = off / s, most = extent[dims - 1] - 1;
        for (long long a = q - 1; a <= q + 1; ++a)
            if (a >= -most && a <= most && meet(off - a * s, dims - 1)) return true;
        return false;
    }
};

// Calls that write K and V: rows must not lie over one another, nor K's over V's.
const char *bad_rows(const pbd_kv_pages *kv) {
    const int D = kv->head_dim;
    if ((kv->page_size > 1 && kv->stride_slot < D) || (kv->n_kv_heads > 1 && kv->stride_head < D) || (kv->n_pages > 1 && kv->stride_page < D))
        return "a cache that is written to has strides of a row or more";
    const Places p(kv);
    if (!p.apart()) return "the rows of a cache that is written to lie over one another";
    return nullptr;
}
const char *k_over_v(const pbd_kv_pages *kv) {
    const Places p(kv);
    const long long off = (long long)(reinterpret_cast<uintptr_t>(kv->d_v) - reinterpret_cast<uintptr_t>(kv->d_k)) / 2;
    return p.meet(off, p.n) ? "K and V of a cache that is written to lie over one another" : nullptr;
}

// bytes from the first value of K (or V) to the last
long long cache_span(const pbd_kv_pages *kv) {
    return 2 * ((kv->n_pages - 1) * kv->stride_page + (kv->n_kv_heads - 1) * kv->stride_head +
                (kv->page_size - 1) * kv->stride_slot + kv->head_dim);
}

// What a call reads and writes: nothing that it writes lies over anything else of it.  (K over V is k_over_v's.)
class Ranges {
    struct Range {
        const void *p;
        long long bytes;
        const char *name;
        bool written;
    } r[16];
    int n = 0;
    bool has_cache = false;  // (its K and V come first)
    char text[96];

public:
    void add(const char *name, const void *p, long long bytes, bool written) {
        if (p && n < 16) r[n++] = Range{p, bytes, name, written};
    }
    void cache(const pbd_kv_pages *kv, bool written) {
        has_cache = true;
        add("K", kv->d_k, cache_span(kv), written);
        add("V", kv->d_v, cache_span(kv), written);
        add("the page table", kv->d_page_table, 4ll * kv->batch * kv->max_pages, false);
        add("the lengths", kv->d_lens, 4ll * kv->batch, false);
    }
    const char *clash() {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j) {
                if (i == j || !r[i].written || !overlap(r[i].p, r[i].bytes, r[j].p, r[j].bytes)) continue;
                if (has_cache && i < 2 && j < 2) continue;
                snprintf(text, sizeof text, "%s, which the call writes, lies over %s", r[i].name, r[j].name);
                return text;
            }
        return nullptr;
    }
};

KvView view(const pbd_kv_pages &kv) {
    KvView v{};
    v.k = static_cast<const uint16_t *>(kv.d_k);
    v.v = static_cast<const uint16_t *>(kv.d_v);
    v.stride_page = kv.stride_page;
    v.stride_head = kv.stride_head;
    v.stride_slot = kv.stride_slot;
    v.table = kv.d_page_table;
    v.lens = kv.d_lens;
    v.weights = kv.d_weights;
    v.positions = kv.d_positions;
    v.cap = (long long)kv.max_pages * kv.page_size;
    v.n_pages = kv.n_pages;
    v.page_size = kv.page_size;
    v.hkv = kv.n_kv_heads;
    v.d = kv.head_dim;
    v.B = kv.batch;
    v.max_pages = kv.max_pages;
    // slot * mul / 2^shift is above slot / page_size by less than slot / 2^shift < 2^30 / (2^30 page_size): never in the next page
    v.page_shift = 30;
    while ((1ll << (v.page_shift - 30)) < kv.page_size) ++v.page_shift;
    v.page_mul = (uint32_t)(((1ull << v.page_shift) + kv.page_size - 1) / kv.page_size);
    return v;
}

const char *bad_heads(const pbd_kv_pages *kv, int hq) {
    if (hq < kv->n_kv_heads || hq % kv->n_kv_heads || hq > 4096) return "n_q_heads must be a multiple of n_kv_heads, at most 4096";
    return nullptr;
}

const char *bad_workspace(const void *ws, size_t have, size_t need) {
    return !ws || !aligned(ws, 1024) || have < need ? "workspace missing, misaligned or too small" : nullptr;
}

size_t evict_bytes(const KvView &v, int n_keep) {
    const long long most = std::max(0ll, std::min((long long)n_keep, v.cap - n_keep));
    return 1024 + ((size_t)v.B * v.hkv * (2 * most + 1) * sizeof(int) + 1023) / 1024 * 1024;
}

}  // namespace

extern "C" {

size_t pbd_op_decode_attention_workspace_bytes(const pbd_kv_pages *kv, int32_t n_q_heads, int32_t accumulate) {
    DecodePlan p;
    if (bad_sizes(kv) || bad_heads(kv, n_q_heads) || !decode_plan(view(*kv), n_q_heads, accumulate != 0, &p)) return 0;
    return p.total;
}

pbd_status pbd_op_decode_attention(const pbd_kv_pages *kv, int32_t n_q_heads, float scale, const void *d_q, int64_t q_stride,
                                   const void *d_k_new, const void *d_v_new, int64_t new_stride,
                                   const int32_t *d_new_positions, int32_t accumulate, void *d_out, float *d_lse_opt,
                                   void *d_ws, size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_decode_attention";
    if (const char *w = bad_cache(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (const char *w = bad_heads(kv, n_q_heads)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (!usable_factor(scale)) return fail(PBD_ERR_INVALID_ARG, who, "scale must be positive and finite");
    if (!d_q || !d_out) return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!d_k_new != !d_v_new) return fail(PBD_ERR_INVALID_ARG, who, "d_k_new and d_v_new come together");
    if (!aligned(d_q, 16) || !aligned(d_out, 16) || !aligned(d_k_new, 16) || !aligned(d_v_new, 16))
        return fail(PBD_ERR_INVALID_ARG, who, "q, out, k_new and v_new must be 16-byte aligned");
    if (!aligned(d_new_positions, 4) || !aligned(d_lse_opt, 4)) return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    const int D = kv->head_dim;
    if (q_stride < (int64_t)n_q_heads * D || q_stride % 8 || (d_k_new && (new_stride < (int64_t)kv->n_kv_heads * D || new_stride % 8)))
        return fail(PBD_ERR_INVALID_ARG, who, "row strides must be multiples of 8 values and hold a row");
    if (!addressable(kv->batch, q_stride) || (d_k_new && !addressable(kv->batch, new_stride)))
        return fail(PBD_ERR_INVALID_ARG, who, "row strides reach further than 2^60 values");
    if (const char *w = d_k_new ? bad_rows(kv) : nullptr) return fail(PBD_ERR_INVALID_ARG, who, w);
    const long long B = kv->batch, out_bytes = 2 * B * n_q_heads * D, new_bytes = 2 * ((B - 1) * new_stride + (long long)kv->n_kv_heads * D);
    if (overlap(d_out, out_bytes, d_q, 2 * ((B - 1) * q_stride + (long long)n_q_heads * D)) ||
        overlap(d_out, out_bytes, kv->d_k, cache_span(kv)) || overlap(d_out, out_bytes, kv->d_v, cache_span(kv)) ||
        (d_k_new && (overlap(d_out, out_bytes, d_k_new, new_bytes) || overlap(d_out, out_bytes, d_v_new, new_bytes))))
        return fail(PBD_ERR_INVALID_ARG, who, "out lies over something that is read");
    if (accumulate && !kv->d_weights) return fail(PBD_ERR_INVALID_ARG, who, "accumulate needs the cache's d_weights");
    DecodePlan p;
    const KvView v = view(*kv);
    if (!decode_plan(v, n_q_heads, accumulate != 0, &p))
        return fail(PBD_ERR_CAPACITY, who, "more than 2^31 tiles of 16 slots in all heads and sequences");
    if (const char *w = bad_workspace(d_ws, ws_bytes, p.total)) return fail(PBD_ERR_WORKSPACE, who, w);
    if (const char *w = d_k_new ? k_over_v(kv) : nullptr) return fail(PBD_ERR_INVALID_ARG, who, w);
    Ranges mem;
    mem.cache(kv, d_k_new != nullptr);
    mem.add("q", d_q, 2 * ((B - 1) * q_stride + (long long)n_q_heads * D), false);
    mem.add("k_new", d_k_new, new_bytes, false);
    mem.add("v_new", d_v_new, new_bytes, false);
    mem.add("out", d_out, out_bytes, true);
    mem.add("lse", d_lse_opt, 4 * B * n_q_heads, true);
    mem.add("the workspace", d_ws, (long long)p.total, true);
    const long long slots = 4 * B * v.hkv * v.cap;
    if (accumulate) mem.add("the weights", kv->d_weights, slots, true);
    if (d_k_new && d_new_positions) {
        mem.add("new_positions", d_new_positions, 4 * B, false);
        mem.add("the positions", kv->d_positions, slots, true);
    }
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    uint8_t *ws = static_cast<uint8_t *>(d_ws);
    DecodeArgs a{};
    a.kv = v;
    a.hq = n_q_heads;
    a.group = n_q_heads / kv->n_kv_heads;
    a.scale = scale;
    a.q = static_cast<const uint16_t *>(d_q);
    a.q_stride = q_stride;
    a.k_new = static_cast<const uint16_t *>(d_k_new);
    a.v_new = static_cast<const uint16_t *>(d_v_new);
    a.new_stride = new_stride;
    a.new_pos = d_new_positions;
    a.out = static_cast<uint16_t *>(d_out);
    a.lse = d_lse_opt;
    a.accumulate = accumulate != 0;
    a.fp16 = kv->dtype == PBD_FP16;
    a.status = reinterpret_cast<int *>(ws);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml);
    a.worker_bad = reinterpret_cast<int *>(ws + p.worker_bad);
    a.row_ml = reinterpret_cast<float2 *>(ws + p.row_ml);
    a.scores = accumulate ? reinterpret_cast<float *>(ws + p.scores) : nullptr;
    a.score_pitch = p.score_pitch;
    const cudaError_t e = launch_decode_attention(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

size_t pbd_op_evict_workspace_bytes(const pbd_kv_pages *kv, int32_t n_keep) {
    return bad_sizes(kv) || n_keep < 0 ? 0 : evict_bytes(view(*kv), n_keep);
}

pbd_status pbd_op_evict(const pbd_kv_pages *kv, int32_t n_keep, int32_t n_recent, int32_t n_sink,
                        const int32_t *d_next_positions, float *d_out_weights, int32_t *d_out_positions, void *d_ws,
                        size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_evict";
    if (const char *w = bad_cache(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (const char *w = bad_rows(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    if (!kv->d_weights || !kv->d_positions || !d_next_positions || !d_out_weights || !d_out_positions)
        return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (n_keep < 0 || n_recent < 0 || n_sink < 0 || (int64_t)n_recent + n_sink > n_keep)
        return fail(PBD_ERR_INVALID_ARG, who, "n_keep, n_recent and n_sink must not be negative, and the last two fit the first");
    if (!aligned(d_next_positions, 4) || !aligned(d_out_weights, 4) || !aligned(d_out_positions, 4))
        return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    const KvView v = view(*kv);
    const long long bytes = (long long)v.B * v.hkv * v.cap * 4;
    const bool in_place = d_out_weights == kv->d_weights && d_out_positions == kv->d_positions;
    if (!in_place && (overlap(d_out_weights, bytes, kv->d_weights, bytes) || overlap(d_out_positions, bytes, kv->d_positions, bytes) ||
                      overlap(d_out_weights, bytes, kv->d_positions, bytes) || overlap(d_out_positions, bytes, kv->d_weights, bytes) ||
                      overlap(d_out_weights, bytes, d_out_positions, bytes)))
        return fail(PBD_ERR_INVALID_ARG, who, "the outputs are the cache's own arrays, both of them, or lie apart from them and from one another");
    if (const char *w = bad_workspace(d_ws, ws_bytes, evict_bytes(v, n_keep))) return fail(PBD_ERR_WORKSPACE, who, w);
    if (const char *w = k_over_v(kv)) return fail(PBD_ERR_INVALID_ARG, who, w);
    Ranges mem;
    mem.cache(kv, true);
    mem.add("the weights", kv->d_weights, bytes, in_place);
    mem.add("the positions", kv->d_positions, bytes, in_place);
    mem.add("the next positions", d_next_positions, 4ll * v.B, false);
    if (!in_place) {
        mem.add("the weights' output", d_out_weights, bytes, true);
        mem.add("the positions' output", d_out_positions, bytes, true);
    }
    mem.add("the workspace", d_ws, (long long)evict_bytes(v, n_keep), true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    uint8_t *ws = static_cast<uint8_t *>(d_ws);
    EvictArgs a{};
    a.kv = v;
    a.n_keep = n_keep;
    a.n_recent = n_recent;
    a.n_sink = n_sink;
    a.next_pos = d_next_positions;
    a.out_weights = d_out_weights;
    a.out_positions = d_out_positions;
    a.status = reinterpret_cast<int *>(ws);
    a.most = std::max(0ll, std::min((long long)n_keep, v.cap - n_keep));
    a.counts = reinterpret_cast<int *>(ws + 1024);
    a.moves = a.counts + (long long)v.B * v.hkv;
    const cudaError_t e = launch_evict(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

size_t pbd_op_token_logprobs_workspace_bytes(int32_t M, int32_t V, int32_t k) {
    if (M < 1 || M > (1 << 30) || V < 1 || V > (1 << 30) || k < 0 || k > LP_MAX_K || k > V) return 0;
    return 1024;  // the status word
}

pbd_status pbd_op_token_logprobs(int32_t M, int32_t V, int32_t dtype, const void *d_logits, int64_t ld, float temperature,
                                 const int32_t *d_tokens_opt, int32_t k, float *d_logprob_opt, float *d_entropy_opt,
                                 int32_t *d_top_ids, float *d_top_logprobs, void *d_ws, size_t ws_bytes, void *d_stream) {
    const char *who = "pbd_op_token_logprobs";
    const size_t need = pbd_op_token_logprobs_workspace_bytes(M, V, k);
    if (need == 0) return fail(PBD_ERR_INVALID_ARG, who, "unsupported sizes");
    if (dtype != PBD_FP32 && dtype != PBD_BF16 && dtype != PBD_FP16) return fail(PBD_ERR_INVALID_ARG, who, "unknown type of logits");
    const int es = dtype == PBD_FP32 ? 4 : 2;
    if (ld < V) return fail(PBD_ERR_INVALID_ARG, who, "rows lie less than V values apart");
    if (!addressable(M, ld)) return fail(PBD_ERR_INVALID_ARG, who, "rows reach further than 2^60 values");
    if (!(temperature > 0.f) || std::isinf(temperature) || !usable_factor(1.f / temperature))
        return fail(PBD_ERR_INVALID_ARG, who, "temperature and its inverse must be positive and finite");
    if (!d_logits || !aligned(d_logits, es)) return fail(PBD_ERR_INVALID_ARG, who, "logits missing or misaligned");
    if (!d_tokens_opt != !d_logprob_opt) return fail(PBD_ERR_INVALID_ARG, who, "d_tokens_opt and d_logprob_opt come together");
    if (k > 0 && (!d_top_ids || !d_top_logprobs)) return fail(PBD_ERR_INVALID_ARG, who, "null pointer");
    if (!aligned(d_tokens_opt, 4) || !aligned(d_logprob_opt, 4) || !aligned(d_entropy_opt, 4) ||
        (k > 0 && (!aligned(d_top_ids, 4) || !aligned(d_top_logprobs, 4))))
        return fail(PBD_ERR_INVALID_ARG, who, "32-bit arrays must be 4-byte aligned");
    if (const char *w = bad_workspace(d_ws, ws_bytes, need)) return fail(PBD_ERR_WORKSPACE, who, w);
    Ranges mem;
    mem.add("the logits", d_logits, es * ((M - 1) * ld + V), false);
    mem.add("the tokens", d_tokens_opt, 4ll * M, false);
    mem.add("the log probabilities", d_logprob_opt, 4ll * M, true);
    mem.add("the entropy", d_entropy_opt, 4ll * M, true);
    if (k > 0) {
        mem.add("the top ids", d_top_ids, 4ll * M * k, true);
        mem.add("their log probabilities", d_top_logprobs, 4ll * M * k, true);
    }
    mem.add("the workspace", d_ws, (long long)need, true);
    if (const char *w = mem.clash()) return fail(PBD_ERR_INVALID_ARG, who, w);
    LogprobArgs a{};
    a.x = d_logits;
    a.ld = ld;
    a.M = M;
    a.V = V;
    a.type = dtype;
    a.inv_t = 1.f / temperature;
    a.tokens = d_tokens_opt;
    a.k = k;
    a.logprob = d_logprob_opt;
    a.entropy = d_entropy_opt;
    a.top_ids = d_top_ids;
    a.top_lp = d_top_logprobs;
    a.status = static_cast<int *>(d_ws);
    const cudaError_t e = launch_logprobs(a, static_cast<cudaStream_t>(d_stream));
    return e == cudaSuccess ? PBD_OK : fail(PBD_ERR_CUDA, who, "launch", e);
}

}  // extern "C"
