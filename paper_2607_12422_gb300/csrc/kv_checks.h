// kv_checks.h -- what the entry points of the operators on a caller's cache, on packed rows and on logits (kv_api.cu,
// packed_api.cu) check before they launch anything.
#pragma once

#include <cmath>
#include <cstdio>

#include "../../include/pbd_ops.h"
#include "kv_ops.h"

namespace pbd {
namespace checks {

inline pbd_status fail(pbd_status s, const char *who, const char *what, cudaError_t e = cudaSuccess) {
    char b[256];
    snprintf(b, sizeof b, "%s: %s%s%s", who, what, e != cudaSuccess ? ": " : "", e != cudaSuccess ? cudaGetErrorString(e) : "");
    op_record_error(b);
    return s;
}

inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The exponents' factor, which kernels hold with log2 e in it, is finite too.
inline bool usable_factor(float f) { return f > 0.f && !std::isinf(f * 1.4426950408889634f); }

inline bool overlap(const void *a, long long na, const void *b, long long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Whether `n` rows `stride` values apart can be addressed: byte offsets and spans stay below 2^63.
inline bool addressable(long long n, long long stride) { return n <= 1 || stride <= (1ll << 60) / (n - 1); }

// What is wrong with a cache's sizes and strides, or null.  Pointers are looked at by the entry points: workspace sizes
// are asked for before there are any.
inline const char *bad_sizes(const pbd_kv_pages *kv) {
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

inline const char *bad_cache(const pbd_kv_pages *kv) {
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
inline const char *bad_rows(const pbd_kv_pages *kv) {
    const int D = kv->head_dim;
    if ((kv->page_size > 1 && kv->stride_slot < D) || (kv->n_kv_heads > 1 && kv->stride_head < D) || (kv->n_pages > 1 && kv->stride_page < D))
        return "a cache that is written to has strides of a row or more";
    const Places p(kv);
    if (!p.apart()) return "the rows of a cache that is written to lie over one another";
    return nullptr;
}
inline const char *k_over_v(const pbd_kv_pages *kv) {
    const Places p(kv);
    const long long off = (long long)(reinterpret_cast<uintptr_t>(kv->d_v) - reinterpret_cast<uintptr_t>(kv->d_k)) / 2;
    return p.meet(off, p.n) ? "K and V of a cache that is written to lie over one another" : nullptr;
}

// bytes from the first value of K (or V) to the last
inline long long cache_span(const pbd_kv_pages *kv) {
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
    bool has_cache = false, full = false;  // (its K and V come first); whether there was one more than there is room for
    char text[96];

public:
    void add(const char *name, const void *p, long long bytes, bool written) {
        if (!p) return;
        if (n == 16)
            full = true;
        else
            r[n++] = Range{p, bytes, name, written};
    }
    void cache(const pbd_kv_pages *kv, bool written) {
        has_cache = true;
        add("K", kv->d_k, cache_span(kv), written);
        add("V", kv->d_v, cache_span(kv), written);
        add("the page table", kv->d_page_table, 4ll * kv->batch * kv->max_pages, false);
        add("the lengths", kv->d_lens, 4ll * kv->batch, false);
    }
    const char *clash() {
        if (full) return "the call has more arrays than are compared";
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

inline KvView view(const pbd_kv_pages &kv) {
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

inline const char *bad_heads(const pbd_kv_pages *kv, int hq) {
    if (hq < kv->n_kv_heads || hq % kv->n_kv_heads || hq > 4096) return "n_q_heads must be a multiple of n_kv_heads, at most 4096";
    return nullptr;
}

inline const char *bad_workspace(const void *ws, size_t have, size_t need) {
    return !ws || !aligned(ws, 1024) || have < need ? "workspace missing, misaligned or too small" : nullptr;
}

}  // namespace checks
}  // namespace pbd
