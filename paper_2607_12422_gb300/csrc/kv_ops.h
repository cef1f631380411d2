// kv_ops.h -- the operators on a caller's paged cache and on logits: what their kernels (kv_attn.cu, kv_evict.cu,
// logprobs.cu) take from their entry points (kv_api.cu).
#pragma once

#include "common.cuh"
#include "pbd_internal.h"

namespace pbd {

// A caller's cache as kernels see it (pbd_kv_pages).  Strides in elements of 16 bits.
struct KvView {
    const uint16_t *k, *v;
    long long stride_page, stride_head, stride_slot;
    const int *table, *lens;
    float *weights;
    int *positions;
    long long cap;  // slots of a sequence: max_pages * page_size
    int n_pages, page_size, hkv, d, B, max_pages;
    uint32_t page_mul, page_shift;  // slot / page_size = slot * page_mul >> page_shift for slots below 2^30
};

#ifdef __CUDACC__
__device__ __forceinline__ int page_index(const KvView &kv, int slot) {
    return (int)((unsigned long long)(uint32_t)slot * kv.page_mul >> kv.page_shift);
}

// Whether a page of the first slots(b) slots of some sequence b lies outside the cache; over a whole CTA, for the call's status.
// `used`: room for a number a sequence in shared memory.  Entries behind a sequence's last page are not looked at, and cost
// nothing: tables have room for a program's longest sequence.  (One loop over [batch][max_pages] instead, eviction of 64 sequences
// of 300 slots in tables of 8192 pages: 229 us instead of 26; 1024 of them 3517 instead of 146.)
template <int THREADS, typename Slots>
__device__ __forceinline__ bool any_bad_page(const KvView &kv, int *used, Slots &&slots) {
    for (int b = threadIdx.x; b < kv.B; b += THREADS) {
        const int n = slots(b);
        used[b] = n > 0 ? page_index(kv, n - 1) + 1 : 0;
    }
    __syncthreads();
    // A warp a sequence for its first LONG entries, the whole CTA for the rest of long ones.  (The whole CTA for each sequence in
    // turn: eviction of 1024 sequences of 300 slots 276 us instead of 60.)
    constexpr int LONG = 4096;
    const int lane = threadIdx.x & 31;
    bool bad = false;
    for (int b = threadIdx.x >> 5; b < kv.B; b += THREADS / 32) {
        const int *table = kv.table + (long long)b * kv.max_pages;
        const int n = min(used[b], LONG);
#pragma unroll 8
        for (int i = lane; i < n; i += 32) bad |= (unsigned)table[i] >= (unsigned)kv.n_pages;
    }
    for (int b0 = 0; b0 < kv.B; b0 += 32)
        for (unsigned m = __ballot_sync(0xffffffffu, b0 + lane < kv.B && used[b0 + lane] > LONG); m; m &= m - 1) {
            const int b = b0 + __ffs(m) - 1;
            const int *table = kv.table + (long long)b * kv.max_pages;
#pragma unroll 8
            for (int i = LONG + threadIdx.x; i < used[b]; i += THREADS) bad |= (unsigned)table[i] >= (unsigned)kv.n_pages;
        }
    return __syncthreads_or(bad);
}
#endif

constexpr int KV_MAX_WORKERS = 2048;  // warps that share a call's units
constexpr int KV_MAX_BATCH = 1024;  // sequences of a call: their lengths and first tiles lie in shared memory

// ---- attention of one token (kv_attn.cu)
struct DecodeArgs {
    KvView kv;
    int hq, group;      // query heads; of one KV head
    float scale;        // of the scores
    const uint16_t *q;  // [B] rows q_stride apart of [hq][d]
    long long q_stride;
    const uint16_t *k_new, *v_new;  // [B] rows new_stride apart of [hkv][d], or null
    long long new_stride;
    const int *new_pos;
    uint16_t *out;  // [B][hq][d]
    float *lse;     // [B][hq] or null
    int accumulate;
    int fp16;
    int *status;
    // scratch (decode_plan)
    float *part_o;    // [workers][2][heads of a chunk][d]
    float2 *part_ml;  // [workers][2][heads of a chunk]: maximum, sum
    int *worker_bad;  // [workers]: a page was outside the cache
    float2 *row_ml;   // [B][hq]: maximum, 1 / sum
    float *scores;    // [B][hq][score_pitch] when accumulating
    long long score_pitch;
    int workers;
};
struct DecodePlan {
    size_t part_o, part_ml, worker_bad, row_ml, scores, total;  // offsets in the workspace
    long long score_pitch;
};
bool decode_plan(const KvView &kv, int hq, bool accumulate, DecodePlan *p);
cudaError_t launch_decode_attention(DecodeArgs &a, cudaStream_t st);

// ---- eviction (kv_evict.cu)
struct EvictArgs {
    KvView kv;
    int n_keep, n_recent, n_sink;
    const int *next_pos;
    float *out_weights;
    int *out_positions;
    int *moves;           // [B * hkv][2][most]: holes in front, kept slots behind
    int *counts;          // [B * hkv]: moves
    long long most;
    int *status;
};
cudaError_t launch_evict(const EvictArgs &a, cudaStream_t st);

// ---- log probabilities (logprobs.cu)
struct LogprobArgs {
    const void *x;  // [M] rows ld apart of [V]
    long long ld;
    int M, V, type;  // type: pbd_dtype
    float inv_t;     // 1 / temperature
    const int *tokens;
    int k;
    float *logprob, *entropy, *top_lp;
    int *top_ids;
    int *status;
    int slices, slice_vecs;  // (launch_logprobs)
};
constexpr int LP_MAX_K = 32;
cudaError_t launch_logprobs(LogprobArgs &a, cudaStream_t st);

}  // namespace pbd
