// packed_ops.h -- operators on packed rows of several sequences and the pages behind them: what their kernels (page_ops.cu,
// prompt_attn.cu, tree_attn.cu) take from their entry points (packed_api.cu).
#pragma once

#include "kv_ops.h"

namespace pbd {

constexpr int TREE_NODES = 64;  // drafted tokens of a sequence at most: a node's ancestors are the bits of one word

// ---- pages from lengths (page_ops.cu)
struct AssignArgs {
    const int *lens, *n_new;  // [B]
    int *table;               // [B][max_pages]
    int *held, *free_list, *n_free;
    int B, max_pages, page_size, n_pages, max_new;
    long long cap;      // slots of a sequence
    int *starts;        // [B + 1]
    long long *slots;   // [max_new]
    int *positions;     // [max_new] or null
    int *status;
};
cudaError_t launch_assign_pages(const AssignArgs &a, cudaStream_t st);

// ---- accepted paths (page_ops.cu)
struct CommitArgs {
    KvView kv;
    const int *path;  // [B][max_path]
    const int *n_accepted;
    int max_path;
    int *status;
};
cudaError_t launch_commit_path(const CommitArgs &a, cudaStream_t st);

// ---- attention of packed rows (prompt_attn.cu, tree_attn.cu)
struct PackedArgs {
    KvView kv;       // tree: the cache; prompt: where K and V are stored (k null: nowhere)
    int T, B, hq, hkv, group, d, fp16;
    float scale;
    const uint16_t *q, *k, *v;  // rows q_stride and kv_stride apart of [heads][d]
    long long q_stride, kv_stride;
    const int *starts;       // [B + 1]
    const long long *slots;  // prompt: [T] or null
    const int *parents;      // tree: [T] or null (a chain)
    const int *new_pos;      // tree: [T] or null
    uint16_t *out;           // [T][hq][d]
    float *lse;              // [T][hq] or null
    int *status;
    uint32_t patience;       // after which a wait in the kernel gives up, in 2^20 ns
    // scratch (tree alone; tree_plan)
    int workers, part_rows;  // CTAs; rows of one's part of a unit
    int *worker_code;        // [workers]
    float2 *part_ml;         // [workers][2][part_rows]: maximum, sum
    float *part_o;           // [workers][2][part_rows][d]
};
cudaError_t launch_prompt_attention(PackedArgs &a, cudaStream_t st);

// Some waits in these kernels last as long as the work between two things that a warp has to do: rows of an item's second tile, when it has
// none, wait for the whole item; the second tile's MMAs of a CTA's stretch for all units of one tile in front.  So a wait gives up after a second
// and 32 us for each block of that work (a block takes 1 to 2 us, copied row by row 5 to 10).
inline uint32_t packed_patience(double blocks) { return (uint32_t)((1e9 + 32e3 * blocks) / (1 << 20)) + 1; }
inline uint32_t prompt_patience(int T) { return packed_patience(T / 128 + 1); }  // the longest item's blocks
inline uint32_t tree_patience(double places, int workers) { return packed_patience(places / workers + 1); }  // of the longest list

#ifdef __CUDACC__
// Whether a sequence's bounds lie inside the packed rows.  Where all do, no row is two sequences'; where some do not, a sequence takes part
// only if it also begins at or behind all bounds in front of its own (behind_all): what follows a descent would lie over rows before it.
__device__ __forceinline__ bool bounds_ok(const PackedArgs &a, int s, int e) { return s >= 0 && e >= s && e <= a.T; }
__device__ __forceinline__ bool behind_all(const int *starts, int b) {
    const int s = starts[b];
#pragma unroll 1
    for (int i = 0; i < b; ++i)
        if (starts[i] > s) return false;
    return true;
}
#endif

constexpr int TREE_MAX_WORKERS = 160;
struct TreePlan {
    size_t codes, part_ml, part_o, total;  // offsets in the workspace
    int rows;
};
double tree_places(const KvView &kv, int T, int hq);  // of the list at most
bool tree_plan(const KvView &kv, int T, int hq, TreePlan *p);
cudaError_t launch_tree_attention(PackedArgs &a, cudaStream_t st);

}  // namespace pbd
