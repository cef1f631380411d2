// page_ops.cu -- pages and slot maps from request lengths (pbd_op_assign_pages) and the move of an accepted path's rows
// (pbd_op_commit_path).
#include <algorithm>

#include "packed_ops.h"

namespace pbd {

namespace {

// ------------------------------------------------------------------ pages from lengths
//
// need_b = ceil((len_b + new_b) / page_size).  Sequences with more pages than that give the rest back, those with fewer
// take what they lack.  With exclusive prefix sums G_b of what is given, T_b of what is taken and N_b of the new tokens:
//     the stack's place n_free + G_b + i holds the i-th page that b gives,
//     the i-th page that b takes is at place n_free + G - 1 - (T_b + i),          G, T: the totals,
//     token N_b + i of the packed rows is at slot len_b + i of b.
// Sequences either give or take, places at or above n_free are only written and those below only read, so nothing has to be
// kept aside and the result does not depend on any order of threads.
//
// One cluster: each of its CTAs makes the sums for itself, a thread a sequence (a chain of latencies: lengths, scans, pages), and they share
// the pages out.  All that will be used is checked before anything is written.  A few packed rows are expanded to slots by
// the same kernel; more by a second one.
constexpr int AP_THREADS = 1024;
static_assert(KV_MAX_BATCH <= AP_THREADS, "a thread a sequence");
// (Two calls of 64 sequences, us, by the packed rows of each: one CTA 13.0 / 14.2 / 17.3 / 23.2 with 500 / 2000 / 4000 / 8000 rows, a cluster 15.2 /
// 15.4 / 15.3 / 15.4: they meet near 2500.  A cluster alone 15.4 / 17.4 / 20.7 / 26.5 / 59 with 8000 / 16000 / 32000 / 64000 / 220000, with the second
// kernel 15.4 / 15.9 / 16.3 / 15.9 / 19.4: they meet near 8000.)
constexpr int AP_CLUSTER = 8;   // CTAs where pages or rows are many
constexpr int AP_FEW = 4096;    // pages and packed rows that one CTA deals with
constexpr int AP_ROWS = 32768;  // packed rows that a cluster expands itself

struct AssignSums {
    int fresh[KV_MAX_BATCH + 1], give[KV_MAX_BATCH + 1], take[KV_MAX_BATCH + 1];  // exclusive, totals behind
    int len[KV_MAX_BATCH], held[KV_MAX_BATCH], need[KV_MAX_BATCH];
    long long warp[4][32];
    int bad[AP_CLUSTER];  // what each CTA of the cluster found
};

// the sequence that place i of a prefix sum belongs to
__device__ __forceinline__ int owner(const int *sum, int n, int i) {
    int lo = 0, hi = n;  // sum[lo] <= i < sum[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= i)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Packed row t; total: rows of all sequences.
__device__ __forceinline__ bool expand(const AssignArgs &a, const int *starts, const int *lens, int total, int t) {
    long long slot = -1;
    int pos = 0;
    bool bad = false;
    if (t < total) {
        const int b = owner(starts, a.B, t);
        pos = lens[b] + (t - starts[b]);
        const int i = pos / a.page_size;
        const int page = a.table[(long long)b * a.max_pages + i];
        bad = (unsigned)page >= (unsigned)a.n_pages;
        if (!bad) slot = (long long)page * a.page_size + (pos - i * a.page_size);
    }
    a.slots[t] = slot;
    if (a.positions) a.positions[t] = pos;
    return bad;
}

__global__ void __launch_bounds__(AP_THREADS) k_assign_pages(const __grid_constant__ AssignArgs a) {
    __shared__ AssignSums S;
    const int b = threadIdx.x, lane = b & 31, warp = b >> 5;
    const int rank = blockIdx.x, ctas = gridDim.x, me = rank * AP_THREADS + b, all = ctas * AP_THREADS;  // (one cluster)
    pdl_launch();
    cluster_arrive();
    const int n_free = *a.n_free;
    int len = 0, fresh = 0, held = 0;
    if (b < a.B) len = a.lens[b], fresh = a.n_new[b], held = a.held[b];
    const bool bad_len = len < 0 || fresh < 0 || (long long)len + fresh > a.cap;
    bool bad_page = held < 0 || held > a.max_pages || n_free < 0 || n_free > a.n_pages;
    if (bad_len) fresh = 0;
    if (bad_page) held = 0;
    const int need = bad_len ? 0 : (int)(((long long)len + fresh + a.page_size - 1) / a.page_size);
    // inclusive sums over the warp, then over the warps (64 bits: nothing is known to be sound yet)
    const long long own[4] = {fresh, max(held - need, 0), max(need - held, 0), held};
    long long sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sum[j] = own[j];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, sum[j], o);
            if (lane >= o) sum[j] += y;
        }
        if (lane == 31) S.warp[j][warp] = sum[j];
    }
    __syncthreads();
    long long total[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        long long w = S.warp[j][lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        total[j] = __shfl_sync(0xffffffffu, w, 31);
        const long long before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
        sum[j] += (warp ? before : 0) - own[j];
    }
    // (sums beyond 32 bits come with one of the totals below out of range, and are not used then)
    if (b < a.B) {
        S.fresh[b] = (int)sum[0], S.give[b] = (int)sum[1], S.take[b] = (int)sum[2];
        S.len[b] = len, S.held[b] = held, S.need[b] = need;
    }
    if (b == 0) S.fresh[a.B] = (int)total[0], S.give[a.B] = (int)total[1], S.take[a.B] = (int)total[2];
    int code = __syncthreads_or(bad_len) || total[0] > a.max_new ? DEV_BAD_POSITION : DEV_OK;
    // (a page that is held and free at once would be given to two sequences)
    if (__syncthreads_or(bad_page) || total[3] + n_free > a.n_pages) code = code ? code : DEV_BAD_PAGE;
    if (code == DEV_OK && total[2] > n_free + total[1]) code = DEV_NO_PAGES;
    const int give = (int)total[1], take = (int)total[2], top = n_free + give;
    auto given = [&](int i) {
        const int s = owner(S.give, a.B, i);
        return a.table[(long long)s * a.max_pages + S.need[s] + (i - S.give[s])];
    };
    auto taken = [&](int i) {
        const int at = top - 1 - i;
        return at < n_free ? a.free_list[at] : given(at - n_free);
    };
    auto valid = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
    // Every page that moves, first those that are taken, then those that stay on the stack: where from, where to.
    const int moves = max(take, give);
    auto source = [&](int i) { return i < take ? taken(i) : given(i - take); };
    auto put = [&](int i, int page) {
        if (i < take) {
            const int s = owner(S.take, a.B, i);
            a.table[(long long)s * a.max_pages + S.held[s] + (i - S.take[s])] = page;
        } else {
            a.free_list[n_free + i - take] = page;
        }
    };
    constexpr int KEPT = 4;  // a thread's first moves stay in registers between the check and the writing
    int page[KEPT];
    bad_page = false;
    if (code == DEV_OK) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            page[k] = me + k * all < moves ? source(me + k * all) : 0;
            bad_page |= !valid(page[k]);
        }
        for (int i = me + KEPT * all; i < moves; i += all) bad_page |= !valid(source(i));
    }
    // (code so far is the same in all CTAs; what all of them found also says that all have read what is written below)
    const int bad_here = __syncthreads_or(bad_page);
    cluster_wait();
    if (b < ctas) st_cluster_u32(map_cta(smem_u32(&S.bad[rank]), b), bad_here);
    cluster_sync();
    for (int i = 0; i < ctas; ++i)
        if (S.bad[i]) code = DEV_BAD_PAGE;
    if (code == DEV_OK) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k)
            if (me + k * all < moves) put(me + k * all, page[k]);
        for (int i = me + KEPT * all; i < moves; i += all) put(i, source(i));
        if (rank == 0 && b < a.B) a.held[b] = need;
        if (me == 0) *a.n_free = top - take;
    }
    if (rank == 0 && b < a.B) a.starts[b] = code == DEV_OK ? S.fresh[b] : 0;
    if (me == 0) a.starts[a.B] = code == DEV_OK ? S.fresh[a.B] : 0, *a.status = code;
    if (a.max_new > AP_ROWS) return;
    cluster_sync();  // (the table's new entries)
    const int rows = code == DEV_OK ? S.fresh[a.B] : 0;
    bool bad = false;
    for (int t = me; t < a.max_new; t += all) bad |= expand(a, S.fresh, S.len, rows, t);
    if (bad) latch_error(a.status, DEV_BAD_PAGE);
}

constexpr int AP_EXPAND = 256;
__global__ void __launch_bounds__(AP_EXPAND) k_expand_slots(const __grid_constant__ AssignArgs a) {
    __shared__ int starts[KV_MAX_BATCH + 1], lens[KV_MAX_BATCH];
    for (int b = threadIdx.x; b < a.B; b += AP_EXPAND) lens[b] = a.lens[b];
    pdl_wait();
    for (int b = threadIdx.x; b <= a.B; b += AP_EXPAND) starts[b] = a.starts[b];
    __syncthreads();
    const int total = starts[a.B];
    bool bad = false;
    for (long long t = blockIdx.x * AP_EXPAND + threadIdx.x; t < a.max_new; t += (long long)gridDim.x * AP_EXPAND)
        bad |= expand(a, starts, lens, total, (int)t);
    if (bad) latch_error(a.status, DEV_BAD_PAGE);
}

// ------------------------------------------------------------------ accepted paths
//
// Row len + path[i] of a sequence goes to len + i, i < n_accepted.  path ascends, so path[i] >= i: a row's target may be an earlier
// row's source, and never a later one's.  So rows are taken in their order, some at a time, which are read before any of them is written.
// One small CTA takes one (sequence, KV head): each is a chain of loads (length, path, table, rows), so that many at once count.
// (512 sequences of 8 KV heads, 12 rows to move in each on average, 26 MB read and as much written: 9.2 us, 5.7 TB/s; with 256 threads 16.2, and 17.7 when
// each takes four heads.  8 sequences: 3.2 us, launches and that chain.)  k_clear_status, which overlaps it, makes room for what any CTA
// finds wrong (one CTA that looks at all paths takes 50 us for 512 of them).
constexpr int CP_THREADS = 128;

// whether a path of n nodes behind len slots can be walked
__device__ __forceinline__ bool path_ok(const CommitArgs &a, int n, int len) {
    return n >= 0 && n <= a.max_path && len >= 0 && len <= a.kv.cap;
}

__global__ void k_clear_status(int *status) {
    pdl_launch();
    *status = DEV_OK;
}
__device__ __noinline__ void report(const CommitArgs &a, int code) {
    pdl_wait();  // (the status has been cleared)
    latch_error(a.status, code);
}

template <int D>
__global__ void __launch_bounds__(CP_THREADS) k_commit_path(const __grid_constant__ CommitArgs a) {
    constexpr int CPR = D / 8, U = 4;  // 16-byte pieces of a row, of a thread at a time
    __shared__ long long of[TREE_NODES], to[TREE_NODES];  // value offsets of the rows, -1: does not move
    __shared__ int slot_of[TREE_NODES];
    const int b = blockIdx.x / a.kv.hkv, h = blockIdx.x - b * a.kv.hkv;
    const int n = a.n_accepted[b], len = a.kv.lens[b], i = threadIdx.x;
    if (!path_ok(a, n, len)) {
        if (h == 0 && i == 0) report(a, DEV_BAD_POSITION);
        return pdl_wait();
    }
    if (n == 0) return pdl_wait();
    bool bad = false, bad_page = false;
    if (i < n) {
        const int p = a.path[(long long)b * a.max_path + i], before = i ? a.path[(long long)b * a.max_path + i - 1] : -1;
        bad = p <= before || p >= TREE_NODES || (long long)len + p >= a.kv.cap;
        long long from = -1, dest = -1;
        if (!bad && p != i) {
            const int *table = a.kv.table + (long long)b * a.kv.max_pages;
            const int si = page_index(a.kv, len + p), di = page_index(a.kv, len + i);
            const int sp = table[si], dp = table[di];
            bad_page = (unsigned)sp >= (unsigned)a.kv.n_pages || (unsigned)dp >= (unsigned)a.kv.n_pages;
            if (!bad_page) {
                from = sp * a.kv.stride_page + h * a.kv.stride_head + (len + p - si * a.kv.page_size) * a.kv.stride_slot;
                dest = dp * a.kv.stride_page + h * a.kv.stride_head + (len + i - di * a.kv.page_size) * a.kv.stride_slot;
            }
        }
        of[i] = from, to[i] = dest, slot_of[i] = len + p;
    }
    if (__syncthreads_or(bad)) {  // the sequence stays as it is, whatever its pages are
        if (h == 0 && bad) report(a, DEV_BAD_TREE);
        return pdl_wait();
    }
    if (h == 0 && bad_page) report(a, DEV_BAD_PAGE);
    for (int x0 = i; x0 < n * 2 * CPR + i; x0 += U * CP_THREADS) {
        uint4 piece[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int x = x0 + j * CP_THREADS, r = x / (2 * CPR), c = x % (2 * CPR);
            if (r < n && of[r] >= 0) piece[j] = *reinterpret_cast<const uint4 *>((c < CPR ? a.kv.k : a.kv.v) + of[r] + (c % CPR) * 8);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int x = x0 + j * CP_THREADS, r = x / (2 * CPR), c = x % (2 * CPR);
            if (r < n && of[r] >= 0) *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(c < CPR ? a.kv.k : a.kv.v) + to[r] + (c % CPR) * 8) = piece[j];
        }
    }
    const long long at = ((long long)b * a.kv.hkv + h) * a.kv.cap;
    float w = 0.f;
    int pos = 0;
    const bool moves = i < n && of[i] >= 0;
    if (moves && a.kv.weights) w = a.kv.weights[at + slot_of[i]];
    if (moves && a.kv.positions) pos = a.kv.positions[at + slot_of[i]];
    __syncthreads();
    if (moves && a.kv.weights) a.kv.weights[at + len + i] = w;
    if (moves && a.kv.positions) a.kv.positions[at + len + i] = pos;
    pdl_wait();
}

}  // namespace

cudaError_t launch_assign_pages(const AssignArgs &a, cudaStream_t st) {
    // (512 sequences, 10000 pages taken, as many given back by the next call, 220000 rows: 200 us the two calls with one CTA, 36 with eight;
    // 8 sequences, few pages: 10.2 us the two with one CTA; 12.7 when that one is launched as a cluster)
    const bool many = a.max_new > AP_FEW || std::min<long long>(a.n_pages, (long long)a.B * a.max_pages) > AP_FEW;
    const cudaError_t e = launch_cluster(k_assign_pages, many ? AP_CLUSTER : 1, AP_THREADS, st, a);
    if (e != cudaSuccess) return e;
    if (a.max_new > AP_ROWS) {
        const int grid = std::min((a.max_new + AP_EXPAND - 1) / AP_EXPAND, 8 * gemm_ctas());
        const cudaError_t e = launch_pdl(k_expand_slots, grid, AP_EXPAND, 0, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaGetLastError();
}

cudaError_t launch_commit_path(const CommitArgs &a, cudaStream_t st) {
    const int grid = a.kv.B * a.kv.hkv;
    k_clear_status<<<1, 1, 0, st>>>(a.status);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    switch (a.kv.d) {
        case 64: return launch_pdl(k_commit_path<64>, grid, CP_THREADS, 0, st, a);
        case 128: return launch_pdl(k_commit_path<128>, grid, CP_THREADS, 0, st, a);
        default: return launch_pdl(k_commit_path<256>, grid, CP_THREADS, 0, st, a);
    }
}

}  // namespace pbd
