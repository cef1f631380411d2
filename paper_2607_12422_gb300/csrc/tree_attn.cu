// tree_attn.cu -- attention of drafted trees over a caller's paged cache (pbd_op_tree_attention).
//
// For node i of a sequence, query head h of KV head h / group and the keys j that the node sees, the cached slots, its ancestors and
// itself:
//     s_ij = q_i . k_j,  p_ij = exp(scale (s_ij - max_j s_ij)),  l_i = sum_j p_ij,  out_i = sum_j p_ij v_j / l_i
// in one pass over the keys (flash.cuh).  All nodes and heads that share a KV head are the rows of one tile, or two: the cache is read
// once for 256 rows, and memory bounds it until rows are that many.
//
// The blocks of 128 keys of all (sequence, KV head, 256 rows) form one list, and each CTA takes one contiguous stretch of it, all
// of about the same cost: how ragged the lengths are does not matter, and the host need not know them.  Where a stretch begins or ends
// inside a (sequence, KV head) the CTA leaves maximum, sum and unnormalised output in scratch, and k_tree_join joins them.
//
// Warps 0-7: rows, a thread each (queries, softmax, outputs).  Warps 8-11 copy K and V, row by row, since pages may have any length:
// 16 bytes a lane, asynchronously.  Warp 12: MMAs.  The blocks with nodes among their keys, a (sequence, KV head)'s last one or
// two, are waited for by the warps that copy them: they store the nodes' rows into the cache, and look for infinite and NaN values
// of V, which would be NaN in rows that do not see them (0 x NaN): such values become zero, and who sees them is noted for each
// dimension.
#include <algorithm>

#include "flash.cuh"
#include "packed_ops.h"

namespace pbd {

using namespace flash;

namespace {

constexpr int TA_THREADS = 512;
constexpr int TA_ROW = 2;        // what beginning and ending a (sequence, KV head) costs a CTA, in blocks
constexpr int TA_MIN = 3;        // places of a CTA's stretch at least
constexpr int TA_MASKS = 8;      // blocks whose masks are kept

template <int D>
struct TreeShape : Shape<D> {
    using S = Shape<D>;
    static constexpr int STAGES = D == 64 ? 8 : 4;
    static constexpr int RING_SEGS = D == 64 ? 8 : 4;  // segments that copies can be ahead, and one more
    static constexpr int ROWS_ALL = S::TILES * ROWS;
    static constexpr int SMEM = S::TILES * S::QT + STAGES * S::UNIT + 1024;
};

// Counts of the list: a (sequence, KV head, chunk of rows) is a unit; it has its blocks and TA_ROW places more in front.
struct TreeList {
    int first[KV_MAX_BATCH + 1];  // places before sequence b
    int start[KV_MAX_BATCH], len[KV_MAX_BATCH], nodes[KV_MAX_BATCH];
};

__device__ __forceinline__ bool tree_ok(const PackedArgs &a, int b) {
    const int s = a.starts[b], e = a.starts[b + 1], len = a.kv.lens[b];
    return s >= 0 && e >= s && e <= a.T && e - s <= TREE_NODES && len >= 0 && len + (long long)(e - s) <= a.kv.cap;
}
__device__ __forceinline__ int blocks_of(int len, int nodes) { return (len + nodes + KEYS - 1) / KEYS; }
template <int D>
__device__ __forceinline__ int chunks_of(int rows) { return (rows + TreeShape<D>::ROWS_ALL - 1) / TreeShape<D>::ROWS_ALL; }

// Whole CTA; returns the list's length.
template <int D>
__device__ __forceinline__ int tree_list(const PackedArgs &a, TreeList &T) {
    __shared__ int warp_sum[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        int x = 0;
        if (b < a.B) {
            const bool ok = tree_ok(a, b);
            const int n = ok ? a.starts[b + 1] - a.starts[b] : 0, len = ok ? a.kv.lens[b] : 0;
            T.start[b] = a.starts[b], T.len[b] = len, T.nodes[b] = n;
            if (n > 0) x = a.hkv * chunks_of<D>(n * a.group) * (blocks_of(len, n) + TA_ROW);
        }
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        int before = carry, all = 0;
        for (int w = 0; w < n_warps; ++w) {
            if (w < warp) before += warp_sum[w];
            all += warp_sum[w];
        }
        if (b < a.B) T.first[b + 1] = before + x;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) T.first[0] = 0;
    __syncthreads();
    return carry;
}

__device__ __forceinline__ int workers_of(const PackedArgs &a, int count) { return max(1, min(a.workers, (count + TA_MIN - 1) / TA_MIN)); }
__device__ __forceinline__ int first_of(int w, int count, int workers) { return (int)((long long)w * count / workers); }
__device__ __forceinline__ int worker_at(long long at, int count, int workers) { return (int)(((at + 1) * workers - 1) / count); }

// Blocks [t, t_end) of one unit: what a CTA works on before it leaves the unit.
struct Segment {
    int b, unit, units, t, t_end, blocks;  // sequence, unit of it, its units, blocks, the unit's blocks
    int at, end;                           // list place of the unit, end of the stretch
    int chunks;
    template <int D>
    __device__ __forceinline__ void enter(const PackedArgs &a, const TreeList &T) {
        blocks = blocks_of(T.len[b], T.nodes[b]);
        chunks = chunks_of<D>(T.nodes[b] * a.group);
        units = a.hkv * chunks;
    }
    __device__ __forceinline__ bool clip() {
        t_end = min(blocks, end - at - TA_ROW);
        return t < t_end;
    }
    // The first segment of the stretch [u, u_end); false if it has none.
    template <int D>
    __device__ __forceinline__ bool seek(int u, int u_end, const PackedArgs &a, const TreeList &T) {
        end = u_end;
        if (u >= end) return false;
        int lo = 0, hi = a.B;  // first[lo] <= u < first[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (T.first[mid] <= u)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
        enter<D>(a, T);
        const int per = blocks + TA_ROW;
        unit = (u - T.first[b]) / per;
        at = T.first[b] + unit * per;
        t = max(0, u - at - TA_ROW);
        return clip() || next<D>(a, T);
    }
    template <int D>
    __device__ __forceinline__ bool next(const PackedArgs &a, const TreeList &T) {
        at += blocks + TA_ROW;
        t = 0;
        if (++unit == units) {
            unit = 0;
            do ++b;
            while (b < a.B && T.first[b + 1] == T.first[b]);
            if (b >= a.B || at >= end) return false;
            enter<D>(a, T);
        }
        return at < end && clip();  // (where only a unit's front is left the stretch is over)
    }
};

template <int D>
struct TreeState {
    using L = TreeShape<D>;
    uint64_t full[L::STAGES], empty[L::STAGES], q_full[2], s_full[2], p_full[2], o_full[2], o_free[2], tail[L::RING_SEGS], cleared, drain;
    uint32_t tmem;
    int abort, bad_page, bad_tree;
    uint32_t valid[TA_MASKS][4];        // keys of a block whose pages are in the cache
    ulonglong2 rows[4][32];             // a copying warp's rows: where K and V come from
    // of a segment: who sees infinite or NaN values, in each dimension: the nodes' bits, or everybody (a cached slot)
    int odd[L::RING_SEGS];
    unsigned long long odd_nodes[L::RING_SEGS][D];
    int odd_all[L::RING_SEGS][D];
};

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool real) {
    const int n = real ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// Arrives on `bar` once this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

template <int D, bool FP16>
__global__ void __launch_bounds__(TA_THREADS, 1) k_tree(const __grid_constant__ PackedArgs a) {
    using L = TreeShape<D>;
    constexpr int TILES = L::TILES, UNITS = L::UNITS, STAGES = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sq = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *ring = sq + TILES * L::QT;
    __shared__ TreeState<D> S;
    __shared__ TreeList T;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    pdl_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&S.full[i], 128);
            mbar_init(&S.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&S.q_full[i], 4);
            mbar_init(&S.s_full[i], 1);
            mbar_init(&S.p_full[i], 4);
            mbar_init(&S.o_full[i], 1);
            mbar_init(&S.o_free[i], 4);
        }
        for (int i = 0; i < L::RING_SEGS; ++i) mbar_init(&S.tail[i], 128);
        mbar_init(&S.cleared, 128);
        mbar_init(&S.drain, 1);
        S.abort = S.bad_page = S.bad_tree = 0;
        fence_mbarrier_init();
        if (blockIdx.x == 0) *a.status = DEV_OK;  // (k_tree_join reports; a wait runs out a second later)
    }
    const int count = tree_list<D>(a, T);
    const int workers = workers_of(a, count), me = blockIdx.x;
    Segment seg;
    const bool has = me < workers && seg.seek<D>(first_of(me, count, workers), first_of(me + 1, count, workers), a, T);
    if (!has) {
        if (threadIdx.x == 0) a.worker_code[me] = DEV_OK;
        return;
    }
    if (warp == 12) tmem_alloc(&S.tmem, TM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S.tmem;
    bool more = true;

    // registers: of the launch's 4 x 128 x 128 the rows' warpgroups take 128 x 200 each, the others keep 128 x 56
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp < 12) {
            // ---- copies: K 0, V 0, K 1, V 1, ... of each segment; warp w rows 32 w .. of each block
            const int w = warp - 8, key0 = 32 * w + lane;
            ulonglong2 *rows = S.rows[w];
            constexpr int CPR = L::DU / 8, RPI = 32 / CPR;  // 16-byte pieces of a unit's row, rows of a step
            const int piece = lane % CPR, r_lane = lane / CPR;
            // where piece `piece` of the warp's row r lies in a unit
            auto place = [&](int r) { return (uint32_t)((piece >> 3) * SUB + (32 * w + r) * 128 + (((piece & 7) ^ (r & 7)) << 4)); };
            auto entry = [&](const Segment &g, int t) {
                const int key = t * KEYS + key0;
                return key < T.len[g.b] + T.nodes[g.b] ? a.kv.table[(long long)g.b * a.kv.max_pages + page_index(a.kv, key)] : 0;
            };
            int issued = 0, block = 0, sn = 0, clears = 0;
            bool ok = true;
            int page = entry(seg, seg.t);
            for (; ok && more; ++sn) {
                const int b = seg.b, len = T.len[b], nodes = T.nodes[b], h = seg.unit / seg.chunks;
                const bool store = seg.unit % seg.chunks == 0;
                const int tail0 = len / KEYS;  // the first block with nodes or places behind them
                const int si = sn % L::RING_SEGS;
                Segment nxt = seg;
                const bool nxt_more = nxt.next<D>(a, T);
                for (int t = seg.t; ok && t < seg.t_end; ++t, ++block) {
                    const int key = t * KEYS + key0;
                    const bool cached = key < len, node = !cached && key < len + nodes;
                    const bool real = (cached || node) && (unsigned)page < (unsigned)a.kv.n_pages;
                    const int pi = page_index(a.kv, key);
                    const long long off = real ? page * a.kv.stride_page + h * a.kv.stride_head + (key - pi * a.kv.page_size) * a.kv.stride_slot : -1;
                    if ((cached || node) && !real) *(volatile int *)&S.bad_page = 1;
                    ulonglong2 at = make_ulonglong2(0, 0);
                    if (real) {
                        const long long src = cached ? off : (long long)(T.start[b] + key - len) * a.kv_stride + h * D;
                        at.x = reinterpret_cast<unsigned long long>((cached ? a.kv.k : a.k) + src);
                        at.y = reinterpret_cast<unsigned long long>((cached ? a.kv.v : a.v) + src);
                    }
                    const unsigned valid = __ballot_sync(0xffffffffu, real);
                    __syncwarp();
                    rows[lane] = at;
                    if (lane == 0) *(volatile uint32_t *)&S.valid[block % TA_MASKS][w] = valid;
                    if (node && store && a.new_pos && a.kv.positions && real)
                        a.kv.positions[((long long)b * a.hkv + h) * a.kv.cap + key] = a.new_pos[T.start[b] + key - len];
                    __syncwarp();
                    // the next block's pages are asked for now
                    const bool last = t + 1 == seg.t_end;
                    const int next_page = !last ? entry(seg, t + 1) : nxt_more ? entry(nxt, nxt.t) : 0;
                    const bool tail = t >= tail0;
                    if (tail && t == max(seg.t, tail0)) {  // nobody looks at this segment's notes yet
                        for (int d = threadIdx.x - 256; d < D; d += 128) S.odd_nodes[si][d] = 0, S.odd_all[si][d] = 0;
                        if (threadIdx.x == 256) S.odd[si] = 0;
                        mbarrier_arrive_one(&S.cleared);
                        ok = mbar_wait(&S.cleared, clears++ & 1, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                        ok = __all_sync(0xffffffffu, ok);
                    }
                    for (int kv = 0; ok && kv < 2; ++kv)
                        for (int u = 0; u < UNITS; ++u) {
                            const int slot = issued % STAGES;
                            ok = mbar_wait(&S.empty[slot], ((issued / STAGES) & 1) ^ 1, a.status, DEV_TIMEOUT_SLOT, &S.abort);
                            if (!(ok = __all_sync(0xffffffffu, ok))) break;
                            ++issued;
                            const uint32_t to = smem_u32(ring + slot * L::UNIT);
#pragma unroll 8
                            for (int x = 0; x < 32; x += RPI) {
                                const int r = x + r_lane;
                                const unsigned long long *p = &rows[r].x + kv;
                                const uint16_t *src = reinterpret_cast<const uint16_t *>(*p);
                                cp_async16_or_zero(to + place(r), src ? src + u * L::DU + piece * 8 : a.q, src != nullptr);
                            }
                            if (!tail) {
                                cp_async_arrive(&S.full[slot]);
                                continue;
                            }
                            cp_async_commit();
                            cp_async_wait_all();
#pragma unroll 4
                            for (int x = 0; x < 32; x += RPI) {  // (each lane its own pieces)
                                const int r = x + r_lane, k = t * KEYS + 32 * w + r, i = k - len;
                                if (!(valid >> r & 1)) continue;
                                const uint4 v = ld_shared_u4(to + place(r));
                                const int d0 = u * L::DU + piece * 8;
                                if (store && i >= 0) {
                                    const int pg = a.kv.table[(long long)b * a.kv.max_pages + page_index(a.kv, k)];
                                    const long long dst = pg * a.kv.stride_page + h * a.kv.stride_head +
                                                          (k - page_index(a.kv, k) * a.kv.page_size) * a.kv.stride_slot + d0;
                                    *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(kv ? a.kv.v : a.kv.k) + dst) = v;
                                }
                                uint32_t wd[4] = {v.x, v.y, v.z, v.w};
                                if (kv == 0 || !(odd_halves<FP16>(wd[0]) | odd_halves<FP16>(wd[1]) | odd_halves<FP16>(wd[2]) | odd_halves<FP16>(wd[3])))
                                    continue;
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const uint32_t half = 0xffffu << (16 * (e & 1));
                                    if (!(odd_halves<FP16>(wd[e >> 1]) & half)) continue;
                                    wd[e >> 1] &= ~half;
                                    if (i < 0)
                                        S.odd_all[si][d0 + e] = 1;
                                    else
                                        atomicOr(&S.odd_nodes[si][d0 + e], 1ull << i);
                                }
                                st_shared_u4(to + place(r), make_uint4(wd[0], wd[1], wd[2], wd[3]));
                                S.odd[si] = 1;
                            }
                            fence_proxy_async_shared();
                            mbarrier_arrive_one(&S.full[slot]);
                        }
                    page = next_page;
                }
                if (ok && seg.t_end > tail0) mbarrier_arrive_one(&S.tail[si]);  // (only a stretch's last segment has no such block)
                seg = nxt;
                more = nxt_more;
            }
            cp_async_commit();
            cp_async_wait_all();  // also on the error path: nothing is in flight when the CTA ends
        } else if (warp == 12 && elect_one()) {
            // ---- MMAs: for every block, tile after tile, O += P V of the block before, then S
            int pos = 0, used_p[2] = {0, 0}, used[2] = {0, 0};  // ring units; blocks and segments of a tile so far
            bool ok = true;
            auto landed = [&](int at) { ok = ok && mbar_wait(&S.full[at % STAGES], (at / STAGES) & 1, a.status, DEV_TIMEOUT_LOAD, &S.abort); };
            while (ok && more) {
                const int nb = seg.t_end - seg.t, all = T.len[seg.b] + T.nodes[seg.b];
                const int n_rows = T.nodes[seg.b] * a.group - (seg.unit % seg.chunks) * L::ROWS_ALL;
                const int tiles = TILES == 2 && n_rows > ROWS ? 2 : 1;
                for (int j = 0; ok && j <= nb; ++j) {
                    const int vp = pos, kp = pos + (j ? UNITS : 0);
                    if (j) pos += UNITS;
                    if (j < nb) pos += UNITS;
                    for (int i = 0; ok && i < tiles; ++i) {
                        if (j > 0) {
                            ok = mbar_wait(&S.p_full[i], used_p[i] & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
                            ++used_p[i];
                            if (j == 1 && used[i] > 0) ok = ok && mbar_wait(&S.o_free[i], (used[i] - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
                            const int steps = min(KEYS, all - (seg.t + j - 1) * KEYS + 15) / 16;
                            for (int u = 0; ok && u < UNITS; ++u) {
                                landed(vp + u);
                                if (!ok) break;
                                fence_proxy_async_shared();  // (copies by cp.async land in the generic proxy)
                                tc_fence_after();
                                mma_values<D, FP16>(tmem + TM_O + i * D, tmem + i * KEYS, ring + ((vp + u) % STAGES) * L::UNIT, u, steps, j == 1);
                            }
                            if (ok && j == nb) mma_commit(&S.o_full[i]);
                        }
                        if (ok && j > 0 && i == tiles - 1)
                            for (int u = 0; u < UNITS; ++u) mma_commit(&S.empty[(vp + u) % STAGES]);
                        if (ok && j < nb) {
                            if (j == 0) ok = mbar_wait(&S.q_full[i], used[i] & 1, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                            for (int u = 0; ok && u < UNITS; ++u) {
                                landed(kp + u);
                                if (!ok) break;
                                fence_proxy_async_shared();
                                tc_fence_after();
                                mma_scores<D, FP16>(tmem + i * KEYS, sq + i * L::QT, ring + ((kp + u) % STAGES) * L::UNIT, u);
                            }
                            if (ok) mma_commit(&S.s_full[i]);
                        }
                    }
                    if (ok && j < nb)
                        for (int u = 0; u < UNITS; ++u) mma_commit(&S.empty[(kp + u) % STAGES]);
                }
                for (int i = 0; i < tiles; ++i) ++used[i];
                more = seg.next<D>(a, T);
            }
            mma_commit(&S.drain);  // also on the error path: every MMA issued completes before TMEM is released
            mbar_wait(&S.drain, 0, nullptr, 0, nullptr);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // ---- rows: thread r of tile i the row r of the unit's 128 i ..: node row / group, head row % group
        const int i = warp >> 2, w = warp & 3;
        const uint32_t lanes = (uint32_t)(w * 32) << 16, ts = tmem + lanes + i * KEYS, to = tmem + lanes + TM_O + i * D;
        const uint32_t mine = smem_u32(sq + i * L::QT);
        const float c = a.scale * 1.4426950408889634f;
        constexpr int CPR = D / 8, RPI = 32 / CPR;
        const int piece = lane % CPR;
        // where piece `piece` of the warp's row r lies in the tile
        auto place = [&](int r, int p) { return mine + (uint32_t)((p >> 3) * SUB + (w * 32 + r) * 128 + (((p & 7) ^ (r & 7)) << 4)); };
        int used = 0, used_s = 0, block = 0, sn = 0;  // segments and blocks of the tile; blocks and segments of the CTA
        bool ok = true;
        for (; ok && more; ++sn, more = seg.next<D>(a, T)) {
            const int b = seg.b, nb = seg.t_end - seg.t, len = T.len[b], nodes = T.nodes[b], h = seg.unit / seg.chunks;
            const int row = (seg.unit % seg.chunks) * L::ROWS_ALL + i * ROWS + w * 32 + lane, n_rows = nodes * a.group;
            const bool whole = nb == seg.blocks, ends = seg.t_end > len / KEYS;  // (with nodes, or places behind them, among its keys)
            const int part = seg.t == 0;  // of units a stretch has at most two parts: an end and a beginning
            if (i >= TILES || i * ROWS + (seg.unit % seg.chunks) * L::ROWS_ALL >= n_rows) {  // (uniform over the tile)
                block += nb;
                continue;
            }
            const bool real = row < n_rows;
            const int node = real ? row / a.group : 0, head = h * a.group + (real ? row - node * a.group : 0);
            const long long q_off = real ? (long long)(T.start[b] + node) * a.q_stride + head * D : -1;
            // the queries (the tile's last MMAs are done, and its outputs have left)
#pragma unroll 4
            for (int x = 0; x < 32; x += RPI) {
                const int r = x + lane / CPR;
                const long long o = __shfl_sync(0xffffffffu, q_off, r);
                cp_async16_or_zero(place(r, piece), o >= 0 ? a.q + o + piece * 8 : a.q, o >= 0);
            }
            cp_async_commit();
            // ancestors: lane x holds nodes x and x + 32
            uint64_t anc = 0;
            if (ends) {
                int p[2];
                uint64_t m[2];
                bool bad = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int x = lane + 32 * e;
                    p[e] = -1;
                    if (x < nodes) {
                        p[e] = a.parents ? a.parents[T.start[b] + x] : x - 1;
                        if (p[e] < -1 || p[e] >= x) bad = true, p[e] = -1;
                    }
                    m[e] = 1ull << x;
                }
                if (__any_sync(0xffffffffu, bad) && lane == 0) *(volatile int *)&S.bad_tree = 1;
                for (int step = 0; step < 6; ++step) {  // whole paths twice as long each time
                    uint64_t up[2];
                    int pp[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint64_t lo = __shfl_sync(0xffffffffu, m[0], p[e] & 31), hi = __shfl_sync(0xffffffffu, m[1], p[e] & 31);
                        const int plo = __shfl_sync(0xffffffffu, p[0], p[e] & 31), phi = __shfl_sync(0xffffffffu, p[1], p[e] & 31);
                        up[e] = p[e] < 0 ? 0 : p[e] < 32 ? lo : hi;
                        pp[e] = p[e] < 0 ? -1 : p[e] < 32 ? plo : phi;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) m[e] |= up[e], p[e] = pp[e];
                }
                const uint64_t lo = __shfl_sync(0xffffffffu, m[0], node & 31), hi = __shfl_sync(0xffffffffu, m[1], node & 31);
                anc = node < 32 ? lo : hi;
            }
            cp_async_wait_all();
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbarrier_arrive_one(&S.q_full[i]);
            Row r;
            for (int j = 0; j < nb; ++j, ++block, ++used_s) {
                ok = mbar_wait(&S.s_full[i], used_s & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                tc_fence_after();
                uint32_t s[KEYS];
#pragma unroll
                for (int x = 0; x < KEYS; x += 32) tmem_ld_32cols(ts + x, *reinterpret_cast<uint32_t(*)[32]>(&s[x]));
                tmem_ld_wait();
                const int k0 = (seg.t + j) * KEYS;
                const bool bad = *(volatile int *)&S.bad_page != 0;
                if (bad || k0 + KEYS > len) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int from = k0 + 32 * x - len;  // of the word's first key: its node
                        uint32_t see = from >= 0 ? (from < 64 ? (uint32_t)(anc >> from) : 0u)
                                                 : from <= -32 ? 0xffffffffu : (uint32_t)(anc << -from) | ((1u << -from) - 1);
                        if (bad) see &= *(volatile uint32_t *)&S.valid[block % TA_MASKS][x];
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (!(see >> y & 1)) s[32 * x + y] = __float_as_uint(-INFINITY);
                    }
                }
                softmax_block<D, FP16>(r, s, c, j == 0, ts, to);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive_one(&S.p_full[i]);
            }
            const int si = sn % L::RING_SEGS;
            if (ok) ok = mbar_wait(&S.o_full[i], used & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
            if (ok && ends) ok = mbar_wait(&S.tail[si], (sn / L::RING_SEGS) & 1, a.status, DEV_TIMEOUT_LOAD, &S.abort);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            tc_fence_after();
            ++used;
            const bool odd = ends && *(volatile int *)&S.odd[si];
            const float f = whole ? row_factor(r) : 1.f;
            const int place_row = i * ROWS + w * 32 + lane;
            float *po = a.part_o + (((long long)me * 2 + part) * a.part_rows + place_row) * D;
#pragma unroll 1
            for (int x = 0; x < D; x += 32) {
                uint32_t o[32];
                tmem_ld_32cols(to + x, o);
                tmem_ld_wait();
                if (odd)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (S.odd_all[si][x + e] || (S.odd_nodes[si][x + e] & anc)) o[e] = 0x7fffffffu;
                if (whole) {  // through the queries' place, so that neighbouring lanes store a row's pieces
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t v[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) v[y] = pack16<FP16>(__uint_as_float(o[e + 2 * y]) * f, __uint_as_float(o[e + 2 * y + 1]) * f);
                        st_shared_u4(place(lane, (x + e) >> 3), make_uint4(v[0], v[1], v[2], v[3]));
                    }
                } else if (real) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4 *>(po + x + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbarrier_arrive_one(&S.o_free[i]);
            const long long out_row = real ? (long long)(T.start[b] + node) * a.hq + head : -1;
            if (!whole) {
                if (real) a.part_ml[((long long)me * 2 + part) * a.part_rows + place_row] = make_float2(r.m, r.l);
                continue;
            }
            if (a.lse && real) a.lse[out_row] = row_lse<FP16>(r, a.scale);
#pragma unroll 4
            for (int x = 0; x < 32; x += RPI) {
                const int rr = x + lane / CPR;
                const long long o = __shfl_sync(0xffffffffu, out_row, rr);
                const uint4 v = ld_shared_u4(place(rr, piece));
                if (o >= 0) *reinterpret_cast<uint4 *>(a.out + o * D + piece * 8) = v;
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) tmem_dealloc(tmem, TM_COLS);
    if (threadIdx.x == 0) a.worker_code[me] = S.bad_page ? DEV_BAD_PAGE : S.bad_tree ? DEV_BAD_TREE : DEV_OK;
}

// Joins the parts of units that several CTAs worked on: a warp a row.  The first CTA reports.
constexpr int TJ_WARPS = 8;
template <int D, bool FP16>
__global__ void __launch_bounds__(32 * TJ_WARPS) k_tree_join(const __grid_constant__ PackedArgs a) {
    using L = TreeShape<D>;
    constexpr int PER = D / 32;
    __shared__ TreeList T;
    const int count = tree_list<D>(a, T), workers = workers_of(a, count);
    const int lane = threadIdx.x & 31;
    const float c = a.scale * 1.4426950408889634f;
    pdl_wait();
    if (blockIdx.x == 0) {
        int code = DEV_OK;
        for (int b = threadIdx.x; b < a.B; b += 32 * TJ_WARPS)
            if (!tree_ok(a, b)) code = DEV_BAD_POSITION;
        const int c5 = __syncthreads_or(code != DEV_OK);
        code = DEV_OK;
        for (int w = threadIdx.x; w < a.workers; w += 32 * TJ_WARPS) code = max(code, a.worker_code[w]);
        const int c7 = __syncthreads_or(code == DEV_BAD_PAGE), c9 = __syncthreads_or(code == DEV_BAD_TREE);
        if (threadIdx.x == 0 && (c5 | c7 | c9)) latch_error(a.status, c5 ? DEV_BAD_POSITION : c7 ? DEV_BAD_PAGE : DEV_BAD_TREE);
    }
    // (packed rows behind the last sequence's may be many)
    __shared__ int rows_end;
    if (threadIdx.x == 0) rows_end = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < a.B; b += 32 * TJ_WARPS)
        if (T.nodes[b] > 0) atomicMax(&rows_end, T.start[b] + T.nodes[b]);
    __syncthreads();
    for (long long x = (long long)blockIdx.x * TJ_WARPS + (threadIdx.x >> 5); x < (long long)rows_end * a.hq; x += (long long)gridDim.x * TJ_WARPS) {
        const int t = (int)(x / a.hq), head = (int)(x - (long long)t * a.hq);
        int b = -1;
        for (int b0 = 0; b < 0 && b0 < a.B; b0 += 32) {
            const int y = b0 + lane;
            const unsigned m = __ballot_sync(0xffffffffu, y < a.B && T.nodes[y] > 0 && T.start[y] <= t && t < T.start[y] + T.nodes[y]);
            if (m) b = b0 + __ffs(m) - 1;
        }
        if (b < 0) continue;
        const int h = head / a.group, row = (t - T.start[b]) * a.group + head - h * a.group, chunk = row / L::ROWS_ALL, pr = row - chunk * L::ROWS_ALL;
        const int blocks = blocks_of(T.len[b], T.nodes[b]), per = blocks + TA_ROW;
        const int at = T.first[b] + (h * chunks_of<D>(T.nodes[b] * a.group) + chunk) * per;
        const int w0 = worker_at(at + TA_ROW, count, workers), w1 = worker_at(at + per - 1, count, workers);
        if (w0 == w1) continue;  // one CTA had all blocks
        auto part = [&](int w) { return ((long long)w * 2 + (w == w0)) * a.part_rows + pr; };
        float m = -INFINITY;
        for (int w = w0; w <= w1; ++w) m = fmaxf(m, a.part_ml[part(w)].x);
        float l = 0.f, o[PER];
        for (int j = 0; j < PER; ++j) o[j] = 0.f;
        for (int w = w0; w <= w1; ++w) {
            const long long p = part(w);
            const float2 ml = a.part_ml[p];
            const float f = ml.x == m ? 1.f : ex2((ml.x - m) * c);
            l += ml.y * f;
            for (int j = 0; j < PER; ++j) o[j] += a.part_o[p * D + lane + 32 * j] * f;
        }
        const Row r{m, l};
        const float inv = row_factor(r);
        for (int j = 0; j < PER; ++j) {
            const float y = o[j] * inv;
            a.out[((long long)t * a.hq + head) * D + lane + 32 * j] = (uint16_t)pack16<FP16>(y, y);
        }
        if (a.lse && lane == 0) a.lse[(long long)t * a.hq + head] = row_lse<FP16>(r, a.scale);
    }
}

int rows_all(int d) { return (d == 256 ? 1 : 2) * ROWS; }

template <int D, bool FP16>
cudaError_t launch(PackedArgs &a, cudaStream_t st) {
    using L = TreeShape<D>;
    static_assert(L::SMEM + sizeof(TreeState<D>) + sizeof(TreeList) + 128 <= 227 * 1024, "shared memory");
    const cudaError_t e = cudaFuncSetAttribute(k_tree<D, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
    if (e != cudaSuccess) return e;
    a.workers = std::min(gemm_ctas(), TREE_MAX_WORKERS);
    if (a.workers < 1) return cudaErrorInvalidDevice;
    k_tree<D, FP16><<<a.workers, TA_THREADS, L::SMEM, st>>>(a);
    const long long rows = std::min<long long>(a.T, (long long)a.B * TREE_NODES) * a.hq;
    const int grid = (int)std::min<long long>((rows + TJ_WARPS - 1) / TJ_WARPS, 8ll * gemm_ctas());
    return launch_pdl(k_tree_join<D, FP16>, grid, 32 * TJ_WARPS, 0, st, a);
}

}  // namespace

bool tree_plan(const KvView &kv, int T, int hq, TreePlan *p) {
    // (places of the list are counted in 32 bits)
    const int most = rows_all(kv.d), group = hq / kv.hkv;
    const double units = (double)kv.B * kv.hkv * ((TREE_NODES * group + most - 1) / most);
    if (units * (double)((kv.cap + KEYS - 1) / KEYS + TA_ROW) >= 2147483647.0) return false;
    p->rows = std::min({most, TREE_NODES * group, std::min(T, 1 << 16) * group});
    size_t at = 1024;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += (bytes + 1023) / 1024 * 1024;
        return o;
    };
    const size_t parts = (size_t)TREE_MAX_WORKERS * 2 * p->rows;
    p->codes = take(TREE_MAX_WORKERS * sizeof(int));
    p->part_ml = take(parts * sizeof(float2));
    p->part_o = take(parts * kv.d * sizeof(float));
    p->total = at;
    return true;
}

cudaError_t launch_tree_attention(PackedArgs &a, cudaStream_t st) {
    if (a.fp16) return a.d == 64 ? launch<64, true>(a, st) : a.d == 128 ? launch<128, true>(a, st) : launch<256, true>(a, st);
    return a.d == 64 ? launch<64, false>(a, st) : a.d == 128 ? launch<128, false>(a, st) : launch<256, false>(a, st);
}

}  // namespace pbd
