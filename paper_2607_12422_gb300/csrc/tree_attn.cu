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
// 64 nodes behind 131071 slots, heads of 128: 106 us, between first and last block 6.4 TB/s (1.54 us a block of 64 KB an SM); the first scores are there
// 7 us after the start, and the join ends 11 us after the last block.  Heads of 64: a block takes the rows 1.0 us (memory 0.76), of two tiles 1.5.
// 17 nodes behind 512: 15 us, of which 5 pass before the first scores (7 with cold caches) and 3 in the join.  Heads of 256: 64 nodes behind 65535 slots
// 117 us, 4.6 TB/s in all.  Row by row, 16 bytes a lane (pages of 5 slots, of one): the first case takes 223 and 255 us.
//
// Warps 0-15: rows (queries, softmax, outputs).  Warp 16 copies K, warp 17 V: tiled copies of the rows that a page has in a piece where
// pages hold a multiple of 8, row by row else, 16 bytes a lane.  Warps 18 and 19: the tiles' MMAs.
// The blocks with nodes among their keys, a (sequence, KV head)'s last one or two, are copied row by row.  The rows' warps, of the second tile
// where a unit has one, store the nodes' rows into the cache and look for infinite and NaN values of V, which would be NaN in rows that
// do not see them (0 x NaN): who has one is noted for each dimension, and the warp that copies V makes such values zero before they are
// multiplied.  (Cached rows are seen by all.)  When the two warps that copy did all of this, eight trees of up to 64 nodes took 31.8 us, now 24.8.
#include <algorithm>

#include "flash.cuh"
#include "packed_ops.h"

namespace pbd {

using namespace flash;

namespace {

// Costs in places: of a block of a unit of one tile, of two, and of a unit besides.  Heads of 64: by the rows' work (1.0 and 1.5 us; 5 us); else
// memory bounds both (1.5 us; 6 us).  Measured, us, with places for a unit in front of the colon:
//     64 sequences of 1 to 26 nodes, seven heads of 64 a KV head      2: 110  6: 81  10: 69  14: 72  18: 75; one cost for all blocks and 3: 81
//     eight of up to 64 nodes, heads of 128                           1: 27.2  2: 27.2  4: 25.6  6: 26.1  8: 26.1  12: 27.4
//     64 nodes behind 131071 slots, heads of 128                      1: 103.7  2: 107  4: 106  6: 104.5  8: 104.2  12: 103.5
//     the eight, heads of 256                                         1: 41.2  2: 41.3  4: 40.0  6: 41.6  8: 42.9
//     the 64, heads of 256                                            1: 245  2: 214  4: 177  6: 174  8: 182
template <int D>
struct Cost {
    static constexpr int ONE = D == 64 ? 2 : 1, TWO = D == 64 ? 3 : 1, ROW = D == 64 ? 10 : 4;
};
constexpr int TA_MIN = 3;        // places of a CTA's stretch at least (17 nodes behind 512 slots: 14.7 us, with 4 15.5, with 6 16.9)
static_assert(TA_MIN >= Cost<64>::TWO, "who is in the middle of a unit has a block");
constexpr int TA_MASKS = 8;      // blocks whose masks are kept

template <int D>
struct TreeShape : Shape<D> {
    using S = Shape<D>;
    static constexpr int STAGES = D == 64 ? 4 : 2;  // units of the ring of K, and of V's
    static constexpr int RING_SEGS = D == 64 ? 8 : 4;  // segments that copies can be ahead, and one more
    static constexpr int ROWS_ALL = S::TILES * ROWS;
    static constexpr int SMEM = S::TILES * S::QT + 2 * STAGES * S::UNIT + 1024;
};

// Counts of the list: a (sequence, KV head, chunk of rows) is a unit; it has places in front, and some for each block.
struct TreeList {
    int first[KV_MAX_BATCH + 1];  // places before sequence b
    int len[KV_MAX_BATCH], nodes[KV_MAX_BATCH];
};

__device__ __forceinline__ int blocks_of(int len, int nodes) { return (len + nodes + KEYS - 1) / KEYS; }
template <int D>
__device__ __forceinline__ int chunks_of(int rows) { return (rows + TreeShape<D>::ROWS_ALL - 1) / TreeShape<D>::ROWS_ALL; }
// of a block of such a sequence's units (the last of several may be of one tile)
template <int D>
__host__ __device__ __forceinline__ int cost_of(int rows) { return TreeShape<D>::TILES == 2 && rows > ROWS ? Cost<D>::TWO : Cost<D>::ONE; }

// Whole CTA; returns the list's length.  bad: whether this thread has seen a sequence that is left out.  (Up to 32 sequences are one
// warp's: what comes before the first copy is what a small call waits for.)
template <int D>
__device__ __forceinline__ int tree_list(const PackedArgs &a, TreeList &T, bool &bad) {
    __shared__ int warp_sum[32], total;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    bool descends = false;
    auto places = [&](int b, bool out = false) {
        const int s = a.starts[b], e = a.starts[b + 1], l = a.kv.lens[b];
        const bool ok = !out && bounds_ok(a, s, e) && e - s <= TREE_NODES && l >= 0 && l + (long long)(e - s) <= a.kv.cap;
        const int n = ok ? e - s : 0, len = ok ? l : 0;
        bad |= !ok;
        descends |= e < s;
        T.len[b] = len, T.nodes[b] = n;
        return n > 0 ? a.hkv * chunks_of<D>(n * a.group) * (blocks_of(len, n) * cost_of<D>(n * a.group) + Cost<D>::ROW) : 0;
    };
    auto scan = [&](int x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        return x;
    };
    if (threadIdx.x == 0) T.first[0] = 0;
    if (a.B <= 32) {
        if (warp == 0) {
            int x = lane < a.B ? places(lane) : 0;
            if (__any_sync(0xffffffffu, descends) && lane < a.B) x = places(lane, !behind_all(a.starts, lane));
            x = scan(x);
            if (lane < a.B) T.first[lane + 1] = x;
            if (lane == 31) total = x;
        }
        __syncthreads();
        return total;
    }
    int carry = 0;
    for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        int x = scan(b < a.B ? places(b) : 0);
        if (lane == 31) warp_sum[warp] = x;
        if (__syncthreads_or(descends)) {  // (here or in front)
            x = scan(b < a.B ? places(b, !behind_all(a.starts, b)) : 0);
            if (lane == 31) warp_sum[warp] = x;
            __syncthreads();
        }
        const int sums = scan(lane < n_warps ? warp_sum[lane] : 0);
        const int before = carry + (warp ? __shfl_sync(0xffffffffu, sums, warp - 1) : 0);
        if (b < a.B) T.first[b + 1] = before + x;
        carry += __shfl_sync(0xffffffffu, sums, 31);
        __syncthreads();
    }
    return carry;
}

// CTAs that share the list, the first place of one of them, and the one that has a place.
struct Shares {
    int workers, each, more;  // places of a CTA; CTAs with one more
    __device__ __forceinline__ Shares(const PackedArgs &a, int count) {
        workers = max(1, min(a.workers, count / TA_MIN));  // (so that one in the middle of a unit has a block)
        each = count / workers;
        more = count - each * workers;
    }
    __device__ __forceinline__ int first(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int at) const {
        const int big = more * (each + 1);
        return at < big ? at / (each + 1) : more + (at - big) / each;
    }
};

// Blocks [t, t_end) of one unit: what a CTA works on before it leaves the unit.
struct Segment {
    int b, unit, units, t, t_end, blocks, cost;  // sequence, unit of it, its units, blocks, the unit's blocks, places of one
    int at, end;                           // list place of the unit, end of the stretch
    int chunks;
    template <int D>
    __device__ __forceinline__ void enter(const PackedArgs &a, const TreeList &T) {
        blocks = blocks_of(T.len[b], T.nodes[b]);
        chunks = chunks_of<D>(T.nodes[b] * a.group);
        cost = cost_of<D>(T.nodes[b] * a.group);
        units = a.hkv * chunks;
    }
    // the block that has place x of the unit or is the first behind it: a block belongs to whom its first place does
    template <int D>
    __device__ __forceinline__ int block_at(int x) const { return max(x - Cost<D>::ROW + cost - 1, 0) / cost; }
    template <int D>
    __device__ __forceinline__ bool clip() {
        t_end = min(blocks, block_at<D>(end - at));
        return t < t_end;
    }
    // The unit that has place u; false if there is none.
    template <int D>
    __device__ __forceinline__ bool find(int u, const PackedArgs &a, const TreeList &T) {
        int lo = 0, hi = a.B;  // first[lo] <= u < first[hi]
        if (u >= T.first[hi]) return false;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (T.first[mid] <= u)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
        enter<D>(a, T);
        const int per = blocks * cost + Cost<D>::ROW;
        unit = (u - T.first[b]) / per;
        at = T.first[b] + unit * per;
        return true;
    }
    // The first segment of the stretch [u, u_end); false if it has none.
    template <int D>
    __device__ __forceinline__ bool seek(int u, int u_end, const PackedArgs &a, const TreeList &T) {
        end = u_end;
        if (u >= end || !find<D>(u, a, T)) return false;
        t = block_at<D>(u - at);
        return clip<D>() || next<D>(a, T);
    }
    template <int D>
    __device__ __forceinline__ bool next(const PackedArgs &a, const TreeList &T) {
        at += blocks * cost + Cost<D>::ROW;
        t = 0;
        if (++unit == units) {
            unit = 0;
            do ++b;
            while (b < a.B && T.first[b + 1] == T.first[b]);
            if (b >= a.B || at >= end) return false;
            enter<D>(a, T);
        }
        return at < end && clip<D>();  // (where only a unit's front is left the stretch is over)
    }
};

template <int D>
struct TreeState {
    using L = TreeShape<D>;
    // s_full, p_full: S and P of the first tile's place, of the second tile, and of the second place where one tile uses both.  (Each has one
    // party that arrives and one that waits, and they see all of its phases: who skips one takes an older one for it.)
    uint64_t full[2][L::STAGES], empty[2][L::STAGES], q_full[2], s_full[3], p_full[3][2], o_done[2], o_free[2], turn[2], drain[2];
    uint64_t notes_ready[L::RING_SEGS], notes_made[L::RING_SEGS], notes_free[L::RING_SEGS];
    uint32_t tmem;
    uint32_t patience;  // mbar_wait_short
    int bad_page, bad_tree;
    float top[2][2][ROWS];              // what the two threads of a row tell each other
    Segment row_seg[ROW_WARPS];         // where each of the rows' warps is (to spare registers)
    alignas(8) uint32_t valid[TA_MASKS][4];  // keys of a block whose pages are in the cache
    unsigned long long rows[2][KEYS];  // where a block's rows of K, and of V, come from; of pieces: the map's coordinates
    // of a segment: whether there are, and which nodes have infinite or NaN values, in each dimension
    int odd[L::RING_SEGS];
    unsigned long long odd_nodes[L::RING_SEGS][D];
};

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool real) {
    const int n = real ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// Arrives on `bar` once this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbarrier_arrive_many(uint64_t *bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}

// box: rows of a page that one tiled copy brings (0: none do); page_step: a page's stride in heads.
template <int D, bool FP16>
__global__ void __launch_bounds__(THREADS, 1)
    k_tree(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ PackedArgs a, int box, int page_step) {
    using L = TreeShape<D>;
    constexpr int TILES = L::TILES, UNITS = L::UNITS, STAGES = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sq = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *ring = sq + TILES * L::QT;
    __shared__ TreeState<D> S;
    __shared__ TreeList T;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    pdl_launch();
    if (warp == 18) tmem_alloc(&S.tmem, TM_COLS);
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            for (int kv = 0; kv < 2; ++kv) {
                mbar_init(&S.full[kv][i], box ? 1 : 32);
                mbar_init(&S.empty[kv][i], 2);
            }
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&S.q_full[i], 8);
            mbar_init(&S.o_done[i], 1);
            mbar_init(&S.o_free[i], 8);
            mbar_init(&S.turn[i], 1);
            mbar_init(&S.drain[i], 1);
        }
        for (int i = 0; i < 3; ++i) {
            mbar_init(&S.s_full[i], 1);
            mbar_init(&S.p_full[i][0], 8);
            mbar_init(&S.p_full[i][1], 8);
        }
        for (int i = 0; i < L::RING_SEGS; ++i) {
            mbar_init(&S.notes_ready[i], 1);
            mbar_init(&S.notes_made[i], ROW_WARPS);
            mbar_init(&S.notes_free[i], ROW_WARPS);
            S.odd[i] = 0;
        }
        S.patience = a.patience;
        S.bad_page = S.bad_tree = 0;
        fence_mbarrier_init();
        if (blockIdx.x == 0) *a.status = DEV_OK;  // (k_tree_join reports; a wait runs out a second later)
    }
    for (int x = threadIdx.x; x < L::RING_SEGS * D; x += THREADS) (&S.odd_nodes[0][0])[x] = 0;
    if (threadIdx.x == 32 && box) {
        prefetch_tensormap(&kmap);
        prefetch_tensormap(&vmap);
    }
    tc_fence_before();
    bool left_out = false;
    const int count = tree_list<D>(a, T, left_out);  // (its barriers order what is above, too)
    const Shares shares(a, count);
    const int me = blockIdx.x;
    tc_fence_after();
    const uint32_t tmem = S.tmem;
    Segment seg{};
    bool more = me < shares.workers && seg.seek<D>(shares.first(me), shares.first(me + 1), a, T);
    // rows of the segment's unit from its chunk's first on
    auto rows_of = [&]() { return T.nodes[seg.b] * a.group - (seg.unit % seg.chunks) * L::ROWS_ALL; };

    if (warp >= ROW_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
        if (warp < 18) {
            // ---- copies: warp 16 K, warp 17 V.  (Warps that run little beside others that run much fetch their code anew each time, at about 6
            // cycles an instruction: whole blocks of cached slots have a short path of their own.)
            const int kv = warp - 16;
            constexpr int CPR = L::DU / 8, RPI = 32 / CPR;  // 16-byte pieces of a unit's row, rows of a step
            using Y = Layout<D, true>;
            const int piece = lane % CPR, r_lane = lane / CPR, pieces = box ? KEYS / box : 0;
            unsigned long long *rows = S.rows[kv];
            const CUtensorMap *map = kv ? &vmap : &kmap;
            uint8_t *units = ring + kv * STAGES * L::UNIT;
            int issued = 0, block = 0, sn = 0;
            bool ok = true;
            int pend = -1, pend_t = 0;  // the unit of rows that has still to be looked at
            // What a lane says of a unit that it has copied: with tiled copies one lane for its warp.
            auto arrive = [&](uint64_t *bar) {
                if (box) __syncwarp();
                if (!box || lane == 0) mbarrier_arrive_one(bar);
            };
            auto next_slot = [&]() {
                const int slot = issued % STAGES;
                ok = __all_sync(0xffffffffu, mbar_wait_short(&S.empty[kv][slot], ((issued / STAGES) & 1) ^ 1, a.status, DEV_TIMEOUT_SLOT, &S.patience));
                ++issued;
                return slot;
            };
            // A piece's place in the map, packed: page and head in one (outside the map for a page outside the cache: the copy brings
            // zeros, which no weight makes NaN), and eights of the page.
            auto packed = [&](int page, int h, int key) {
                const bool bad = (unsigned)page >= (unsigned)a.kv.n_pages;
                return (unsigned long long)(unsigned)(bad ? -1 : page * page_step + h) << 32 | (unsigned)(key - page_index(a.kv, key) * a.kv.page_size) / 8;
            };
            auto copy_piece = [&](uint8_t *unit, int r, int u, uint64_t *bar) {
                const unsigned long long at = rows[r];
                tma_load_5d(unit + r / 8 * Y::EIGHT, map, 0, 0, u * (L::DU / 64), (int)(unsigned)at, (int)(at >> 32), bar);
            };
            for (; ok && more; ++sn) {
                const int b = seg.b, len = T.len[b], nodes = T.nodes[b], h = seg.unit / seg.chunks;
                const int tail0 = len / KEYS, si = sn % L::RING_SEGS;  // (the first block with nodes or places behind them)
                const int *table = a.kv.table + (long long)b * a.kv.max_pages;
                int t = seg.t;
                if (tail0 * KEYS + lane < len + nodes)  // (a load each in turn later)
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(table + page_index(a.kv, min(tail0 * KEYS + 4 * lane, len + nodes - 1))));
                if (kv && seg.t_end > tail0) {
                    // room for this segment's notes: all rows are through with those that were there.  (Said before the first copy: rows wait for it.)
                    if (sn >= L::RING_SEGS)
                        ok = __all_sync(0xffffffffu, mbar_wait_short(&S.notes_free[si], (sn / L::RING_SEGS - 1) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience));
                    if (ok && S.odd[si]) {
                        __syncwarp();
                        for (int d = lane; d < D; d += 32) S.odd_nodes[si][d] = 0;
                        if (lane == 0) S.odd[si] = 0;
                    }
                    __syncwarp();
                    if (ok && lane == 0) mbarrier_arrive_one(&S.notes_ready[si]);
                }
                if (box && t < min(tail0, seg.t_end)) {
                    int page = lane < pieces ? table[page_index(a.kv, t * KEYS + lane * box)] : 0;
#pragma unroll 1
                    for (; ok && t < min(tail0, seg.t_end); ++t) {
                        const int key = t * KEYS + lane * box;
                        __syncwarp();
                        if (lane < pieces) rows[lane * box] = packed(page, h, key);
                        const unsigned lost = __ballot_sync(0xffffffffu, lane < pieces && (unsigned)page >= (unsigned)a.kv.n_pages);
                        if (lost) *(volatile int *)&S.bad_page = 1;
                        if (kv == 0 && lane < 4) {
                            uint32_t valid = 0xffffffffu;
                            if (lost)
                                for (int r = 0; r < 32; ++r)
                                    if (lost >> ((32 * lane + r) / box) & 1) valid &= ~(1u << r);
                            *(volatile uint32_t *)&S.valid[(block + t - seg.t) % TA_MASKS][lane] = valid;
                        }
                        if (lane < pieces && t + 1 < min(tail0, seg.t_end)) page = table[page_index(a.kv, key + KEYS)];
                        __syncwarp();
#pragma unroll 1
                        for (int u = 0; u < UNITS; ++u) {
                            const int slot = next_slot();
                            if (!ok) break;
                            if (elect_one()) {
                                uint64_t *bar = &S.full[kv][slot];
                                mbar_arrive_expect_tx(bar, (uint32_t)L::UNIT);
#pragma unroll 1
                                for (int r = 0; r < KEYS; r += box) copy_piece(units + slot * L::UNIT, r, u, bar);
                            }
                            __syncwarp();
                        }
                    }
                }
                // Blocks with nodes, and all where pages hold no multiple of 8.  Rows behind `hi` are not multiplied.
                const int start = a.starts[b];
                auto row_hi = [&](int t) { return min(((len + nodes + 15) & ~15) - t * KEYS, KEYS); };
                // The last unit that was copied.  V: once the rows have looked at the nodes' values, of which some become zero.
                auto finish = [&]() {
                    if (kv) {
                        ok = __all_sync(0xffffffffu, mbar_wait_short(&S.notes_made[si], (sn / L::RING_SEGS) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience));
                        if (*(volatile int *)&S.odd[si]) {
                            const uint32_t to = smem_u32(units + pend * L::UNIT);
                            const int k0 = pend_t * KEYS;
#pragma unroll 1
                            for (int r = max(len - k0, 0) / RPI * RPI + r_lane; r < row_hi(pend_t); r += RPI) {  // (each lane its own pieces)
                                if (k0 + r < len) continue;
#pragma unroll 1
                                for (int e = 0; e < 8; ++e) {  // (value by value: this is rare)
                                    const uint32_t at = to + Y::at(r, piece) + 2 * e;
                                    uint16_t y;
                                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(at) : "memory");
                                    if (odd_halves<FP16>(y)) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"((uint16_t)0) : "memory");
                                }
                            }
                        }
                    }
                    fence_proxy_async_shared();
                    arrive(&S.full[kv][pend]);
                    pend = -1;
                };
#pragma unroll 1
                for (; ok && t < seg.t_end; ++t) {
                    const bool tail = t >= tail0;
                    const int lo = box ? max(min((len - t * KEYS) / box * box, KEYS), 0) : 0, hi = row_hi(t);  // (rows below lo come in pieces)
                    if (pend >= 0) {  // (its rows are looked up below)
                        cp_async_wait_all();
                        finish();
                    }
                    __syncwarp();
                    auto page_of = [&](int key) { return key < len + nodes ? table[page_index(a.kv, key)] : -1; };
                    int next_page = page_of(t * KEYS + lane);
#pragma unroll 1
                    for (int e = 0; 32 * e < hi; ++e) {
                        const int r = 32 * e + lane, key = t * KEYS + r, pi = page_index(a.kv, key), page = next_page;
                        next_page = page_of(key + 32);
                        const bool cached = key < len, node = !cached && key < len + nodes;
                        const bool real = (unsigned)page < (unsigned)a.kv.n_pages;
                        if ((cached || node) && !real) *(volatile int *)&S.bad_page = 1;
                        unsigned long long at = 0;
                        if (r < lo) {
                            at = packed(page, h, key);
                        } else if (real) {
                            const long long slot = page * a.kv.stride_page + h * a.kv.stride_head + (key - pi * a.kv.page_size) * a.kv.stride_slot;
                            const uint16_t *from = cached ? (kv ? a.kv.v : a.kv.k) + slot : (kv ? a.v : a.k) + (long long)(start + key - len) * a.kv_stride + h * D;
                            at = reinterpret_cast<unsigned long long>(from);
                        }
                        rows[r] = at;
                        const unsigned valid = __ballot_sync(0xffffffffu, real);
                        if (kv == 0 && lane == 0) *(volatile uint32_t *)&S.valid[(block + t - seg.t) % TA_MASKS][e] = valid;
                    }
                    __syncwarp();
#pragma unroll 1
                    for (int u = 0; ok && u < UNITS; ++u) {
                        const int slot = next_slot();
                        if (!ok) break;
                        uint64_t *bar = &S.full[kv][slot];
                        uint8_t *unit = units + slot * L::UNIT;
                        if (lo > 0 && elect_one()) {
                            mbar_expect_tx(bar, (uint32_t)(lo * L::DU * 2));
#pragma unroll 1
                            for (int r = 0; r < lo; r += box) copy_piece(unit, r, u, bar);
                        }
                        __syncwarp();
                        if (hi <= lo) {
                            arrive(bar);
                            continue;
                        }
                        const uint32_t to = smem_u32(unit);
#pragma unroll 1
                        for (int x0 = lo; x0 < hi; x0 += 8 * RPI) {
                            unsigned long long src[8];
#pragma unroll
                            for (int y = 0; y < 8; ++y) src[y] = rows[min(x0 + y * RPI, KEYS - RPI) + r_lane];
#pragma unroll
                            for (int y = 0; y < 8; ++y)
                                if (x0 + y * RPI < hi)
                                    cp_async16_or_zero(to + Y::at(x0 + y * RPI + r_lane, piece),
                                                       src[y] ? reinterpret_cast<const uint16_t *>(src[y]) + u * L::DU + piece * 8 : a.q, src[y] != 0);
                        }
                        if (!tail) {
                            cp_async_arrive(bar);
                            continue;
                        }
                        cp_async_commit();
                        if (pend >= 0) {
                            cp_async_wait_1();
                            finish();
                        }
                        pend = slot, pend_t = t;
                    }
                }
                if (ok && pend >= 0) {
                    cp_async_wait_all();
                    finish();
                }
                block += seg.t_end - seg.t;
                more = seg.next<D>(a, T);
            }
            cp_async_commit();
            cp_async_wait_all();  // also on the error path: nothing is in flight when the CTA ends
            if (*(volatile uint32_t *)&S.patience == 0) {  // (and tiled copies get a bounded chance to land)
                const uint64_t t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < WAIT_LIMIT_NS / 100) __nanosleep(1000);
            }
        } else if (warp < 18 + TILES && elect_one()) {
            // ---- MMAs of tile i
            const int i = warp - 18;
            const uint8_t *q = sq + i * L::QT;
            const uint32_t o = tmem + TM_O + i * D;
            int pos = 0, step = 0, used_o = 0, cnt0 = 0, cnt1 = 0, cnt2 = 0, twos = 0;  // blocks, sections, segments of the tile, phases of s_full, segments of two tiles
            bool ok = true;
            auto wait = [&](uint64_t *bar, int phase, int code) { ok = ok && mbar_wait_short(bar, phase & 1, a.status, code, &S.patience); };
            auto landed = [&](int kv, int j) {  // K or V of the CTA's block j
                for (int u = 0; u < UNITS; ++u) wait(&S.full[kv][(j * UNITS + u) % STAGES], (j * UNITS + u) / STAGES, DEV_TIMEOUT_LOAD);
                if (!box) fence_proxy_async_shared();  // (cp.async's copies land in the generic proxy)
            };
            auto unit = [&](int kv, int j, int u) { return ring + (kv * STAGES + (j * UNITS + u) % STAGES) * L::UNIT; };
            auto scores = [&](int buf, int bar, int j) {
                for (int u = 0; u < UNITS; ++u) mma_scores<D, FP16, true>(tmem + buf * KEYS, q, unit(0, pos + j, u), u);
                mma_commit(&S.s_full[bar]);
            };
            while (ok && more) {
                const int nb = seg.t_end - seg.t, keys = T.len[seg.b] + T.nodes[seg.b] - seg.t * KEYS;
                const bool two = TILES == 2 && rows_of() > ROWS;
                auto values = [&](int buf, int bar, int j, int phase) {
                    const int steps = min(KEYS, keys - j * KEYS + 15) / 16;  // (keys behind the last are not multiplied, to 16)
                    for (int u = 0; u < UNITS; ++u) mma_values<D, FP16, true>(o, tmem + buf * KEYS, unit(1, pos + j, u), u, 0, steps, j == 0);
                    wait(&S.p_full[bar][1], phase, DEV_TIMEOUT_MMA);
                    if (!ok) return;
                    tc_fence_after();
                    for (int u = 0; u < UNITS; ++u) mma_values<D, FP16, true>(o, tmem + buf * KEYS, unit(1, pos + j, u), u, 1, steps, j == 0);
                };
                auto values_ready = [&](int j) {
                    landed(1, pos + j);
                    if (j == 0 && used_o > 0) wait(&S.o_free[i], used_o - 1, DEV_TIMEOUT_MMA);
                };
                if (two) {  // for every block O += P V of the one before, then S; the tiles in turns
                    const int cnt = i ? cnt1 : cnt0;
                    wait(&S.q_full[i], used_o, DEV_TIMEOUT_LOAD);
#pragma unroll 1
                    for (int j = 0; ok && j <= nb; ++j, ++step) {
                        if (i + step > 0) wait(&S.turn[i], step + i - 1, DEV_TIMEOUT_MMA);
                        if (j > 0) values_ready(j - 1);
                        if (j < nb) landed(0, pos + j);
                        if (j > 0) wait(&S.p_full[i][0], cnt + j - 1, DEV_TIMEOUT_MMA);
                        if (!ok) break;
                        tc_fence_after();
                        if (j > 0) values(i, i, j - 1, cnt + j - 1);
                        if (ok && j < nb) scores(i, i, j);
                        mbarrier_arrive_one(&S.turn[i ^ 1]);
                        if (j == nb) mma_commit(&S.o_done[i]);
                    }
                    cnt0 += nb, cnt1 += nb;
                    ++used_o, ++twos;
                } else {  // S of the next block, then O += P V of this one
                    if (i == 0) {
                        wait(&S.q_full[0], used_o, DEV_TIMEOUT_LOAD);
                        landed(0, pos);
                        if (ok) {
                            tc_fence_after();
                            scores(0, 0, 0);
                        }
                        if (twos > 0) wait(&S.o_done[1], twos - 1, DEV_TIMEOUT_MMA);  // (the second tile has left the second place)
#pragma unroll 1
                        for (int j = 0; ok && j < nb; ++j) {
                            const int buf = j & 1;
                            if (j + 1 < nb) {
                                landed(0, pos + j + 1);
                                if (!ok) break;
                                tc_fence_after();
                                scores(buf ^ 1, buf ? 0 : 2, j + 1);
                            }
                            const int phase = (buf ? cnt2 : cnt0) + (j >> 1), bar = 2 * buf;
                            values_ready(j);
                            wait(&S.p_full[bar][0], phase, DEV_TIMEOUT_MMA);
                            if (!ok) break;
                            tc_fence_after();
                            values(buf, bar, j, phase);
                            mma_commit(&S.o_done[0]);
                        }
                        ++used_o;
                    }
                    cnt0 += (nb + 1) / 2, cnt2 += nb / 2;
                }
                pos += nb;
                more = seg.next<D>(a, T);
            }
            mma_commit(&S.drain[i]);  // every MMA issued completes before TMEM is released
            mbar_wait_short(&S.drain[i], 0, nullptr, 0, nullptr);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ROW_REGS));
        // ---- rows: row r of tile i is the unit's row 128 i + r: node row / group, head row % group
        const int i = warp >> 3, half = (warp >> 2) & 1, w = warp & 3, id = 1 + i * 4 + w, place_row = i * ROWS + w * 32 + lane;
        const uint32_t lanes = (uint32_t)(w * 32) << 16, ts = tmem + lanes + 64 * half, to = tmem + lanes + TM_O + i * D + half * (D / 2);
        const float c = a.scale * 1.4426950408889634f;
        float *top = S.top[i][0];
        Row r{0.f, 0.f};
        int o_phase = 0, cnt = 0, cnt2 = 0, block = 0, sn = 0;  // phases of o_done, of the tile's s_full, of the second place's; blocks, segments
        bool ok = true;
        S.row_seg[warp] = seg;
        auto advance = [&]() {
            __syncwarp();
            Segment g = S.row_seg[warp];
            const bool any = g.next<D>(a, T);
            __syncwarp();
            S.row_seg[warp] = g;
            return any;
        };
        for (; ok && more; ++sn, more = advance()) {
            __syncwarp();
            const Segment *g = &S.row_seg[warp];
            const int b = g->b, nb = g->t_end - g->t, first_row = g->unit % g->chunks * L::ROWS_ALL, n_rows = T.nodes[b] * a.group - first_row;
            const int from0 = g->t * KEYS + 64 * half - T.len[b];  // the node of this thread's first key, cached ones below 0
            const bool two = TILES == 2 && n_rows > ROWS, whole = nb == g->blocks, ends = g->t_end > T.len[b] / KEYS;  // (ends: nodes among its keys)
            const int pos = block;
            block += nb;
            const bool idle = i && !two;  // the second tile's rows of a unit of one
            auto release = [&](int kv, int j) {  // K or V of a block is not needed any more
                if (w == 0 && half == 0 && lane == 0)
                    for (int u = 0; u < UNITS; ++u) mbarrier_arrive_many(&S.empty[kv][((pos + j) * UNITS + u) % STAGES], two ? 1 : 2);
            };
            const bool real = place_row < n_rows;
            const int node = real ? (place_row + first_row) / a.group : 0;
            uint64_t anc = 0;
            if (!idle) {
                int p[2];  // ancestors: lane x holds nodes x and x + 32
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int x = lane + 32 * e;
                    p[e] = ends && x < T.nodes[b] ? (a.parents ? a.parents[a.starts[b] + x] : x - 1) : -1;
                }
                {  // the queries (the tile's last MMAs are done); a row's two warps share its pieces
                    constexpr int CPH = D / 16, RPI = 32 / CPH;
                    const int piece = half * CPH + lane % CPH;
                    const uint32_t mine = smem_u32(sq + i * L::QT) + (piece >> 3) * SUB + w * 32 * 128;
                    const int head = g->unit / g->chunks * a.group + place_row + first_row - node * a.group;
                    const long long q_off = real ? (long long)(a.starts[b] + node) * a.q_stride + head * D : -1;
#pragma unroll 4
                    for (int x = 0; x < 32; x += RPI) {
                        const int rr = x + lane / CPH;
                        const long long off = __shfl_sync(0xffffffffu, q_off, rr);
                        cp_async16_or_zero(mine + rr * 128 + (((piece & 7) ^ (rr & 7)) << 4), off >= 0 ? a.q + off + piece * 8 : a.q, off >= 0);
                    }
                    cp_async_commit();
                }
                if (ends) {
                    uint64_t m[2];
                    bool bad = false;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int x = lane + 32 * e;
                        if (p[e] < -1 || p[e] >= x) bad = true, p[e] = -1;
                        m[e] = 1ull << x;
                    }
                    if (__any_sync(0xffffffffu, bad) && lane == 0) *(volatile int *)&S.bad_tree = 1;
#pragma unroll 1
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
            }
            if (ends && (two || i)) {  // the nodes' K and V go to the cache, and V is looked at: by rows that have nothing else to do, if there are
                constexpr int CPR = D / 8;
                const int si = sn % L::RING_SEGS;
                const bool room = __all_sync(0xffffffffu, mbar_wait_short(&S.notes_ready[si], (sn / L::RING_SEGS) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience));
                const int h = g->unit / g->chunks, start = a.starts[b], len = T.len[b], first = two ? 0 : ROW_WARPS * 16;
                const int from = max(g->t * KEYS - len, 0), to = min(T.nodes[b], g->t_end * KEYS - len);  // (of this stretch's blocks)
#pragma unroll 1
                for (int x = threadIdx.x - first; room && x < (to - from) * CPR; x += ROW_WARPS * 32 - first) {
                    const int n = from + x / CPR, p = x % CPR, key = len + n, pi = page_index(a.kv, key);
                    const long long src = (long long)(start + n) * a.kv_stride + h * D + p * 8;
                    const uint4 k = *reinterpret_cast<const uint4 *>(a.k + src), v = *reinterpret_cast<const uint4 *>(a.v + src);
                    const int page = a.kv.table[(long long)b * a.kv.max_pages + pi];
                    if ((unsigned)page >= (unsigned)a.kv.n_pages) continue;
                    if (first_row == 0) {
                        const long long dst = page * a.kv.stride_page + h * a.kv.stride_head + (key - pi * a.kv.page_size) * a.kv.stride_slot + p * 8;
                        *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.k) + dst) = k;
                        *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.v) + dst) = v;
                        if (p == 0 && a.new_pos && a.kv.positions) a.kv.positions[((long long)b * a.hkv + h) * a.kv.cap + key] = a.new_pos[start + n];
                    }
                    if (!(odd_halves<FP16>(v.x) | odd_halves<FP16>(v.y) | odd_halves<FP16>(v.z) | odd_halves<FP16>(v.w))) continue;
#pragma unroll 1
                    for (int e = 0; e < 8; ++e)  // (value by value: this is rare)
                        if (odd_halves<FP16>(a.v[src + e])) atomicOr(&S.odd_nodes[si][p * 8 + e], 1ull << n);
                    *(volatile int *)&S.odd[si] = 1;
                }
                __syncwarp();
                if (room && lane == 0) mbarrier_arrive_many(&S.notes_made[si], two ? 1 : 2);
            }
            if (idle) continue;
            for (int j = 0; ok && j < nb; ++j) {
                const int buf = two ? i : j & 1, bar = two ? i : 2 * buf, phase = two ? cnt + j : (buf ? cnt2 : cnt) + (j >> 1);
                bool there = mbar_wait_short(&S.s_full[bar], phase & 1, a.status, DEV_TIMEOUT_MMA, &S.patience), o_waited = two || j == 0;
                there = __all_sync(0xffffffffu, there);
                release(0, j);
                if (two && j > 0) release(1, j - 1);
                tc_fence_after();
                uint32_t s[64];
#pragma unroll
                for (int x = 0; x < 64; x += 32) tmem_ld_32cols(ts + buf * KEYS + x, *reinterpret_cast<uint32_t(*)[32]>(&s[x]));
                tmem_ld_wait();
                const bool bad = *(volatile int *)&S.bad_page != 0;
                if (bad || from0 + j * KEYS + 64 > 0) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int from = from0 + j * KEYS + 32 * x;  // of the word's first key
                        uint32_t see = from >= 0 ? (from < 64 ? (uint32_t)(anc >> from) : 0u)
                                                 : from <= -32 ? 0xffffffffu : (uint32_t)(anc << -from) | ((1u << -from) - 1);
                        if (bad) see &= *(volatile uint32_t *)&S.valid[(pos + j) % TA_MASKS][2 * half + x];
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (!(see >> y & 1)) s[32 * x + y] = __float_as_uint(-INFINITY);
                    }
                }
                auto o_ready = [&]() {  // (with two tiles S of this block has come after O of the one before)
                    bool o = true;
                    if (!o_waited) {
                        o = mbar_wait_short(&S.o_done[0], (o_phase + j - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.patience);
                        release(1, j - 1);
                    }
                    o_waited = true;
                    return __all_sync(0xffffffffu, o) != 0;
                };
                ok = softmax_half<D, FP16>(r, s, there, c, j == 0, ts + buf * KEYS, to, id, top, half, w * 32 + lane, o_ready, [&](int part) {
                    if (!two && part == 1) o_ready();  // (every phase is waited for)
                    if (lane == 0) mbarrier_arrive_one(&S.p_full[bar][part]);
                });
            }
            cnt += two ? nb : (nb + 1) / 2;
            if (!two) cnt2 += nb / 2;
            o_phase += two ? 1 : nb;
            const int si = sn % L::RING_SEGS;
            bool there = mbar_wait_short(&S.o_done[i], (o_phase - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.patience);
            if (there && ends) there = mbar_wait_short(&S.notes_made[si], (sn / L::RING_SEGS) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience);
            release(1, nb - 1);
            if (!ok || pair_any(id, !there)) break;
            top[half * ROWS + w * 32 + lane] = r.l;
            pair_sync(id);
            r.l += top[(half ^ 1) * ROWS + w * 32 + lane];
            tc_fence_after();
            const bool odd = ends && *(volatile int *)&S.odd[si];
            auto drop = [&](int d) { return (S.odd_nodes[si][half * (D / 2) + d] & anc) != 0; };
            const Segment *e = &S.row_seg[warp];  // (read again)
            const int row = place_row + e->unit % e->chunks * L::ROWS_ALL, head = e->unit / e->chunks * a.group + row % a.group;
            const long long out_row = (long long)(a.starts[e->b] + row / a.group) * a.hq + head;
            if (whole) {
                store_half<D, FP16>(to, row_factor(r), a.out + out_row * D + half * (D / 2), real, (reinterpret_cast<uintptr_t>(a.out) & 31) == 0, odd, drop);
                if (a.lse && half == 0 && real) a.lse[out_row] = row_lse<FP16>(r, a.scale);
            } else {  // a row's four values beside those of its neighbours
                const long long part = (long long)me * 2 + (e->t == 0);  // of units a stretch has at most two parts: an end and a beginning
                float4 *po = reinterpret_cast<float4 *>(a.part_o) + (part * (D / 4) + half * (D / 8)) * a.part_rows + place_row;
#pragma unroll 1
                for (int x = 0; x < D / 2; x += 16) {
                    uint32_t v[16];
                    tmem_ld_16cols(to + x, v);
                    tmem_ld_wait();
                    if (odd)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (drop(x + e)) v[e] = 0x7fffffffu;
                    if (real)
#pragma unroll
                        for (int e = 0; e < 16; e += 4)
                            po[(long long)((x + e) / 4) * a.part_rows] =
                                make_float4(__uint_as_float(v[e]), __uint_as_float(v[e + 1]), __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
                }
                if (real && half == 0) a.part_ml[part * a.part_rows + place_row] = make_float2(r.m, r.l);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbarrier_arrive_one(&S.o_free[i]);
                mbarrier_arrive_many(&S.notes_free[si], two ? 1 : 2);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 18) tmem_dealloc(tmem, TM_COLS);
    if (threadIdx.x == 0) a.worker_code[me] = S.bad_page ? DEV_BAD_PAGE : S.bad_tree ? DEV_BAD_TREE : DEV_OK;
}

// Joins the parts of units that several CTAs worked on: a warp 32 dimensions of four rows of a unit (node by node, the heads of its
// group innermost), eight lanes a row.  Parts are taken eight at a time, whose loads go out together (one after the other, 64 nodes
// behind 131071 slots, whose units have 20 parts, took 50 us here).  Every CTA counts the tasks of such units, so that all warps get as
// many (going over all rows instead and leaving out most: 64 ragged sequences 75.6 us instead of 71.3; 17 nodes behind 512 slots 16 instead of 14.5).
// The first CTA reports.
constexpr int TJ_WARPS = 8, TJ_ROWS = 4;
static_assert(TREE_MAX_WORKERS <= 32 * TJ_WARPS, "a thread a CTA of k_tree");
struct JoinUnit {
    int b, h, last, row0, rows;  // sequence, KV head, its last CTA, first row in the (sequence, KV head), rows
};
template <int D, bool FP16>
__global__ void __launch_bounds__(32 * TJ_WARPS) k_tree_join(const __grid_constant__ PackedArgs a) {
    using L = TreeShape<D>;
    __shared__ TreeList T;
    __shared__ JoinUnit units[TREE_MAX_WORKERS];
    __shared__ int first[32 * TJ_WARPS + 1], warp_tasks[TJ_WARPS];  // tasks before a unit
    bool left_out = false;
    const int count = tree_list<D>(a, T, left_out);
    const Shares shares(a, count);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lr = lane >> 3, ld = lane & 7;
    const float c = a.scale * 1.4426950408889634f;
    // A thread a CTA of k_tree: the unit that it begins and others continue, if there is one, has the place where the next one's stretch begins.
    int tasks = 0;
    Segment seg{};
    if ((int)threadIdx.x + 1 < shares.workers && seg.find<D>(shares.first(threadIdx.x + 1), a, T)) {
        const int at = seg.at + Cost<D>::ROW, w0 = threadIdx.x, w1 = shares.owner(at + (seg.blocks - 1) * seg.cost), h = seg.unit / seg.chunks;
        const int row0 = (seg.unit - h * seg.chunks) * L::ROWS_ALL, n = min(T.nodes[seg.b] * a.group - row0, L::ROWS_ALL);
        if (shares.owner(at) == w0 && w1 > w0) tasks = (n + TJ_ROWS - 1) / TJ_ROWS * (D / 32);
        units[w0] = {seg.b, h, w1, row0, n};
    }
    int sum = tasks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 31) warp_tasks[warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += warp_tasks[w];
    first[threadIdx.x + 1] = sum;
    if (threadIdx.x == 0) first[0] = 0;
    __syncthreads();
    pdl_wait();
    if (blockIdx.x == 0) {
        const int c5 = __syncthreads_or(left_out);
        int code = DEV_OK;
        for (int w = threadIdx.x; w < a.workers; w += 32 * TJ_WARPS) code = max(code, a.worker_code[w]);
        const int c7 = __syncthreads_or(code == DEV_BAD_PAGE), c9 = __syncthreads_or(code == DEV_BAD_TREE);
        if (threadIdx.x == 0 && (c5 | c7 | c9)) latch_error(a.status, c5 ? DEV_BAD_POSITION : c7 ? DEV_BAD_PAGE : DEV_BAD_TREE);
    }
    for (int x = blockIdx.x * TJ_WARPS + warp; x < first[32 * TJ_WARPS]; x += gridDim.x * TJ_WARPS) {
        int w0 = 0, hi = 32 * TJ_WARPS;  // first[w0] <= x < first[hi]
        while (hi - w0 > 1) {
            const int mid = (w0 + hi) >> 1;
            if (first[mid] <= x)
                w0 = mid;
            else
                hi = mid;
        }
        const JoinUnit u = units[w0];
        const int b = u.b, h = u.h, w1 = u.last, n = u.rows, y = x - first[w0];
        const int row0 = y / (D / 32) * TJ_ROWS, d4 = y % (D / 32) * 8 + ld, pr = min(row0 + lr, n - 1);
        auto part = [&](int w) { return (long long)w * 2 + (w == w0); };
        auto max_sum = [&](int w) { return w <= w1 ? a.part_ml[part(w) * a.part_rows + pr] : make_float2(-INFINITY, 0.f); };
        float m = -INFINITY;
#pragma unroll 4
        for (int w = w0 + ld; w <= w1; w += 8) m = fmaxf(m, max_sum(w).x);
#pragma unroll
        for (int o = 4; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 *po = reinterpret_cast<const float4 *>(a.part_o) + (long long)d4 * a.part_rows + pr;
        for (int w8 = w0; w8 <= w1; w8 += 8) {
            const float2 ml = max_sum(w8 + ld);
            const float f = ml.x == m ? 1.f : ex2((ml.x - m) * c);
            l += ml.y * f;  // (NaN where ml is: a part that nobody has adds 0)
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = w8 + k <= w1 ? po[part(w8 + k) * (D / 4) * a.part_rows] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float g = __shfl_sync(0xffffffffu, f, (lane & 24) + k);
                if (w8 + k <= w1) o.x += v[k].x * g, o.y += v[k].y * g, o.z += v[k].z * g, o.w += v[k].w * g;
            }
        }
#pragma unroll
        for (int e = 4; e; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
        if (row0 + lr < n) {
            const Row r{m, l};
            const float inv = row_factor(r);
            const int row = u.row0 + row0 + lr, node = row / a.group;
            const long long out_row = (long long)(a.starts[b] + node) * a.hq + h * a.group + row - node * a.group;
            *reinterpret_cast<uint2 *>(a.out + out_row * D + d4 * 4) = make_uint2(pack16<FP16>(o.x * inv, o.y * inv), pack16<FP16>(o.z * inv, o.w * inv));
            if (a.lse && d4 == 0) a.lse[out_row] = row_lse<FP16>(r, a.scale);
        }
    }
}

int rows_all(int d) { return (d == 256 ? 1 : 2) * ROWS; }

// Rows of a page that one tiled copy can bring: a power of two that divides its length, 8 (a swizzle's rows) to 32, and 0 where
// there is none or a tensor map cannot express the cache.  Its dimensions: 64 of a row, eight rows, the row's other 64s,
// the other eights, and page and head in one (a page's stride is one of whole heads in both of the usual orders).
int tree_box(const KvView &kv, CUtensorMap *kmap, CUtensorMap *vmap, int *page_step) {
    int box = 1;
    while (box < 32 && kv.page_size % (2 * box) == 0) box *= 2;
    auto some = [&](long long s, long long n) { return n > 1 ? s : std::max(s, (long long)kv.d); };  // (one place has any stride)
    const long long head = kv.hkv > 1 ? kv.stride_head : some(kv.stride_page, kv.n_pages), slot = some(kv.stride_slot, kv.page_size);
    const long long most = 1ll << 35;  // (tensor maps hold strides below 2^40 bytes)
    long long step = kv.n_pages > 1 ? kv.stride_page / head : kv.hkv;
    if (box < 8 || head >= most || slot >= most || (kv.n_pages > 1 && kv.stride_page % head) || step < 1 || step * kv.n_pages + kv.hkv > 0x7fffffffll) return 0;
    *page_step = (int)step;
    const uint64_t dims[5] = {64, 8, (uint64_t)kv.d / 64, (uint64_t)kv.page_size / 8, (uint64_t)(step * (kv.n_pages - 1) + kv.hkv)};
    const uint64_t st[4] = {(uint64_t)slot * 2, 128, (uint64_t)slot * 16, (uint64_t)head * 2};
    const uint32_t bx[5] = {64, 8, (uint32_t)std::min(kv.d, 128) / 64, (uint32_t)box / 8, 1};
    return encode_map_16(kmap, kv.k, 5, dims, st, bx) && encode_map_16(vmap, kv.v, 5, dims, st, bx) ? box : 0;
}

template <int D, bool FP16>
cudaError_t launch(PackedArgs &a, cudaStream_t st) {
    using L = TreeShape<D>;
    static_assert(L::SMEM + sizeof(TreeState<D>) + sizeof(TreeList) + 128 <= 227 * 1024, "shared memory");
    static std::atomic<uint64_t> set{0};
    const cudaError_t e = once_per_device(set, [] { return cudaFuncSetAttribute(k_tree<D, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM); });
    if (e != cudaSuccess) return e;
    a.workers = std::min(gemm_ctas(), TREE_MAX_WORKERS);
    if (a.workers < 1) return cudaErrorInvalidDevice;
    a.patience = tree_patience(tree_places(a.kv, a.T, a.hq), a.workers);
    CUtensorMap kmap{}, vmap{};
    int step = 0;
    const int box = tree_box(a.kv, &kmap, &vmap, &step);
    k_tree<D, FP16><<<a.workers, THREADS, L::SMEM, st>>>(kmap, vmap, a, box, step);
    const cudaError_t c = cudaGetLastError();
    if (c != cudaSuccess) return c;
    const int most = (std::min({TREE_NODES * a.group, L::ROWS_ALL, std::min(a.T, 1 << 16) * a.group}) + TJ_ROWS - 1) / TJ_ROWS * (D / 32);  // tasks of a unit
    return launch_pdl(k_tree_join<D, FP16>, std::min((a.workers * most + TJ_WARPS - 1) / TJ_WARPS, 4 * gemm_ctas()), 32 * TJ_WARPS, 0, st, a);
}

}  // namespace

double tree_places(const KvView &kv, int T, int hq) {
    // (no row is two sequences': T rows are those of T sequences at most, and of a sequence as many)
    const int most = rows_all(kv.d), rows = std::min(TREE_NODES, T) * (hq / kv.hkv);
    const double units = (double)std::min(kv.B, T) * kv.hkv * ((rows + most - 1) / most), blocks = (double)((kv.cap + KEYS - 1) / KEYS);
    const int cost = kv.d == 64 ? cost_of<64>(rows) : kv.d == 128 ? cost_of<128>(rows) : cost_of<256>(rows);
    const int row = kv.d == 64 ? Cost<64>::ROW : kv.d == 128 ? Cost<128>::ROW : Cost<256>::ROW;
    return units * (blocks * cost + row);
}

bool tree_plan(const KvView &kv, int T, int hq, TreePlan *p) {
    const int most = rows_all(kv.d), group = hq / kv.hkv;
    if (tree_places(kv, T, hq) >= 2147483647.0) return false;  // (counted in 32 bits)
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
