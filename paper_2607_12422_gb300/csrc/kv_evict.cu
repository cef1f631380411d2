// kv_evict.cu -- eviction from a caller's paged cache by accumulated attention weight (pbd_op_evict).
//
// Of the n slots of one (sequence, KV head) the `keep` = min(n, n_keep) with the largest weight stay; tokens at the first
// n_sink positions and the last n_recent always do.  Attention does not mind the order of slots, so nothing is
// shifted: kept slots at or behind `keep` move into the holes in front, the i-th into the i-th.  That moves the
// fewest bytes there are, and no move's source is another's target.
//
// One cluster works on one (sequence, KV head), each CTA on a stretch of its slots.  The keep-th largest key is found by radix
// selection over 32-bit keys in shared memory, 11, 11 and 10 bits a round (11 put sign, exponent and two bits of the mantissa
// into the first: weights of few magnitudes still spread over many counters).  After a round every CTA adds its counters that are
// not zero, which are few, to totals in distributed shared memory: the first CTA's, which all then read, or each CTA's own in
// the last round, where a handful is left (with each CTA's own in all rounds 131072 slots take 33 us instead of 31).  Then warps count and place holes and kept slots with ballots.  The moves
// follow in the same kernel where a CTA does a row alone (the step of a bounded cache: few moves, and a launch saved); after
// clusters another kernel makes them, spread over the whole GPU.
#include <algorithm>

#include "kv_ops.h"

namespace pbd {

namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_CLUSTER = 8;        // CTAs of a cluster at most
constexpr int EV_KEYS = 48 * 1024;   // keys of a CTA that fit shared memory
constexpr int EV_BINS = 2048;
static_assert(KV_MAX_BATCH <= EV_BINS, "check_cache keeps a number a sequence in the counters' place");
constexpr int EV_BATCH = 8;          // moves of a warp at a time: with 32, 8 sequences of 4112 took 17.5 us instead of 15.8

__device__ __forceinline__ uint2 ld_cluster_u32x2(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ld_cluster_u32x4(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void red_cluster_add(uint32_t a, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

// Order of the slots: kept tokens first (all ones), then by weight, NaN last (0).
__device__ __forceinline__ uint32_t order_key(float w, int pos, int n_sink, int recent_from) {
    if (pos < n_sink || pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);  // (-0 counts as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Slots of sequence b; none where the length is outside its range.  Such lengths and pages are reported once for the call: the
// grid's last cluster looks at all of them that are in use, so that the status word has one writer and needs no clearing before.
__device__ __forceinline__ int slots_of(const EvictArgs &a, int b) {
    const int n = a.kv.lens[b];
    return n >= 0 && n <= a.kv.cap ? n : 0;
}
__device__ void check_cache(const EvictArgs &a, int *used) {
    bool length = false;
    for (int b = threadIdx.x; b < a.kv.B; b += EV_THREADS) length |= a.kv.lens[b] != slots_of(a, b);
    length = __syncthreads_or(length);
    const bool page = any_bad_page<EV_THREADS>(a.kv, used, [&](int b) {
        const int n = slots_of(a, b);
        return n > a.n_keep ? n : 0;
    });
    if (threadIdx.x == 0) *a.status = length ? DEV_BAD_POSITION : page ? DEV_BAD_PAGE : DEV_OK;
}

// The moves of a row that warp `w` of `warps` makes, EV_BATCH at a time: each lane finds the places of one, then all copy, in 16-byte
// pieces, 32 / pieces rows of K and V at a time.
__device__ __forceinline__ void move_rows(const EvictArgs &a, int row, int w, int warps, int moves) {
    const int lane = threadIdx.x & 31, b = row / a.kv.hkv, h = row - b * a.kv.hkv;
    const float *weights = a.kv.weights + row * a.kv.cap;
    const int *pos = a.kv.positions + row * a.kv.cap, *to = a.moves + (long long)row * 2 * a.most, *of = to + a.most;
    float *out_w = a.out_weights + row * a.kv.cap;
    int *out_pos = a.out_positions + row * a.kv.cap;
    const int pieces = a.kv.d / 8, lg = 31 - __clz(pieces);
    const int *table = a.kv.table + (long long)b * a.kv.max_pages;
    auto place = [&](int slot) {  // -1: no such page
        const int q = page_index(a.kv, slot), p = table[q];
        if ((unsigned)p >= (unsigned)a.kv.n_pages) return -1ll;
        return (long long)p * a.kv.stride_page + h * a.kv.stride_head + (long long)(slot - q * a.kv.page_size) * a.kv.stride_slot;
    };
    for (int m0 = w * EV_BATCH; m0 < moves; m0 += warps * EV_BATCH) {
        long long dst = -1, src = -1;
        const bool real = lane < EV_BATCH && m0 + lane < moves;
        const int d = real ? to[m0 + lane] : 0, s = real ? of[m0 + lane] : 0;
        if (real) {
            dst = place(d);
            src = place(s);
            if (dst < 0 || src < 0) dst = src = -1;
        }
        const int units = min(EV_BATCH, moves - m0) << (lg + 1);  // pieces of this batch: move, K or V, piece
        constexpr int U = 4;
        for (int u0 = 0; u0 < units; u0 += 32 * U) {
            uint4 x[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int u = u0 + j * 32 + lane;
                const long long from = __shfl_sync(0xffffffffu, src, (u >> (lg + 1)) & 31);
                if (u < units && from >= 0) x[j] = *reinterpret_cast<const uint4 *>((u >> lg & 1 ? a.kv.v : a.kv.k) + from + (u & (pieces - 1)) * 8);
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int u = u0 + j * 32 + lane;
                const long long at = __shfl_sync(0xffffffffu, dst, (u >> (lg + 1)) & 31);
                if (u < units && at >= 0)
                    *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(u >> lg & 1 ? a.kv.v : a.kv.k) + at + (u & (pieces - 1)) * 8) = x[j];
            }
        }
        if (dst >= 0) {  // (a move that a bad page leaves out keeps its weight and position as well)
            out_w[d] = weights[s];
            out_pos[d] = pos[s];
        }
    }
}

template <bool IN_SMEM, bool ALONE>  // ALONE: clusters of one CTA
__global__ void __launch_bounds__(EV_THREADS, 2) k_evict(const EvictArgs a, int cluster) {
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ __align__(16) uint32_t hist[EV_BINS];                 // this CTA's counters of a round
    __shared__ __align__(16) uint32_t totals[ALONE ? 1 : 3][EV_BINS];  // the cluster's, of each round
    __shared__ uint32_t pick[3], warp_cnt[2][EV_WARPS];
    __shared__ __align__(8) uint2 cta_cnt[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = ALONE ? 1 : cluster;
    const int rank = ALONE ? 0 : blockIdx.x % C, row = ALONE ? blockIdx.x : blockIdx.x / C;
    if (!ALONE) pdl_launch();
    if (row == a.kv.B * a.kv.hkv) {
        if (rank == 0) check_cache(a, reinterpret_cast<int *>(hist));
        return;
    }
    auto sync = [&]() {
        if (ALONE)
            __syncthreads();
        else
            cluster_sync();
    };
    const int b = row / a.kv.hkv, n = slots_of(a, b), keep = min(n, a.n_keep);
    if (!ALONE && rank == 0 && tid == 0) a.counts[row] = 0;  // (if there is nothing to move)
    if (keep == 0) return;
    const long long cap = a.kv.cap;
    const float *w = a.kv.weights + row * cap;
    const int *pos = a.kv.positions + row * cap;
    float *out_w = a.out_weights + row * cap;
    int *out_pos = a.out_positions + row * cap;
    const int copied = out_w != w ? keep : 0;  // slots in front are copied as they are, and holes then filled
    const int recent_from = (int)max(-2147483647ll - 1, (long long)a.next_pos[b] - a.n_recent);
    // this CTA's slots, and a warp's part of them (whole groups of 32)
    const int per_warp = ((n + C - 1) / C + EV_THREADS - 1) / EV_THREADS * 32, per = per_warp * EV_WARPS;
    const int s0 = (int)min((long long)n, (long long)rank * per), s1 = (int)min((long long)n, (long long)s0 + per);
    const uint4 zeros = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4 *>(hist + tid * 4) = zeros;
    if (!ALONE)
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint4 *>(totals[i] + tid * 4) = zeros;
    if (!ALONE) cluster_arrive();  // (this CTA runs, and its totals are zero)
    constexpr int AHEAD = 8;
    for (int i0 = s0 + tid; i0 < s1; i0 += EV_THREADS * AHEAD) {
        float x[AHEAD];
        int p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = i0 + j * EV_THREADS;
            if (i < s1) {
                x[j] = w[i];
                p[j] = pos[i];
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = i0 + j * EV_THREADS;
            if (i >= s1) continue;
            if (IN_SMEM) keys[i - s0] = order_key(x[j], p[j], a.n_sink, recent_from);
            if (i < copied) {
                out_w[i] = x[j];
                out_pos[i] = p[j];
            }
        }
    }
    if (n == keep) return;
    auto key_at = [&](int slot) {
        return IN_SMEM ? keys[slot - s0] : order_key(w[slot], pos[slot], a.n_sink, recent_from);
    };

    if (ALONE)
        __syncthreads();
    else
        cluster_wait();  // (all of the cluster's CTAs)
    uint32_t prefix = 0;  // the digits found so far
    int want = keep;      // the want-th largest of the keys that begin with them
    bool all_equal_kept = false;
#pragma unroll
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, above = round == 1 ? 21 : 10;
        const uint32_t mask = round == 2 ? 1023u : 2047u;
        for (int i = s0 + tid; i < s1; i += EV_THREADS) {
            const uint32_t k = key_at(i);
            if (round == 0 || (k >> above) == prefix) atomicAdd(&hist[(k >> shift) & mask], 1u);
        }
        __syncthreads();
        // this thread's four digits, from the largest down
        const int at = EV_BINS - 4 - tid * 4;
        uint4 d = *reinterpret_cast<const uint4 *>(hist + at);
        *reinterpret_cast<uint4 *>(hist + at) = zeros;
        if (!ALONE) {
            const uint32_t own[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (own[i])
                    for (int c = 0; c < (round == 2 ? C : 1); ++c) red_cluster_add(map_cta(smem_u32(&totals[round][at + i]), c), own[i]);
            sync();
            d = round == 2 ? *reinterpret_cast<const uint4 *>(totals[round] + at) : ld_cluster_u32x4(map_cta(smem_u32(&totals[round][at]), 0));
        }
        const uint32_t mine = d.x + d.y + d.z + d.w;
        uint32_t x = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_cnt[0][warp] = x;
        __syncthreads();
        uint32_t before = x - mine;
        for (int i = 0; i < warp; ++i) before += warp_cnt[0][i];
        const uint32_t ds[4] = {d.w, d.z, d.y, d.x};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (before < (uint32_t)want && before + ds[i] >= (uint32_t)want) {
                pick[0] = at + 3 - i;
                pick[1] = before;
                pick[2] = ds[i];
            }
            before += ds[i];
        }
        __syncthreads();
        prefix = prefix << (round == 2 ? 10 : 11) | pick[0];
        want -= (int)pick[1];
        all_equal_kept = (int)pick[2] == want;
    }
    const uint32_t T = prefix;  // kept: larger keys, and of the equal ones the first `want`
    const int w0 = min(s1, s0 + warp * per_warp), w1 = min(s1, w0 + per_warp);

    // two sums over the warps before this one, in the cluster's order of slots, and over all
    auto before_me = [&](uint2 mine, int which, uint2 *sum) {
        if (lane == 0) warp_cnt[0][warp] = mine.x, warp_cnt[1][warp] = mine.y;
        __syncthreads();
        uint2 b4 = make_uint2(0, 0), all = b4;
        for (int i = 0; i < EV_WARPS; ++i) {
            const uint32_t x = warp_cnt[0][i], y = warp_cnt[1][i];
            if (i < warp) b4.x += x, b4.y += y;
            all.x += x, all.y += y;
        }
        if (!ALONE) {
            if (tid == 0) cta_cnt[which] = all;
            sync();
            const uint32_t at = smem_u32(&cta_cnt[which]);
            all = make_uint2(0, 0);
            for (int c = 0; c < C; ++c) {
                const uint2 x = ld_cluster_u32x2(map_cta(at, c));
                if (c < rank) b4.x += x.x, b4.y += x.y;
                all.x += x.x, all.y += x.y;
            }
        }
        *sum = all;
        return b4;
    };
    uint2 all;
    int eq0 = 0;
    if (!all_equal_kept) {
        int eq = 0;
        for (int i = w0; i < w1; i += 32) {
            const int s = i + lane;
            eq += __popc(__ballot_sync(0xffffffffu, s < w1 && key_at(s) == T));
        }
        eq0 = before_me(make_uint2(eq, 0), 0, &all).x;
        __syncthreads();  // (warp_cnt has been read)
    }
    auto walk = [&](auto &&f) {  // f(slot, whether it is one, kept) for the warp's slots, 32 at a time
        int e = eq0;
        for (int i = w0; i < w1; i += 32) {
            const int s = i + lane;
            const uint32_t k = s < w1 ? key_at(s) : 0u;
            bool kept = k >= T;
            if (!all_equal_kept) {
                const uint32_t m = __ballot_sync(0xffffffffu, s < w1 && k == T);
                kept = k > T || (k == T && e + __popc(m & ((1u << lane) - 1)) < want);
                e += __popc(m);
            }
            f(s, s < w1, s < w1 && kept);
        }
    };
    int holes = 0, tails = 0;
    walk([&](int s, bool real, bool kept) {
        holes += __popc(__ballot_sync(0xffffffffu, real && s < keep && !kept));
        tails += __popc(__ballot_sync(0xffffffffu, real && s >= keep && kept));
    });
    const uint2 b4 = before_me(make_uint2(holes, tails), 1, &all);
    int hole = b4.x, tail = b4.y;
    int *to = a.moves + (long long)row * 2 * a.most, *of = to + a.most;
    walk([&](int s, bool real, bool kept) {
        const bool is_hole = real && s < keep && !kept, is_tail = real && s >= keep && kept;
        const uint32_t mh = __ballot_sync(0xffffffffu, is_hole), mt = __ballot_sync(0xffffffffu, is_tail);
        const uint32_t below = (1u << lane) - 1;
        if (is_hole) to[hole + __popc(mh & below)] = s;
        if (is_tail) of[tail + __popc(mt & below)] = s;
        hole += __popc(mh);
        tail += __popc(mt);
    });
    sync();  // the lists are whole, and nobody's counts are read any more

    if (ALONE) {
        move_rows(a, row, warp, EV_WARPS, all.x);
    } else if (rank == 0 && tid == 0) {
        a.counts[row] = all.x;  // (k_evict_moves)
    }
}

constexpr int EM_THREADS = 256;

// The moves of all rows, in small batches, so that every SM has its share however the rows differ.
__global__ void __launch_bounds__(EM_THREADS, 4) k_evict_moves(const EvictArgs a) {
    pdl_wait();
    const int row = blockIdx.x, warp = blockIdx.y * (EM_THREADS / 32) + (threadIdx.x >> 5);
    move_rows(a, row, warp, gridDim.y * (EM_THREADS / 32), a.counts[row]);
}

template <bool IN_SMEM, bool ALONE>
cudaError_t launch(const EvictArgs &a, int C, size_t smem, cudaStream_t st) {
    static thread_local int configured = -1;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && configured != dev) {
        e = cudaFuncSetAttribute(k_evict<IN_SMEM, ALONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_KEYS * 4);
        if (e == cudaSuccess) configured = dev;
    }
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.kv.B * a.kv.hkv + 1) * C));  // (one cluster more: check_cache)
    cfg.blockDim = dim3(EV_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, k_evict<IN_SMEM, ALONE>, a, C);
    if (e != cudaSuccess || ALONE || a.most == 0) return e;
    // a batch a warp; fewer warps where rows are many
    const int rows = a.kv.B * a.kv.hkv;
    const long long blocks = (a.most + EM_THREADS / 32 * EV_BATCH - 1) / (EM_THREADS / 32 * EV_BATCH), most = std::max(1, gemm_ctas() * 32 / rows);
    cfg.gridDim = dim3((unsigned)rows, (unsigned)std::min(blocks, most));
    cfg.blockDim = dim3(EM_THREADS);
    cfg.dynamicSmemBytes = 0;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    return cudaLaunchKernelEx(&cfg, k_evict_moves, a);
}

}  // namespace

cudaError_t launch_evict(const EvictArgs &a, cudaStream_t st) {
    const int rows = a.kv.B * a.kv.hkv;
    // CTAs of a cluster: as many as run at once, two an SM, each with more than 1024 slots; more where keys ask for it.
    // (8 KV heads, us with C = 1, 2, 4, 8: 1 x 4096 slots 31, 13.2, 13.5, 14.9; 16 x 4096 48, 42, 53, 84; 64 x 4096 129, 162, 198,
    // 317: a second wave of clusters costs more than longer rows do. 8 x 1025 6.7, 10.8, 13.4, 29.)
    int C = 1;
    while (C < EV_CLUSTER && (long long)C * 2048 < a.kv.cap && (rows * C * 2 <= 2 * gemm_ctas() || a.kv.cap > (long long)C * EV_KEYS)) C *= 2;
    const long long per = (((a.kv.cap + C - 1) / C) + EV_THREADS - 1) / EV_THREADS * EV_THREADS;
    if (per > EV_KEYS) return launch<false, false>(a, C, 0, st);  // (C is EV_CLUSTER)
    return C == 1 ? launch<true, true>(a, C, (size_t)per * 4, st) : launch<true, false>(a, C, (size_t)per * 4, st);
}

}  // namespace pbd
