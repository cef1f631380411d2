// kv_evict.cu -- eviction from a caller's paged cache by accumulated attention weight (pbd_op_evict).
//
// Of the n slots of one (sequence, KV head) the `keep` = min(n, n_keep) with the largest weight stay; tokens at the first
// n_sink positions and the last n_recent always do.  Attention does not mind the order of slots, so nothing is
// shifted: kept slots at or behind `keep` move into the holes in front, the i-th into the i-th.  That moves the
// fewest bytes there are, and no move's source is another's target.
//
// One cluster works on one (sequence, KV head), each CTA on a stretch of its slots.  The keep-th largest key is found by radix
// selection, 8 bits a round, over 32-bit keys in shared memory; a round's histograms are exchanged through
// distributed shared memory.  Then warps count and place holes and kept slots with ballots, and the CTAs share the
// moves.
#include <algorithm>

#include "kv_ops.h"

namespace pbd {

namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_CLUSTER = 8;        // CTAs of a cluster at most
constexpr int EV_KEYS = 48 * 1024;   // keys of a CTA that fit shared memory

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// Order of the slots: kept tokens first (all ones), then by weight, NaN last (0).
__device__ __forceinline__ uint32_t order_key(float w, int pos, int n_sink, int recent_from) {
    if (pos < n_sink || pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);  // (-0 counts as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <bool IN_SMEM>
__global__ void __launch_bounds__(EV_THREADS) k_evict(const EvictArgs a, int C) {
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ uint32_t hist[2][256];
    __shared__ uint32_t total[256];
    __shared__ uint32_t pick[2];
    __shared__ uint32_t warp_cnt[EV_WARPS], cta_cnt[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x % C, row = blockIdx.x / C, b = row / a.kv.hkv, h = row - b * a.kv.hkv;
    const long long cap = a.kv.cap, raw = a.kv.lens[b];
    const int n = (int)max(0ll, min(raw, cap)), keep = min(n, a.n_keep);
    if (tid == 0 && rank == 0 && raw != n) latch_error(a.status, DEV_BAD_POSITION);
    const float *w = a.kv.weights + row * cap;
    const int *pos = a.kv.positions + row * cap;
    float *out_w = a.out_weights + row * cap;
    int *out_pos = a.out_positions + row * cap;
    const bool copy = out_w != w;
    if (n == keep) {
        if (copy)
            for (int i = rank * EV_THREADS + tid; i < n; i += C * EV_THREADS) {
                out_w[i] = w[i];
                out_pos[i] = pos[i];
            }
        return;
    }
    if (keep == 0) return;
    const long long rf = (long long)a.next_pos[b] - a.n_recent;
    const int recent_from = (int)max(-2147483647ll - 1, rf);
    // this CTA's slots, and a warp's part of them (whole groups of 32)
    const int per_warp = ((n + C - 1) / C + EV_THREADS - 1) / EV_THREADS * 32, per = per_warp * EV_WARPS;
    const int s0 = (int)min((long long)n, (long long)rank * per), s1 = (int)min((long long)n, (long long)s0 + per);
    auto key_at = [&](int slot) {
        return IN_SMEM ? keys[slot - s0] : order_key(w[slot], pos[slot], a.n_sink, recent_from);
    };
    if (IN_SMEM)
        for (int i = s0 + tid; i < s1; i += EV_THREADS) keys[i - s0] = order_key(w[i], pos[i], a.n_sink, recent_from);

    uint32_t prefix = 0;  // the digits found so far
    int want = keep;      // the want-th largest of the keys that begin with them
    for (int round = 0; round < 4; ++round) {
        const int shift = 24 - 8 * round;
        uint32_t *hs = hist[round & 1];
        for (int i = tid; i < 256; i += EV_THREADS) hs[i] = 0;
        __syncthreads();
        for (int i = s0 + tid; i < s1; i += EV_THREADS) {
            const uint32_t k = key_at(i);
            const bool in = round == 0 || (k >> (shift + 8)) == prefix;
            if (in) atomicAdd(&hs[(k >> shift) & 255], 1u);
        }
        cluster_sync();
        if (tid < 256) {
            uint32_t sum = 0;
            const uint32_t at = smem_u32(&hs[tid]);
            for (int c = 0; c < C; ++c) sum += ld_cluster_u32(map_cta(at, c));
            total[tid] = sum;
        }
        __syncthreads();
        if (warp == 0) {
            // lane's 8 digits, from the largest down
            uint32_t mine = 0, d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = total[255 - (lane * 8 + i)];
                mine += d[i];
            }
            uint32_t x = mine;
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            uint32_t before = x - mine;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < (uint32_t)want && before + d[i] >= (uint32_t)want) {
                    pick[0] = 255 - (lane * 8 + i);
                    pick[1] = before;
                }
                before += d[i];
            }
        }
        __syncthreads();
        prefix = prefix << 8 | pick[0];
        want -= (int)pick[1];
    }
    const uint32_t T = prefix;  // kept: larger keys, and of the equal ones the first `want`
    const int w0 = min(s1, s0 + warp * per_warp), w1 = min(s1, w0 + per_warp);

    // equal keys before this warp
    int eq = 0;
    for (int i = w0; i < w1; i += 32) {
        const int s = i + lane;
        eq += __popc(__ballot_sync(0xffffffffu, s < w1 && key_at(s) == T));
    }
    // the sum of `mine` over the warps before this one, in the cluster's order of slots
    auto before_me = [&](int mine, int which) {
        if (lane == 0) warp_cnt[warp] = mine;
        __syncthreads();
        int b4 = 0, all = 0;
        for (int i = 0; i < EV_WARPS; ++i) {
            if (i < warp) b4 += warp_cnt[i];
            all += warp_cnt[i];
        }
        if (tid == 0) cta_cnt[which] = all;
        cluster_sync();
        const uint32_t at = smem_u32(&cta_cnt[which]);
        for (int c = 0; c < rank; ++c) b4 += ld_cluster_u32(map_cta(at, c));
        return b4;
    };
    const int eq0 = before_me(eq, 0);
    auto walk = [&](auto &&f) {  // f(slot, kept) for the warp's slots, 32 at a time
        int e = eq0;
        for (int i = w0; i < w1; i += 32) {
            const int s = i + lane;
            const uint32_t k = s < w1 ? key_at(s) : 0u;
            const bool same = s < w1 && k == T;
            const uint32_t m = __ballot_sync(0xffffffffu, same);
            f(s, s < w1, s < w1 && (k > T || (same && e + __popc(m & ((1u << lane) - 1)) < want)));
            e += __popc(m);
        }
    };
    int holes = 0, tails = 0;
    walk([&](int s, bool real, bool kept) {
        holes += __popc(__ballot_sync(0xffffffffu, real && s < keep && !kept));
        tails += __popc(__ballot_sync(0xffffffffu, real && s >= keep && kept));
    });
    int hole = before_me(holes, 1), tail = before_me(tails, 2);
    int *to = a.moves + (long long)row * 2 * a.most, *of = to + a.most;
    walk([&](int s, bool real, bool kept) {
        const bool is_hole = real && s < keep && !kept, is_tail = real && s >= keep && kept;
        const uint32_t mh = __ballot_sync(0xffffffffu, is_hole), mt = __ballot_sync(0xffffffffu, is_tail);
        const uint32_t below = (1u << lane) - 1;
        if (is_hole) to[hole + __popc(mh & below)] = s;
        if (is_tail) of[tail + __popc(mt & below)] = s;
        hole += __popc(mh);
        tail += __popc(mt);
        if (copy && real && s < keep && kept) {
            out_w[s] = w[s];
            out_pos[s] = pos[s];
        }
    });
    uint32_t moves = 0;
    for (int c = 0; c < C; ++c) moves += ld_cluster_u32(map_cta(smem_u32(&cta_cnt[1]), c));
    cluster_sync();  // the lists are whole, and nobody's counts are read any more
    for (uint32_t i = rank * EV_THREADS + tid; i < moves; i += C * EV_THREADS) {
        const int d = to[i], s = of[i];
        out_w[d] = w[s];
        out_pos[d] = pos[s];
    }
    // rows of K and V in 16-byte pieces
    const int pieces = a.kv.d / 8, lg = 31 - __clz(pieces);
    const int *table = a.kv.table + (long long)b * a.kv.max_pages;
    uint16_t *kv[2] = {const_cast<uint16_t *>(a.kv.k), const_cast<uint16_t *>(a.kv.v)};
    auto place = [&](int slot) {
        const int p = table[slot / a.kv.page_size];
        if ((unsigned)p >= (unsigned)a.kv.n_pages) {
            latch_error(a.status, DEV_BAD_PAGE);
            return -1ll;
        }
        return (long long)p * a.kv.stride_page + h * a.kv.stride_head + (long long)(slot % a.kv.page_size) * a.kv.stride_slot;
    };
    const long long all = (long long)moves << (lg + 1);
    for (long long i = rank * EV_THREADS + tid; i < all; i += C * EV_THREADS) {
        const int mv = (int)(i >> (lg + 1)), which = (int)(i >> lg) & 1, piece = (int)i & (pieces - 1);
        const long long d = place(to[mv]), s = place(of[mv]);
        if (d >= 0 && s >= 0)
            *reinterpret_cast<int4 *>(kv[which] + d + piece * 8) = *reinterpret_cast<const int4 *>(kv[which] + s + piece * 8);
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs &a, cudaStream_t st) {
    cudaError_t e = cudaMemsetAsync(a.status, 0, sizeof(int), st);
    if (e != cudaSuccess) return e;
    const int rows = a.kv.B * a.kv.hkv;
    // CTAs of a cluster: enough for two CTAs an SM in all, each with at least 1024 slots; more where keys ask for it
    int C = 1;
    while (C < EV_CLUSTER && (long long)C * 1024 < a.kv.cap && (rows * C < 2 * gemm_ctas() || a.kv.cap > (long long)C * EV_KEYS)) C *= 2;
    const long long per = (((a.kv.cap + C - 1) / C) + EV_THREADS - 1) / EV_THREADS * EV_THREADS;
    const bool in_smem = per <= EV_KEYS;
    static thread_local int configured = -1;
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (configured != dev) {
        e = cudaFuncSetAttribute(k_evict<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_KEYS * 4);
        if (e != cudaSuccess) return e;
        configured = dev;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * C));
    cfg.blockDim = dim3(EV_THREADS);
    cfg.dynamicSmemBytes = in_smem ? (size_t)per * 4 : 0;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, in_smem ? k_evict<true> : k_evict<false>, a, C);
}

}  // namespace pbd
