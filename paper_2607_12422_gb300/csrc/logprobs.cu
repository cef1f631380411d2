// logprobs.cu -- log probabilities of given tokens, entropy and top alternatives from logits (pbd_op_token_logprobs).
//
// Of a row x of V logits at temperature T, with m = max x, S = sum exp((x - m) / T):
//     logprob(t) = (x_t - m) / T - ln S
//     entropy    = ln S + sum (m - x) / T exp((x - m) / T) / S      (both terms >= 0: nothing cancels)
//     top k      by value, then by the lower index
// in one pass over the logits, which bounds it: running maximum and sums in fp32 per thread, joined at the end.  A CTA
// streams tiles of its rows through a ring in shared memory, filled by bulk copies that run ahead into the next row while
// it finishes one.  A thread's part of a tile, a group, is 32 values that lie together: 32-KB tiles of fp32, two in the ring, and 16-KB
// tiles of 16-bit values, three.  (16-KB tiles of fp32, groups of 16, 2048 x 151936, k = 8: 191 us instead of 185; 32-KB tiles of 16-bit
// values, groups of 64: 125 instead of 132 there, but 346 instead of 278 for 20000 x 8000, where a tile holds two rows and more, and
// 22.9 instead of 21.7 for 136 x 151936, k = 32.)  Few rows are cut into
// slices: a cluster of CTAs a row, whose parts are joined through distributed shared memory.
//
// The alternatives come from the same pass.  The k best values lie in the k groups with the largest maxima (k values, those
// maxima, already reach the k-th of them), so at the end k groups are picked and read again.  Each thread keeps the three
// largest of its groups' maxima, and nothing else is stored: should a fourth matter, its warp reads the thread's groups again,
// which an order at random asks of one CTA in five for k = 32 and of one in 500 for k = 8.  (2048 x 151936 bf16, k = 8: 128 us with 2
// kept, 132 with 3, 138 with 4, 145 with 5; 136 rows, k = 32: 23.7 with 2, 21.7 with 3 and 21.6 with 4.)  Groups are contiguous, so
// that among equal maxima the lower group holds the lower ids.
//
// The loop over the halves of fp32 tiles stays a loop: unrolled, for twice the code, it takes as long (2048 x 151936 183 us, 8192 x 32000
// without alternatives 147).
#include <algorithm>
#include <cuda_fp16.h>

#include "../../include/pbd_ops.h"
#include "kv_ops.h"

namespace pbd {

namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_GROUP = 32;                      // values of a group: what a thread has of a tile
constexpr int LP_STEP = 4;                        // 16-byte vectors of it at a time
constexpr int LP_CTAS = 3;                        // of an SM
constexpr int LP_TOP = 3;                         // groups that a thread keeps
constexpr int LP_CLUSTER = 16;                    // slices of a row at most
constexpr int LP_BINS = LP_THREADS / 4;           // of the selections below
constexpr int LP_LIST = 512;                      // keys of a list: ten times what an order at random needs (bin_bound)
constexpr float LP_FLOOR = -1000.f;               // 2^-1000 is 0 in fp32

typedef unsigned long long u64;

__device__ __forceinline__ float lp_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// max that hands NaN on
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Order of values as a number: NaN (1) below everything, 0 is nobody's.
__device__ __forceinline__ uint32_t lp_order(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);  // (-0 counts as 0)
    return x != x ? 1u : (u & 0x80000000u ? ~u : u | 0x80000000u);
}
// (value, lower index first) as one number
__device__ __forceinline__ u64 lp_key(uint32_t order, int i) { return (u64)order << 32 | (uint32_t)~i; }
__device__ __forceinline__ float key_value(u64 k) {
    const uint32_t v = (uint32_t)(k >> 32);
    return v <= 1 ? __uint_as_float(0x7fffffffu) : __uint_as_float(v & 0x80000000u ? v & 0x7fffffffu : ~v);
}
__device__ __forceinline__ int key_index(u64 k) { return (int)~(uint32_t)k; }

template <int TYPE>
struct Elem;  // values of a 16-byte vector, and what stands for a masked one in it
template <>
struct Elem<PBD_FP32> {
    static constexpr int N = 4, SIZE = 4, STAGES = 2;
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    // the largest value (NaN only where there is nothing else)
    static __device__ __forceinline__ float largest(const uint4 &v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return static_cast<const float *>(p)[i]; }
    static __device__ __forceinline__ void put(uint32_t *u, int i, const void *p, long long at, bool real) {
        u[i] = real ? static_cast<const uint32_t *>(p)[at] : 0xff800000u;
    }
    static __device__ __forceinline__ float round(float x) { return x; }
    static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ void set(uint32_t *u, int i, uint32_t b) { u[i] = b; }
};
template <uint32_t LOWEST>
struct Elem16 {
    static constexpr int N = 8, SIZE = 2, STAGES = 3;
    static __device__ __forceinline__ void put(uint32_t *u, int i, const void *p, long long at, bool real) {
        const uint32_t x = real ? static_cast<const uint16_t *>(p)[at] : LOWEST;
        u[i / 2] = i & 1 ? u[i / 2] | x << 16 : x;
    }
    static __device__ __forceinline__ void set(uint32_t *u, int i, uint32_t b) {
        u[i / 2] = i & 1 ? (u[i / 2] & 0xffffu) | b << 16 : (u[i / 2] & 0xffff0000u) | b;
    }
};
template <>
struct Elem<PBD_BF16> : Elem16<0xff80u> {
    static __device__ __forceinline__ float round(float x) { return rbf(x); }
    static __device__ __forceinline__ uint32_t bits(float x) { return __bfloat16_as_ushort(f2bf(x)); }
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float largest(const uint4 &v) {  // (two values an operation)
        const auto *b = reinterpret_cast<const __nv_bfloat162 *>(&v);
        const float2 f = __bfloat1622float2(__hmax2(__hmax2(b[0], b[1]), __hmax2(b[2], b[3])));
        return fmaxf(f.x, f.y);
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return bf2f(static_cast<const bf16 *>(p)[i]); }
};
template <>
struct Elem<PBD_FP16> : Elem16<0xfc00u> {
    static __device__ __forceinline__ float round(float x) { return __half2float(__float2half_rn(x)); }
    static __device__ __forceinline__ uint32_t bits(float x) { return __half_as_ushort(__float2half_rn(x)); }
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float largest(const uint4 &v) {
        const auto *b = reinterpret_cast<const __half2 *>(&v);
        const float2 f = __half22float2(__hmax2(__hmax2(b[0], b[1]), __hmax2(b[2], b[3])));
        return fmaxf(f.x, f.y);
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return __half2float(static_cast<const __half *>(p)[i]); }
};

// Maximum m, sum of e = exp((x - m) / T) without one value that is m (if m is not -inf), sum of e * log2(e).  The 1 that is
// left out stays apart to the end: a sum of 1 and what is small beside it would lose the small part, which is all that the
// log probability of an almost certain token and the entropy then consist of.
struct Stat {
    float m, s, h;
};
// `low`, whose maximum is not above m, at the maximum m, with the value that was left out if it is its own to add: e 2^d has the
// logarithm log2 e + d
__device__ __forceinline__ void lower(Stat &low, float m, float c, bool own) {
    const float d = max_nan((low.m - (m == -INFINITY ? 0.f : m)) * c, LP_FLOOR), f = lp_ex2(d);
    const float all = own && low.m > -INFINITY ? low.s + 1.f : low.s;
    low.h = (low.h + all * d) * f;
    low.s = all * f;
}
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
    const bool first = a.m >= b.m;
    Stat &low = first ? b : a;
    const float m = first ? a.m : b.m;
    lower(low, m, c, true);
    return Stat{m, a.s + b.s, a.h + b.h};
}

// What the selections share (one CTA).
struct Shared {
    u64 list[LP_LIST], best[LP_MAX_K], bins[LP_BINS], bar;
    int count;
};

// The number of the n keys in shared memory that are larger than x, by four lanes (lane % 4 = part).
__device__ __forceinline__ int rank_of(u64 x, const u64 *keys, int n, int part) {
    int r = 0;
#pragma unroll 4
    for (int j = part; j < n; j += 4) r += keys[j] > x;
    r += __shfl_xor_sync(0xffffffffu, r, 1);
    return r + __shfl_xor_sync(0xffffffffu, r, 2);
}

// A lower bound of the k-th largest of all keys, from each thread's largest (0: none): the k-th largest of the maxima of 64
// bins of four threads, which k keys reach; 0 if fewer bins have one.  Of keys in any order some 64 ln(64 / (64 - k))
// reach it: 44 for k = 32.  Whole CTA.
__device__ __forceinline__ u64 bin_bound(u64 mine, int k, Shared &s) {
    // (lanes 4 and 8 apart: where only lanes with bit 2 clear have keys, every bin still has two of them)
    mine = max(mine, (u64)__shfl_xor_sync(0xffffffffu, mine, 4));
    mine = max(mine, (u64)__shfl_xor_sync(0xffffffffu, mine, 8));
    const int lane = threadIdx.x & 31;
    if ((lane & 12) == 0) s.bins[(threadIdx.x >> 5) * 8 + (lane & 3) + (lane >> 4) * 4] = mine;
    if (threadIdx.x == 0) s.bar = 0, s.count = 0;
    __syncthreads();
    const u64 x = s.bins[threadIdx.x >> 2];
    if (rank_of(x, s.bins, LP_BINS, threadIdx.x & 3) == k - 1 && x) s.bar = x;
    __syncthreads();
    return s.bar;
}

// The k largest of the CTA's keys, which differ, sorted, into s.best, zeros behind them.  mine: the thread's largest (0: none);
// each(f), by whole warps: f(key) for all of their keys that may matter, the same ones at every call; at_least: what k of the keys are known to
// reach (0: nothing is known).  Whole CTA.
template <typename Each>
__device__ __forceinline__ void select_best(u64 mine, int k, Shared &s, u64 at_least, Each &&each) {
    u64 bar = at_least;
#pragma unroll 1
    for (int way = at_least ? 0 : 1;; ++way) {
        if (way == 0) {
            if (threadIdx.x == 0) s.count = 0;
            __syncthreads();
        } else if (way == 1) {
            bar = bin_bound(mine, k, s);
        } else {
            // few bins hold nearly all of the largest: the k-th key bit by bit
            bar = 0;
#pragma unroll 1
            for (int bit = 63; bit >= 0; --bit) {
                const u64 tried = bar | 1ull << bit;
                __syncthreads();
                if (threadIdx.x == 0) s.count = 0;
                __syncthreads();
                int c = 0;
                if (__any_sync(0xffffffffu, mine >= tried)) each([&](u64 x) { c += x >= tried; });
                if (c) atomicAdd(&s.count, c);
                __syncthreads();
                if (s.count >= k) bar = tried;
            }
            __syncthreads();
            if (threadIdx.x == 0) s.count = 0;
            __syncthreads();
        }
        if (__any_sync(0xffffffffu, mine && mine >= bar))
            each([&](u64 x) {
                if (x && x >= bar) {
                    const int p = atomicAdd(&s.count, 1);
                    if (p < LP_LIST) s.list[p] = x;
                }
            });
        if (threadIdx.x < k) s.best[threadIdx.x] = 0;
        __syncthreads();
        if (s.count <= LP_LIST) break;
        __syncthreads();
    }
    const int have = s.count;
    for (int i0 = 0; i0 < have; i0 += LP_THREADS / 4) {
        const int i = i0 + (threadIdx.x >> 2);
        const u64 x = i < have ? s.list[i] : 0;
        const int r = rank_of(x, s.list, have, threadIdx.x & 3);
        if (i < have && r < k) s.best[r] = x;
    }
    __syncthreads();
}

struct Finish {  // a row's results
    const LogprobArgs &a;
    __device__ __forceinline__ void operator()(int row, const Stat &s, const u64 *best, float x_t, bool has_token, int token) const {
        const float none = __uint_as_float(0x7fffffffu), t = a.inv_t, mu = s.m == -INFINITY ? 0.f : s.m;
        const float ls = s.m == INFINITY ? none : log1pf(s.s);  // ln of the sum
        const bool empty = s.m == -INFINITY && s.s == 0.f;  // nothing but -inf
        if (threadIdx.x == 0) {
            if (a.logprob) {
                float lp = token < 0 ? 0.f : none;
                if (has_token) lp = empty ? -INFINITY : (x_t - mu) * t - ls;
                a.logprob[row] = lp;
            }
            if (a.entropy) a.entropy[row] = empty ? 0.f : ls - 0.6931471805599453f * (s.h / (1.f + s.s));
        }
        for (int i = threadIdx.x; i < a.k; i += LP_THREADS) {  // (k is at most 32: all by the first warp)
            a.top_ids[(long long)row * a.k + i] = key_index(best[i]);
            a.top_lp[(long long)row * a.k + i] = empty ? -INFINITY : (key_value(best[i]) - mu) * t - ls;
        }
    }
};

// Every row's token, by one CTA.
__device__ __forceinline__ void check_tokens(const LogprobArgs &a) {
    bool bad = false;
    if (a.tokens)
        for (int i = threadIdx.x; i < a.M; i += LP_THREADS) bad |= a.tokens[i] >= a.V;
    if (bad) latch_error(a.status, DEV_BAD_TOKEN);
}

// A row as its CTAs see it: vectors are counted from the 16-byte boundary at or before its first value.
template <int TYPE>
struct Row {
    const char *base, *vbase;  // first value, first vector
    int skew;                  // values of the first vector that are not the row's
    int v0, v1;                // vectors of this slice
    int whole0, whole1;        // vectors that hold nothing but values of the row
    __device__ __forceinline__ Row(const LogprobArgs &a, int row, int slice) {
        using E = Elem<TYPE>;
        base = static_cast<const char *>(a.x) + row * a.ld * E::SIZE;
        skew = (int)(reinterpret_cast<uintptr_t>(base) & 15) / E::SIZE;
        vbase = base - skew * E::SIZE;
        const int vecs = (a.V + skew + E::N - 1) / E::N;
        v0 = min(vecs, slice * a.slice_vecs);
        v1 = min(vecs, v0 + a.slice_vecs);
        whole0 = skew ? 1 : 0;
        whole1 = (a.V + skew) / E::N;
    }
};

template <int TYPE, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, LP_CTAS) k_logprobs(const LogprobArgs a) {
    using E = Elem<TYPE>;
    constexpr int VECS = LP_GROUP / E::N, TILE = LP_THREADS * VECS, STAGES = E::STAGES;  // vectors of a group, of a tile
    extern __shared__ __align__(128) uint8_t dyn[];
    uint4 *ring = reinterpret_cast<uint4 *>(dyn);
    __shared__ Shared sh;
    __shared__ Stat ws[LP_WARPS], slice_stat[LP_CLUSTER];                       // of warps; of slices (the first CTA's)
    __shared__ __align__(8) u64 slice_best[TOP ? LP_CLUSTER : 1][LP_MAX_K];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES];
    __shared__ int abort, sent[STAGES];  // (sent: tiles sent for into each stage)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int slice = blockIdx.x % a.slices, first_row = blockIdx.x / a.slices, rows_apart = gridDim.x / a.slices;
    if (tid == 0) {
        abort = 0;
        if (blockIdx.x == 0) *a.status = DEV_OK;  // (before anything is latched: waits that give up take a second, and tokens come last)
        for (int i = 0; i < STAGES; ++i) {
            sent[i] = 0;
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], LP_WARPS);
        }
        fence_mbarrier_init();
    }
    __syncthreads();
    const float c = a.inv_t * 1.4426950408889634f, far = 150.f / c;

    // The next tile to be sent for, in all threads: of row `p_row`, vectors [p_v, p_v1) of which are left.  Warps take turns in
    // sending: it holds a thread up for 600 cycles, and one warp that always did so would hold up all (a third of the time
    // of 16-bit rows).
    int p_row = first_row, p_v = 0, p_v1 = 0, sender = 0;
    const uint64_t policy = l2_policy_evict_first();
    auto enter_row = [&]() {  // the first row from p_row on that has a tile
        for (; p_row < a.M; p_row += rows_apart) {
            const Row<TYPE> r(a, p_row, slice);
            p_v = r.v0;
            p_v1 = r.v1;
            if (p_v < p_v1) return;
        }
    };
    auto send = [&](int st) {  // (one thread; the stage is free)
        const Row<TYPE> r(a, p_row, slice);
        const int b = max(p_v, r.whole0), e = max(b, min(min(p_v + TILE, r.v1), r.whole1));
        ++sent[st];
        mbar_arrive_expect_tx(&full[st], (e - b) * 16);
        if (e > b) bulk_g2s(ring + st * TILE + (b - p_v), r.vbase + (long long)b * 16, (e - b) * 16, &full[st], policy);
    };
    auto advance = [&]() {
        p_v += TILE;
        if (p_v >= p_v1) {
            p_row += rows_apart;
            enter_row();
        }
        sender = sender + 1 == LP_WARPS ? 0 : sender + 1;
    };
    enter_row();
#pragma unroll
    for (int i = 0; i < STAGES; ++i)
        if (p_row < a.M) {
            if (tid == i * 32) send(i);  // (each holds a warp up)
            advance();
        }
    if (a.slices > 1) cluster_arrive();

    // the i-th vector of a tile and half that this thread reads: its VECS lie together, in turns, so that eight threads read from all banks
    auto vec_of = [&](int half, int i) { return tid * VECS + ((half * LP_STEP + i + tid * VECS / 8) & (VECS - 1)); };
    int stage = 0, turn = 0;
    for (int row = first_row; row < a.M; row += rows_apart) {
        const Row<TYPE> r(a, row, slice);
        Stat st{-INFINITY, 0.f, 0.f};
        const int token = tid == 0 && slice == 0 && a.logprob ? a.tokens[row] : -1;
        // the thread's groups, one a tile: the largest maxima, the largest first, and their tiles (-1: none)
        const int group0 = r.v0 / VECS + tid;  // the first one's number
        float top[LP_TOP];
        int top_tile[LP_TOP], tile = 0;
#pragma unroll
        for (int i = 0; i < LP_TOP; ++i) top[i] = __uint_as_float(0x7fffffffu), top_tile[i] = -1;
        const bool given_up = __any_sync(0xffffffffu, *(volatile int *)&abort);  // (further rows have no tiles then)
        for (int v = given_up ? r.v1 : r.v0; v < r.v1; v += TILE, ++tile) {
            // (after a wait that ran out the row goes on with whatever the ring holds, and no thread waits for long again)
            mbar_wait(&full[stage], turn, a.status, DEV_TIMEOUT_LOAD, &abort);
            const int w0 = v + warp * (32 * VECS);  // the warp's first vector
            const bool edge = w0 < r.whole0 || w0 + 32 * VECS > min(r.v1, r.whole1);
            if (w0 < r.v1) {  // (else the warp has nothing of the row's last tile)
                float m_group = __uint_as_float(0x7fffffffu);
#pragma unroll 1
                for (int half = 0; half < VECS / LP_STEP; ++half) {
                    uint4 raw[LP_STEP];
#pragma unroll
                    for (int i = 0; i < LP_STEP; ++i) raw[i] = ring[stage * TILE + vec_of(half, i)];
                    if (half == VECS / LP_STEP - 1) {
                        __syncwarp();
                        if (lane == 0) mbarrier_arrive_one(&empty[stage]);
                    }
                    if (edge) {
                        // value by value at a row's ends; -inf behind the slice
#pragma unroll
                        for (int i = 0; i < LP_STEP; ++i) {
                            const int at = v + vec_of(half, i);
                            if (at < r.v1 && at >= r.whole0 && at < r.whole1) continue;
                            uint32_t u[4];
#pragma unroll
                            for (int j = 0; j < E::N; ++j) {
                                const int e = at * E::N - r.skew + j;
                                E::put(u, j, r.base, e, at < r.v1 && e >= 0 && e < a.V);
                            }
                            raw[i] = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                    }
                    float mx[LP_STEP];
#pragma unroll
                    for (int i = 0; i < LP_STEP; ++i) mx[i] = E::largest(raw[i]);
                    const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    m_group = fmaxf(m_group, mt);
                    if (__any_sync(0xffffffffu, mt > st.m)) {
                        // the warp has a new maximum, and a lane leaves one value of it out of its sum
                        int owner;
                        const float mw = warp_max(mt, &owner);
                        lower(st, mw, c, lane == 0);  // (the value left out was the warp's)
                        st.m = mw;
                        if (lane == owner) {
                            // The value becomes one whose term is 0: 150 below in the exponent to base 2, and far enough for 16 bits; a
                            // masked one where there is no such value.
                            float low = E::round(mw - fmaxf(far, fabsf(mw) * 0x1p-6f));
                            if (!((low - mw) * c < -140.f)) low = -INFINITY;
                            const uint32_t gone = E::bits(low);
                            uint4 y = raw[LP_STEP - 1];  // the first vector that has it
#pragma unroll
                            for (int i = LP_STEP - 2; i >= 0; --i)
                                if (mx[i] == mw) y = raw[i];
                            float x[E::N];
                            E::open(y, x);
                            int at = 0;
#pragma unroll
                            for (int j = 1; j < E::N; ++j)
                                if (x[j] == mw) at = j;
                            uint32_t u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int j = 0; j < E::N; ++j)
                                if (j == at) E::set(u, j, gone);
                            bool found = false;
#pragma unroll
                            for (int i = 0; i < LP_STEP; ++i) {
                                if (!found && mx[i] == mw) raw[i] = make_uint4(u[0], u[1], u[2], u[3]);
                                found |= mx[i] == mw;
                            }
                        }
                    }
                    const float mu = st.m == -INFINITY ? 0.f : st.m;
                    float ds = 0.f, dh = 0.f;
                    if (!edge) {
                        F2 s2 = f2(0.f, 0.f), h2 = s2;
                        const F2 nm = f2(-mu, -mu), cc = f2(c, c);
#pragma unroll
                        for (int i = 0; i < LP_STEP; ++i) {
                            float x[E::N];
                            E::open(raw[i], x);
#pragma unroll
                            for (int j = 0; j < E::N; j += 2) {
                                const F2 t = mulp2(add2(f2(x[j], x[j + 1]), nm), cc);
                                const float2 tt = unpack2(t);
                                const F2 e = f2(lp_ex2(tt.x), lp_ex2(tt.y));
                                s2 = add2(s2, e);
                                h2 = fma2(e, t, h2);
                            }
                        }
                        const float2 s = unpack2(s2), h = unpack2(h2);
                        ds = s.x + s.y;
                        dh = h.x + h.y;
                    }
                    if (edge || dh != dh) {  // masked values give 0 * -inf: a floor under the exponents
                        ds = dh = 0.f;
#pragma unroll
                        for (int i = 0; i < LP_STEP; ++i) {
                            float x[E::N];
                            E::open(raw[i], x);
#pragma unroll
                            for (int j = 0; j < E::N; ++j) {
                                const float t = max_nan((x[j] - mu) * c, LP_FLOOR), e = lp_ex2(t);
                                ds += e;
                                dh += e * t;
                            }
                        }
                    }
                    st.s += ds;
                    st.h += dh;
                }
                if (TOP) {
                    if (!(m_group <= top[LP_TOP - 1]) && w0 + lane * VECS < r.v1) {  // (no maximum is NaN)
                        int at = tile;
                        float o = m_group;
#pragma unroll
                        for (int i = 0; i < LP_TOP; ++i)
                            if (!(o <= top[i])) {
                                const float x = top[i];
                                const int y = top_tile[i];
                                top[i] = o, top_tile[i] = at;
                                o = x, at = y;
                            }
                    }
                }
            } else if (lane == 0) {
                mbarrier_arrive_one(&empty[stage]);
            }
            if (p_row < a.M) {  // the stage goes out again
                if (warp == sender && lane == 0) {
                    if (mbar_wait(&empty[stage], turn, a.status, DEV_TIMEOUT_SLOT, &abort) && !*(volatile int *)&abort) send(stage);
                }
                __syncwarp();
                advance();
            }
            if (++stage == STAGES) stage = 0, turn ^= 1;
        }
        const bool has = token >= 0 && token < a.V;
        const float x_t = has ? E::one(r.base, token) : 0.f;  // (asked for here: the token has arrived)
        // the CTA's sums
        for (int o = 16; o; o >>= 1) {  // (lanes share the maximum)
            st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
            st.h += __shfl_xor_sync(0xffffffffu, st.h, o);
        }
        if (lane == 0) ws[warp] = st;
        __syncthreads();
        if (warp == 0) {
            st = ws[lane % LP_WARPS];
            for (int o = LP_WARPS / 2; o; o >>= 1)
                st = join(st, Stat{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o),
                                   __shfl_xor_sync(0xffffffffu, st.h, o)}, c);
        }
        if (TOP) {
            // the k groups of largest maxima
            auto key_of = [&](int i) { return top_tile[i] >= 0 ? lp_key(lp_order(top[i]), group0 + top_tile[i] * LP_THREADS) : 0; };
            const u64 mine = key_of(0);
            select_best(mine, a.k, sh, 0, [&](auto &&f) {
#pragma unroll
                for (int i = 0; i < LP_TOP; ++i) f(key_of(i));
                // others of a thread may matter: the warp reads its groups once more, a group a lane
                unsigned more = __ballot_sync(0xffffffffu, top_tile[LP_TOP - 1] >= 0 && lp_order(top[LP_TOP - 1]) >= (uint32_t)(sh.bar >> 32));
                for (; more; more &= more - 1) {
                    const int of = __ffs(more) - 1;
                    int kept[LP_TOP];
#pragma unroll
                    for (int i = 0; i < LP_TOP; ++i) kept[i] = __shfl_sync(0xffffffffu, top_tile[i], of);
                    for (int t = lane, g = group0 - lane + of + t * LP_THREADS; g * VECS < r.v1; t += 32, g += 32 * LP_THREADS) {
                        bool known = false;
#pragma unroll
                        for (int i = 0; i < LP_TOP; ++i) known |= t == kept[i];
                        if (known) continue;
                        uint32_t o = 0;
#pragma unroll
                        for (int i = 0; i < VECS; ++i) {
                            const int at = g * VECS + i;
                            if (at < r.v1 && at >= r.whole0 && at < r.whole1) {
                                o = max(o, lp_order(E::largest(*(reinterpret_cast<const uint4 *>(r.vbase) + at))));
                            } else if (at < r.v1) {
                                for (int e = max(0, at * E::N - r.skew); e < min(a.V, (at + 1) * E::N - r.skew); ++e)
                                    o = max(o, lp_order(E::one(r.base, e)));
                            }
                        }
                        f(lp_key(o, g));
                    }
                }
            });
        }
        if (a.slices > 1) {
            // the slices' results go to the first CTA (which waits for no answer, as it would if it fetched them)
            cluster_wait();  // (it has read those of the row before)
            if (warp == 0) {
                if (lane == 0) {
                    const uint32_t to = map_cta(smem_u32(&slice_stat[slice]), 0);
                    st_cluster(to, st.m);
                    st_cluster(to + 4, st.s);
                    st_cluster(to + 8, st.h);
                }
                if (TOP && lane < a.k) {
                    const u64 x = sh.best[lane];
                    st_cluster_v2(map_cta(smem_u32(&slice_best[slice][lane]), 0), __uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
                }
            }
            cluster_sync();
            if (slice == 0) {
                if (warp == 0) {
                    st = lane < a.slices ? slice_stat[lane] : Stat{-INFINITY, 0.f, 0.f};
                    for (int o = 16; o; o >>= 1)
                        st = join(st, Stat{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o),
                                           __shfl_xor_sync(0xffffffffu, st.h, o)}, c);
                }
                if (TOP) {
                    constexpr int PER = LP_CLUSTER * LP_MAX_K / LP_THREADS;
                    u64 keys[PER], best = 0;
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const int q = (tid + i * LP_THREADS) / LP_MAX_K, j = tid % LP_MAX_K;
                        keys[i] = q < a.slices && j < a.k ? slice_best[q][j] : 0;
                        best = max(best, keys[i]);
                    }
                    select_best(best, a.k, sh, 0, [&](auto &&f) {
#pragma unroll
                        for (int i = 0; i < PER; ++i) f(keys[i]);
                    });
                }
            }
            cluster_arrive();
        }
        if (slice == 0) {
            // (one lane's sums for all: joined the other way round they may differ by a rounding)
            st = Stat{__shfl_sync(0xffffffffu, st.m, 0), __shfl_sync(0xffffffffu, st.s, 0), __shfl_sync(0xffffffffu, st.h, 0)};
            if (TOP) {
                // the k best of the groups' values (of all slices: groups are counted over the whole row)
                // The k groups' maxima reach the k-th of them, wherever in its group it lies.
                constexpr int PER = LP_MAX_K * LP_GROUP / LP_THREADS;
                const u64 kth = sh.best[a.k - 1];
                const u64 at_least = kth ? lp_key((uint32_t)(kth >> 32), key_index(kth) * LP_GROUP + LP_GROUP - 1 - r.skew) : 0;
                float x[PER];
                int e[PER];  // -1: none
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int at = tid + i * LP_THREADS;
                    const u64 group = at < a.k * LP_GROUP ? sh.best[at / LP_GROUP] : 0;
                    e[i] = group ? key_index(group) * LP_GROUP + at % LP_GROUP - r.skew : -1;
                    if (e[i] >= a.V) e[i] = -1;
                    x[i] = e[i] >= 0 ? E::one(r.base, e[i]) : 0.f;
                }
                u64 keys[PER], best = 0;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    keys[i] = e[i] >= 0 ? lp_key(lp_order(x[i]), e[i]) : 0;
                    best = max(best, keys[i]);
                }
                auto each = [&](auto &&f) {
#pragma unroll
                    for (int i = 0; i < PER; ++i) f(keys[i]);
                };
                __syncthreads();  // (sh.best has been read)
                select_best(best, a.k, sh, at_least, each);
            }
            if (warp == 0) Finish{a}(row, st, sh.best, x_t, has, token);  // (the warp that has the row's sums)
        }
        __syncthreads();  // (best and ws are the next row's)
    }
    if (a.slices > 1) cluster_wait();
    if (tid == 0 && *(volatile int *)&abort)  // error path: the copies in flight get a bounded chance to land
        for (int i = 0; i < STAGES; ++i)
            if (sent[i] > 0 && !mbar_wait(&full[i], (sent[i] - 1) & 1, nullptr, 0, nullptr)) break;  // (all had this second)
    if (blockIdx.x == a.slices - 1) check_tokens(a);  // (which has nothing else to do by now)
}

// Slices of a row, CTAs of its cluster, by estimated time.  Rows run in rounds of as many as the GPU holds at once.  A full
// round takes its bytes at the memory's rate; in the last one fewer CTAs share it, up to what one CTA gets through alone
// (`cta`: its instructions follow one another, 16-bit values have twice as many a byte).  Each round has a fixed part, longer
// for clusters, whose CTAs wait for one another.  Clusters of 16 are for rows that leave them SMs of their own, and sizes between
// these lose more than they give, since GPCs do not divide by them.  Rows of 151936 values with alternatives, us with 1, 2, 3, 4,
// 6, 8, 10, 16 slices: 17 fp32 21, 16.2, 13.5, 11.8, 10.8, 10.9, 10.2, 11.2; 32 bf16 19.2, 15.2, 12.8, 11.4, 12.0, 10.9, 11.7, 18;
// 64 fp32 22, 17.7, 16.9, 16.3, 17.4, 22, 22, 35; 136 bf16 21.3, 20.6, 21.3, 27 (4); 300 fp32 33, 43 (2); 1 fp32 20.8, 16.2, 13.9,
// 11.9 (4), 10.0 (8), 9.2 (16).
int pick_slices(int M, int vecs, int tile, int size, const int (&clusters)[LP_CLUSTER + 1], bool top) {
    const double rate = 6.6e6, cta = size == 2 ? 22e3 : 34e3;  // bytes a us
    int best = 1;
    double least = 0;
    for (const int s : {1, 2, 4, 8, 10, 16}) {
        if (s > 1 && ((long long)(s - 1) * tile >= vecs || clusters[s] < 1 || (s == 16 && (long long)M * s > gemm_ctas()))) continue;
        const double bytes = 16.0 * vecs / s;  // of a CTA and round
        const int full = M / clusters[s], rest = M % clusters[s];
        double us = full * (bytes * clusters[s] * s / rate + (s > 1 ? 6.0 : 1.0)) + (top ? (s > 1 ? 4.0 : 2.5) : 0.0);
        if (rest > 0) us += bytes / std::min(cta, rate / ((double)rest * s)) + (s > 1 ? 2.0 : 1.0);
        if (s == 1 || us < least) best = s, least = us;
    }
    return best;
}

template <int TYPE, bool TOP>
cudaError_t launch(LogprobArgs &a, cudaStream_t st) {
    using E = Elem<TYPE>;
    constexpr size_t MOST = (size_t)E::STAGES * LP_THREADS * LP_GROUP * E::SIZE;  // the ring
    static thread_local int configured = -1, clusters[LP_CLUSTER + 1];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(LP_THREADS);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (configured != dev) {
        const void *f = reinterpret_cast<const void *>(k_logprobs<TYPE, TOP>);
        e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        cfg.dynamicSmemBytes = MOST;
        clusters[1] = gemm_ctas() * LP_CTAS;
        for (int s = 2; s <= LP_CLUSTER; ++s) {
            cfg.gridDim = dim3((unsigned)s);
            attr[0].val.clusterDim.x = (unsigned)s;
            if (cudaOccupancyMaxActiveClusters(&clusters[s], f, &cfg) != cudaSuccess) {
                clusters[s] = 0;
                cudaGetLastError();  // (the answer is not an error of a later call)
            }
        }
        configured = dev;
    }
    // (a row that starts off a 16-byte boundary has one vector more)
    const int vecs = (a.V + E::N - 1) / E::N + 1;
    a.slices = pick_slices(a.M, vecs, LP_THREADS * LP_GROUP / E::N, E::SIZE, clusters, TOP);
    a.slice_vecs = ((vecs + a.slices - 1) / a.slices + LP_THREADS - 1) / LP_THREADS * LP_THREADS;
    cfg.gridDim = dim3((unsigned)(std::min(a.M, clusters[a.slices]) * a.slices));
    cfg.dynamicSmemBytes = MOST;
    cfg.stream = st;
    attr[0].val.clusterDim.x = (unsigned)a.slices;
    return cudaLaunchKernelEx(&cfg, k_logprobs<TYPE, TOP>, static_cast<const LogprobArgs>(a));
}

template <int TYPE>
cudaError_t launch_type(LogprobArgs &a, cudaStream_t st) {
    return a.k > 0 ? launch<TYPE, true>(a, st) : launch<TYPE, false>(a, st);
}

}  // namespace

cudaError_t launch_logprobs(LogprobArgs &a, cudaStream_t st) {
    return a.type == PBD_FP32 ? launch_type<PBD_FP32>(a, st) : a.type == PBD_BF16 ? launch_type<PBD_BF16>(a, st) : launch_type<PBD_FP16>(a, st);
}

}  // namespace pbd
