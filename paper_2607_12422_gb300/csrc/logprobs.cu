// logprobs.cu -- log probabilities of given tokens, entropy and top alternatives from logits (pbd_op_token_logprobs).
//
// Of a row x of V logits at temperature T, with m = max x, S = sum exp((x - m) / T):
//     logprob(t) = (x_t - m) / T - ln S
//     entropy    = ln S + sum (m - x) / T exp((x - m) / T) / S      (both terms >= 0: nothing cancels)
//     top k      by value, then by the lower index
// in one pass over the logits, which bounds it: running maximum and sums in fp32 per thread, joined at the end.  Few
// rows are cut into slices, one CTA each, and k_logprobs_join joins them.
//
// The alternatives come from the same pass.  The first tile of a slice (16 KB) gives a threshold: the k-th largest of the
// threads' own maxima, which at least k values reach.  Only k threads can hold values that reach it, so
// few do; they go to a list in shared memory.  Of later tiles only what is above the threshold is added, some k / i of the i-th
// tile when the order is random.  If an unlucky order fills the list, it is cut to its k best, which raise the
// threshold.
#include <algorithm>
#include <cuda_fp16.h>

#include "../../include/pbd_ops.h"
#include "kv_ops.h"

namespace pbd {

namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_VECS = 4;                        // 16-byte loads of a thread and tile
constexpr int LP_TILE = LP_THREADS * LP_VECS;     // vectors of a tile
constexpr int LP_LIST = 2048;                     // more than k of the list and a tile's k threads' 32 values each
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

// (value, lower index first) as one number; NaN below everything, 0 is nobody's
__device__ __forceinline__ u64 lp_key(float x, int i) {
    const uint32_t u = __float_as_uint(x + 0.f);  // (-0 counts as 0)
    const uint32_t v = x != x ? 0u : (u & 0x80000000u ? ~u : u | 0x80000000u);
    return (u64)v << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(u64 k) {
    const uint32_t v = (uint32_t)(k >> 32);
    return v == 0 ? __uint_as_float(0x7fffffffu) : __uint_as_float(v & 0x80000000u ? v & 0x7fffffffu : ~v);
}
__device__ __forceinline__ int key_index(u64 k) { return (int)~(uint32_t)k; }

template <int TYPE>
struct Elem;  // values of a 16-byte vector
template <>
struct Elem<PBD_FP32> {
    static constexpr int N = 4, SIZE = 4;
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return static_cast<const float *>(p)[i]; }
};
template <>
struct Elem<PBD_BF16> {
    static constexpr int N = 8, SIZE = 2;
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return bf2f(static_cast<const bf16 *>(p)[i]); }
};
template <>
struct Elem<PBD_FP16> {
    static constexpr int N = 8, SIZE = 2;
    static __device__ __forceinline__ void open(const uint4 &v, float *x) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float one(const void *p, long long i) { return __half2float(static_cast<const __half *>(p)[i]); }
};

// maximum, sum of e = exp((x - m) / T), sum of e * log2(e)
struct Stat {
    float m, s, h;
};
// b's sums at a's maximum, and the other way round
__device__ __forceinline__ Stat join(const Stat &a, const Stat &b, float c) {
    const float m = fmaxf(a.m, b.m), mu = m == -INFINITY ? 0.f : m;
    // e 2^d has the logarithm log2 e + d; a part without anything (m = -inf, s = 0) stays 0
    const float da = max_nan((a.m - mu) * c, LP_FLOOR), db = max_nan((b.m - mu) * c, LP_FLOOR);
    const float fa = lp_ex2(da), fb = lp_ex2(db);
    return Stat{m, a.s * fa + b.s * fb, (a.h + a.s * da) * fa + (b.h + b.s * db) * fb};
}

// The k best of n keys of a list in shared memory, sorted, to its front (and the k-th returned; 0 if there are
// fewer).  Keys differ, so a key's place is the number of larger ones.  Whole CTA; `tmp` holds k keys.
__device__ __forceinline__ u64 keep_best(u64 *list, int n, int k, u64 *tmp) {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
        const u64 mine = list[i];
        int r = 0;
        for (int j = 0; j < n; ++j) r += list[j] > mine;
        if (r < k) tmp[r] = mine;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < min(n, k); i += LP_THREADS) list[i] = tmp[i];
    const u64 last = n >= k ? tmp[k - 1] : 0;
    __syncthreads();
    return last;
}

// The k-th largest of one key a thread (0: none); 0 if fewer than k threads have one.  Whole CTA.
__device__ __forceinline__ u64 kth_of_threads(u64 mine, int k, u64 *all, u64 *out) {
    __syncthreads();
    all[threadIdx.x] = mine;
    if (threadIdx.x == 0) *out = 0;
    __syncthreads();
    int r = 0;
    for (int j = 0; j < LP_THREADS; ++j) r += all[j] > mine;
    if (mine && r == k - 1) *out = mine;
    __syncthreads();
    return *out;
}

struct Finish {  // a row's results
    const LogprobArgs &a;
    __device__ __forceinline__ void operator()(int row, const Stat &s, const u64 *best, float x_t, bool has_token) const {
        const float ls = logf(s.s), t = a.inv_t, mu = s.m == -INFINITY ? 0.f : s.m;
        const bool empty = s.m == -INFINITY && s.s == 0.f;  // nothing but -inf
        if (threadIdx.x == 0) {
            if (a.logprob) {
                const int token = a.tokens[row];
                float lp = token < 0 ? 0.f : __uint_as_float(0x7fffffffu);
                if (has_token) lp = empty ? -INFINITY : (x_t - mu) * t - ls;
                a.logprob[row] = lp;
            }
            if (a.entropy) a.entropy[row] = empty ? 0.f : ls - 0.6931471805599453f * (s.h / s.s);
        }
        for (int i = threadIdx.x; i < a.k; i += LP_THREADS) {
            a.top_ids[(long long)row * a.k + i] = key_index(best[i]);
            a.top_lp[(long long)row * a.k + i] = empty ? -INFINITY : (key_value(best[i]) - mu) * t - ls;
        }
    }
};

template <int TYPE>
__device__ __forceinline__ float token_logit(const LogprobArgs &a, int row, bool *has) {
    *has = false;
    if (!a.logprob || threadIdx.x != 0) return 0.f;
    const int t = a.tokens[row];
    *has = t >= 0 && t < a.V;
    if (t >= a.V) latch_error(a.status, DEV_BAD_TOKEN);
    return *has ? Elem<TYPE>::one(a.x, row * a.ld + t) : 0.f;
}

template <int TYPE, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs(const LogprobArgs a) {
    using E = Elem<TYPE>;
    constexpr int PER = LP_VECS * E::N;
    __shared__ u64 list[TOP ? LP_LIST : 1], tmp[TOP ? LP_THREADS : 1], kth;
    __shared__ int added[3];
    __shared__ Stat ws[LP_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices;
    if (a.slices > 1) {
        pdl_launch();
        if (blockIdx.x == 0 && tid == 0) *a.status = DEV_OK;  // (k_logprobs_join latches)
    }
    const float c = a.inv_t * 1.4426950408889634f;
    // vectors are counted from the 16-byte boundary at or before the row's first value
    const char *base = static_cast<const char *>(a.x) + row * a.ld * E::SIZE;
    const int skew = (int)(reinterpret_cast<uintptr_t>(base) & 15) / E::SIZE;
    const char *vbase = base - skew * E::SIZE;
    const int vecs = (a.V + skew + E::N - 1) / E::N;
    const int v0 = slice * a.slice_vecs, v1 = min(vecs, v0 + a.slice_vecs);

    Stat st{-INFINITY, 0.f, 0.f};
    float bar = -INFINITY;  // threshold of later tiles
    int have = 0, turn = 0;
    bool first = true;
    if (TOP && tid < 3) added[tid] = 0;
    if (TOP) __syncthreads();
    for (int v = v0; v < v1; v += LP_TILE, first = false) {
        float x[PER];
        uint4 raw[LP_VECS];
#pragma unroll
        for (int i = 0; i < LP_VECS; ++i) {
            const int at = v + i * LP_THREADS + tid, e0 = at * E::N - skew;
            if (at < v1 && e0 >= 0 && e0 + E::N <= a.V)
                raw[i] = __ldcs(reinterpret_cast<const uint4 *>(vbase) + at);
        }
#pragma unroll
        for (int i = 0; i < LP_VECS; ++i) {
            const int at = v + i * LP_THREADS + tid, e0 = at * E::N - skew;
            if (at < v1 && e0 >= 0 && e0 + E::N <= a.V) {
                E::open(raw[i], x + i * E::N);
            } else {  // a row's ends, value by value; nothing behind the slice
#pragma unroll
                for (int j = 0; j < E::N; ++j)
                    x[i * E::N + j] = at < v1 && e0 + j >= 0 && e0 + j < a.V ? E::one(base, e0 + j) : -INFINITY;
            }
        }
        float mx = x[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) mx = fmaxf(mx, x[i]);
        const float mn = fmaxf(st.m, mx);
        if (mn > st.m) {
            const float d = max_nan((st.m - mn) * c, LP_FLOOR), f = lp_ex2(d);
            st.h = (st.h + st.s * d) * f;
            st.s *= f;
            st.m = mn;
        }
        const float mu = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // (-inf would give 0 * -inf)
            const float t = max_nan((x[i] - mu) * c, LP_FLOOR), e = lp_ex2(t);
            st.s += e;
            st.h += e * t;
        }
        if (TOP) {
            auto index = [&](int i) { return (v + (i / E::N) * LP_THREADS + tid) * E::N + i % E::N - skew; };
            auto real = [&](int i) {
                const int at = v + (i / E::N) * LP_THREADS + tid, e = index(i);
                return at < v1 && e >= 0 && e < a.V;
            };
            // adds the thread's values that reach T
            auto add = [&](u64 T, int *count, int from) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const u64 k = lp_key(x[i], index(i));
                    if (real(i) && k >= T) list[from + atomicAdd(count, 1)] = k;
                }
            };
            auto by_threads = [&](u64 floor) {  // by the k-th of the threads' maxima
                u64 best = 0;
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (real(i)) best = max(best, lp_key(x[i], index(i)));
                const u64 T = max(floor, kth_of_threads(best, a.k, tmp, &kth));
                if (best >= T && best) add(T, &added[turn], have);
                return T;
            };
            const int next = turn == 2 ? 0 : turn + 1;
            if (first) {
                const u64 T = by_threads(0);
                bar = T ? key_value(T) : -INFINITY;
            } else {
                if (mx > bar) {
#pragma unroll
                    for (int i = 0; i < PER; ++i)
                        if (x[i] > bar) {
                            const int p = have + atomicAdd(&added[turn], 1);
                            if (p < LP_LIST) list[p] = lp_key(x[i], index(i));
                        }
                }
            }
            if (tid == 0) added[next] = 0;  // (last read before the barrier that ended the tile before)
            __syncthreads();
            int now = added[turn];
            if (have + now > LP_LIST) {  // what this tile added is dropped, the list cut, the tile looked at again
                const u64 T = keep_best(list, have, a.k, tmp);
                have = min(have, a.k);
                if (tid == 0) added[turn] = 0;
                __syncthreads();
                by_threads(T);
                __syncthreads();
                now = added[turn];
                const u64 T2 = keep_best(list, have + now, a.k, tmp);
                have = min(have + now, a.k);
                bar = T2 ? key_value(T2) : bar;
            } else {
                have += now;
            }
            turn = next;
        }
    }
    // the CTA's sums
    for (int o = 16; o; o >>= 1)
        st = join(st, Stat{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o),
                           __shfl_xor_sync(0xffffffffu, st.h, o)}, c);
    if (lane == 0) ws[warp] = st;
    if (TOP) keep_best(list, have, a.k, tmp);
    __syncthreads();
    st = ws[0];
    for (int i = 1; i < LP_WARPS; ++i) st = join(st, ws[i], c);
    if (a.slices == 1) {
        bool has;
        const float xt = token_logit<TYPE>(a, row, &has);
        Finish{a}(row, st, list, xt, has);
        return;
    }
    if (tid == 0) reinterpret_cast<float4 *>(a.stats)[blockIdx.x] = make_float4(st.m, st.s, st.h, 0.f);
    if (TOP)
        for (int i = tid; i < a.k; i += LP_THREADS) a.cand[(long long)blockIdx.x * a.k + i] = i < have ? list[i] : 0;
}

// Joins a row's slices: one CTA a row.
template <int TYPE, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs_join(const LogprobArgs a) {
    __shared__ u64 list[TOP ? LP_LIST : 1], tmp[TOP ? LP_THREADS : 1], kth;
    __shared__ int added;
    __shared__ Stat ws[LP_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x;
    const float c = a.inv_t * 1.4426950408889634f;
    pdl_wait();
    bool has;
    const float xt = token_logit<TYPE>(a, row, &has);
    Stat st{-INFINITY, 0.f, 0.f};
    const float4 *stats = reinterpret_cast<const float4 *>(a.stats) + (long long)row * a.slices;
    for (int i = tid; i < a.slices; i += LP_THREADS) {
        const float4 p = stats[i];
        st = join(st, Stat{p.x, p.y, p.z}, c);
    }
    for (int o = 16; o; o >>= 1)
        st = join(st, Stat{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o),
                           __shfl_xor_sync(0xffffffffu, st.h, o)}, c);
    if (lane == 0) ws[warp] = st;
    if (TOP) {
        // of slices * k keys (at most 32 a thread) those that reach the k-th of the threads' maxima
        const u64 *cand = a.cand + (long long)row * a.slices * a.k;
        const int n = a.slices * a.k;
        u64 best = 0;
        for (int i = tid; i < n; i += LP_THREADS) best = max(best, cand[i]);
        if (tid == 0) added = 0;
        const u64 T = kth_of_threads(best, a.k, tmp, &kth);
        if (best >= T)
            for (int i = tid; i < n; i += LP_THREADS) {
                const u64 k = cand[i];
                if (k && k >= T) list[atomicAdd(&added, 1)] = k;
            }
        __syncthreads();
        keep_best(list, added, a.k, tmp);
    }
    __syncthreads();
    st = ws[0];
    for (int i = 1; i < LP_WARPS; ++i) st = join(st, ws[i], c);
    Finish{a}(row, st, list, xt, has);
}

template <int TYPE, bool TOP>
cudaError_t launch(LogprobArgs &a, cudaStream_t st) {
    using E = Elem<TYPE>;
    cudaError_t e;
    // (a row that starts off a 16-byte boundary has one vector more)
    const int vecs = (a.V + E::N - 1) / E::N + 1;
    a.slice_vecs = ((vecs + a.slices - 1) / a.slices + LP_THREADS - 1) / LP_THREADS * LP_THREADS;
    if (a.slices == 1 && (e = cudaMemsetAsync(a.status, 0, sizeof(int), st)) != cudaSuccess) return e;
    k_logprobs<TYPE, TOP><<<a.M * a.slices, LP_THREADS, 0, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess || a.slices == 1) return e;
    return launch_pdl(k_logprobs_join<TYPE, TOP>, a.M, LP_THREADS, 0, st, a);
}

template <int TYPE>
cudaError_t launch_type(LogprobArgs &a, cudaStream_t st) {
    return a.k > 0 ? launch<TYPE, true>(a, st) : launch<TYPE, false>(a, st);
}

}  // namespace

// Slices of a row: enough CTAs to fill the GPU, each with a tile of 16 KB or more; at most 256, so that the join's
// threads see at most 32 candidates each.
int logprob_slices(int M, int V, int es) {
    const long long tiles = ((long long)V * es / 16 + LP_TILE - 1) / LP_TILE;
    const long long want = (152 * 4 + M - 1) / M;
    return (int)std::max(1ll, std::min(std::min(tiles, want), 256ll));
}

cudaError_t launch_logprobs(LogprobArgs &a, cudaStream_t st) {
    return a.type == PBD_FP32 ? launch_type<PBD_FP32>(a, st) : a.type == PBD_BF16 ? launch_type<PBD_BF16>(a, st) : launch_type<PBD_FP16>(a, st);
}

}  // namespace pbd
