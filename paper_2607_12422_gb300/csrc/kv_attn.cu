// kv_attn.cu -- attention of one new token a sequence over a caller's paged cache (pbd_op_decode_attention).
//
// For query head h of KV head h / group and cached slot j:
//     s_hj = q_h . k_j,   p_hj = exp(scale (s_hj - max_j s_hj)),   l_h = sum_j p_hj,   out_h = sum_j p_hj v_j / l_h
// in one pass over K and V with a running maximum and sum.  Every cached byte is read once and used for the few
// query heads of its group, so memory bounds it.
//
// Work is cut into units of 16 slots of one (sequence, KV head).  All units of the batch form one list,
// [sequence][KV head][tile], and each warp takes one contiguous stretch of it, all of the same length: how ragged the
// lengths are does not matter, and the host need not know them.  A warp has its own ring of units in shared memory, filled by
// 16-byte asynchronous copies, and never waits for another warp.  Where a stretch begins or ends inside a
// (sequence, KV head) the warp leaves maximum, sum and unnormalised output in scratch, and k_decode_join joins them.
//
// Tensor cores: scores are taken as S^T = K Q^T, 16 slots by 8 heads a tile, and outputs as O^T = V^T P^T, 16 dims by 8 heads,
// so groups of up to 8 heads waste no rows of a tile; groups up to 16 take two tiles, larger ones are cut
// into chunks of 16.  (mma.sync: a tcgen05 tile of 128 rows would be one sixteenth full.)
#include <algorithm>
#include <cuda_fp16.h>

#include "kv_ops.h"

namespace pbd {

namespace {

constexpr int DA_WARPS = 4;
constexpr int DA_SLOTS = 16;  // slots of a unit
constexpr int DA_MIN_UNITS = 2;

// stages of a warp's ring and CTAs that fit an SM's shared memory: 96 KB (d = 256: 192 KB) a CTA
template <int D>
struct DaShape {
    static constexpr int UNIT = DA_SLOTS * D * 2 * 2;  // bytes: K rows, then V rows
    static constexpr int STAGES = D == 64 ? 6 : 3;
    static constexpr int CTAS = D == 256 ? 1 : 2;
    static constexpr int RING = DA_WARPS * STAGES * UNIT;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool read) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(read ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <bool FP16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (FP16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        mma_m16n8k16_bf16(d, a, b0, b1);
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
    if (FP16) {
        __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<uint32_t *>(&h);
    }
    return pack_bf162(x, y);
}
template <bool FP16>
__device__ __forceinline__ float2 unpack16(uint32_t a) {
    if (FP16) return __half22float2(*reinterpret_cast<__half2 *>(&a));
    return make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
}
template <bool FP16>
__device__ __forceinline__ uint16_t round16(float x) {
    if (FP16) return __half_as_ushort(__float2half_rn(x));
    return __bfloat16_as_ushort(f2bf(x));
}

// Slots that the call attends to in sequence b.  Lengths outside the table (which k_decode_join reports) are cut.
__device__ __forceinline__ int attended(const DecodeArgs &a, int b) {
    const int add = a.k_new ? 1 : 0;
    const long long most = a.kv.cap - add;
    return (int)max(0ll, min((long long)a.kv.lens[b], most)) + add;
}

// first[b]: 16-slot tiles of the sequences before b, first[B] all of them; len[b]: slots attended to.  Whole CTA.
__device__ __forceinline__ void tile_lists(const DecodeArgs &a, int *first, int *len) {
    __shared__ int warp_sum[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < a.kv.B; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        const int n = b < a.kv.B ? attended(a, b) : 0;
        if (b < a.kv.B) len[b] = n;
        int x = (n + DA_SLOTS - 1) / DA_SLOTS;
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
        if (b < a.kv.B) first[b + 1] = before + x;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) first[0] = 0;
    __syncthreads();
}

// warps that share `units` units, and the first unit of one of them
__device__ __forceinline__ int workers_of(const DecodeArgs &a, int units) {
    return max(1, min(a.workers, (units + DA_MIN_UNITS - 1) / DA_MIN_UNITS));
}
__device__ __forceinline__ int first_unit(int w, int units, int workers) {
    return (int)((long long)w * units / workers);
}

// A place in the list of units.
struct UnitAt {
    int b, hc, t, tiles;  // sequence, KV head and chunk of its query heads, tile, tiles of the sequence
    __device__ __forceinline__ void seek(int u, const int *first, int B, int HC) {
        int lo = 0, hi = B;  // first[lo] * HC <= u < first[hi] * HC
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((long long)first[mid] * HC <= u)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
        tiles = first[b + 1] - first[b];
        const int r = u - first[b] * HC;
        hc = r / tiles;
        t = r - hc * tiles;
    }
    __device__ __forceinline__ void next(const int *first, int B, int HC) {
        if (++t < tiles) return;
        t = 0;
        if (++hc < HC) return;
        hc = 0;
        do ++b;
        while (b < B && first[b + 1] == first[b]);
        if (b < B) tiles = first[b + 1] - first[b];
    }
};

template <bool FP16, int D, int NT>
__global__ void __launch_bounds__(DA_WARPS * 32) k_decode_split(const DecodeArgs a) {
    using S = DaShape<D>;
    constexpr int HEADS = 8 * NT, KS = D / 16, CPR = D / 8;  // heads of a chunk, k steps, 16-byte pieces of a row
    extern __shared__ __align__(128) uint8_t smem[];
    const int B = a.kv.B, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t ring = smem_u32(smem) + warp * S::STAGES * S::UNIT;
    int *first = reinterpret_cast<int *>(smem + S::RING), *len = first + B + 1;
    pdl_launch();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = DEV_OK;  // (k_decode_join latches)
    tile_lists(a, first, len);
    const int chunks = (a.group + HEADS - 1) / HEADS, HC = a.kv.hkv * chunks;
    const int units = first[B] * HC, workers = workers_of(a, units);
    const int w = warp * gridDim.x + blockIdx.x;  // neighbours in the list on different SMs
    if (units == 0 || w >= workers) return;
    const int u_end = first_unit(w + 1, units, workers);
    int u = first_unit(w, units, workers);
    UnitAt ld, at;
    ld.seek(u, first, B, HC);
    at = ld;
    const bool append = a.k_new != nullptr;
    // P's scale: weights of fp16 lie in 2^-24 .. 2^14, so that what is far below the maximum keeps its bits
    const float shift = FP16 ? 14.f : 0.f, c = a.scale * 1.4426950408889634f;

    // page of slot lane % 16 of the unit at ld; -1: none
    auto page_of = [&]() {
        const int slot = ld.t * DA_SLOTS + (lane & 15);
        if (slot >= len[ld.b]) return -1;
        const int p = a.kv.table[(long long)ld.b * a.kv.max_pages + slot / a.kv.page_size];
        return (unsigned)p < (unsigned)a.kv.n_pages ? p : -1;
    };
    // Copies the unit at ld into a stage: lanes 0-15 know K's rows, 16-31 V's.  Rows that are none arrive as zeros.
    auto issue = [&](int page, int stage) {
        const int slot = ld.t * DA_SLOTS + (lane & 15), h = ld.hc / chunks, n = len[ld.b];
        const bool is_new = append && slot == n - 1;
        const long long off = (long long)page * a.kv.stride_page + h * a.kv.stride_head +
                              (long long)(slot % a.kv.page_size) * a.kv.stride_slot;
        const uint16_t *row = nullptr;
        if (is_new)
            row = (lane < 16 ? a.k_new : a.v_new) + ld.b * a.new_stride + (long long)h * D;
        else if (page >= 0)
            row = (lane < 16 ? a.kv.k : a.kv.v) + off;
        const uint32_t st = ring + stage * S::UNIT;
#pragma unroll
        for (int j = 0; j < CPR / 2; ++j) {
            const int i = j * 32 + lane, r = i / CPR, cc = i % CPR;
            const uint32_t dst = st + r * (D * 2) + ((cc ^ (r & 7)) << 4);
            const uint16_t *ks = reinterpret_cast<const uint16_t *>(
                __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), r));
            const uint16_t *vs = reinterpret_cast<const uint16_t *>(
                __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), r + 16));
            cp_async16_or_zero(dst, ks ? ks + cc * 8 : a.kv.k, ks != nullptr);
            cp_async16_or_zero(dst + DA_SLOTS * D * 2, vs ? vs + cc * 8 : a.kv.v, vs != nullptr);
        }
        if (append && ld.t == ld.tiles - 1 && ld.hc % chunks == 0) {
            // the new token's row joins the cache; nobody reads it there in this call
            const int r = (n - 1) & 15;
            const long long o = __shfl_sync(0xffffffffu, off, r);
            const bool ok = __shfl_sync(0xffffffffu, page, r) >= 0;
            if (ok) {
                const long long src = ld.b * a.new_stride + (long long)h * D;
                for (int i = lane; i < CPR; i += 32) {
                    *reinterpret_cast<int4 *>(const_cast<uint16_t *>(a.kv.k) + o + i * 8) =
                        *reinterpret_cast<const int4 *>(a.k_new + src + i * 8);
                    *reinterpret_cast<int4 *>(const_cast<uint16_t *>(a.kv.v) + o + i * 8) =
                        *reinterpret_cast<const int4 *>(a.v_new + src + i * 8);
                }
            }
            if (lane == 0 && a.new_pos && a.kv.positions)
                a.kv.positions[((long long)ld.b * a.kv.hkv + h) * a.kv.cap + n - 1] = a.new_pos[ld.b];
        }
    };

    int to_load = u_end - u, page = page_of(), stage_in = 0;
    auto load_next = [&]() {
        if (to_load > 0) {
            issue(page, stage_in);
            stage_in = stage_in + 1 == S::STAGES ? 0 : stage_in + 1;
            if (--to_load > 0) {
                ld.next(first, B, HC);
                page = page_of();  // one unit ahead: its latency is not waited for here
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) load_next();

    uint32_t qf[KS][NT][2];
    float o[KS][NT][4], m[NT][2], l[NT][2];
    int stage = 0;
    bool fresh = true;
    int t_first = 0;
    // lane constants of the fragments' addresses
    const int k_row = (lane & 7) + ((lane >> 3) & 1) * 8, k_c = lane >> 4;
    const int v_row = (lane & 7) + (lane >> 4) * 8, v_c = (lane >> 3) & 1;
    for (; u < u_end; ++u) {
        const int n = len[at.b];
        if (fresh) {
            fresh = false;
            t_first = at.t;
            const int h = at.hc / chunks, ch = at.hc - h * chunks;
            const uint16_t *q = a.q + at.b * a.q_stride + (long long)(h * a.group + ch * HEADS) * D;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int j = nt * 8 + (lane >> 2);
                const bool real = ch * HEADS + j < a.group;
                const uint32_t *src = reinterpret_cast<const uint32_t *>(q + j * D + (lane & 3) * 2);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qf[ks][nt][0] = real ? src[ks * 8] : 0u;
                    qf[ks][nt][1] = real ? src[ks * 8 + 4] : 0u;
                }
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) o[ks][nt][0] = o[ks][nt][1] = o[ks][nt][2] = o[ks][nt][3] = 0.f;
            }
        }
        cp_async_wait<S::STAGES - 2>();
        __syncwarp();  // everybody's copies are there, and everybody is done with the stage that is filled next
        load_next();
        const uint32_t kst = ring + stage * S::UNIT, vst = kst + DA_SLOTS * D * 2;
        stage = stage + 1 == S::STAGES ? 0 : stage + 1;

        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint32_t f[4];
            ldmatrix4(f, kst + k_row * (D * 2) + (((ks * 2 + k_c) ^ (k_row & 7)) << 4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_16816<FP16>(s[nt], f, qf[ks][nt][0], qf[ks][nt][1]);
        }
        // s[nt]: slots lane / 4 and lane / 4 + 8, heads 2 (lane % 4) and the next
        const int slot = at.t * DA_SLOTS + (lane >> 2);
        if (slot >= n)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = -INFINITY;
        if (slot + 8 >= n)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][2] = s[nt][3] = -INFINITY;
        if (a.scores) {
            const int h = at.hc / chunks, ch = at.hc - h * chunks;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = ch * HEADS + nt * 8 + (lane & 3) * 2 + e;
                    if (j < a.group) {
                        float *dst = a.scores + ((long long)at.b * a.hq + h * a.group + j) * a.score_pitch + slot;
                        dst[0] = s[nt][e];
                        dst[8] = s[nt][2 + e];
                    }
                }
        }
        float mn[NT][2];
        bool grew = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = fmaxf(s[nt][e], s[nt][2 + e]);
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                mn[nt][e] = fmaxf(x, m[nt][e]);
                grew |= mn[nt][e] > m[nt][e];
            }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // (a maximum of -inf goes with a sum of 0: any finite factor will do)
                    const float f = mn[nt][e] > m[nt][e] ? ex2((m[nt][e] - mn[nt][e]) * c) : 1.f;
                    m[nt][e] = mn[nt][e];
                    l[nt][e] *= f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        o[ks][nt][e] *= f;
                        o[ks][nt][2 + e] *= f;
                    }
                }
        }
        // P^T as the B operand, 16 slots by 8 heads: high and low halves, each rounded to 16 bits, so that P keeps 16 bits
        // (22 in fp16) and the output's error is that of its own rounding
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mu = m[nt][e & 1] == -INFINITY ? 0.f : m[nt][e & 1];
                p[e] = ex2((s[nt][e] - mu) * c + shift);
                l[nt][e & 1] += p[e];
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t hi = pack2<FP16>(p[2 * half], p[2 * half + 1]);
                const float2 r = unpack16<FP16>(hi);
                ph[nt][half] = transpose8x8(hi);
                pl[nt][half] = transpose8x8(pack2<FP16>(p[2 * half] - r.x, p[2 * half + 1] - r.y));
            }
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint32_t f[4];
            ldmatrix4_trans(f, vst + v_row * (D * 2) + (((ks * 2 + v_c) ^ (v_row & 7)) << 4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                mma_16816<FP16>(o[ks][nt], f, ph[nt][0], ph[nt][1]);
                mma_16816<FP16>(o[ks][nt], f, pl[nt][0], pl[nt][1]);
            }
        }

        if (at.t == at.tiles - 1 || u == u_end - 1) {
            fresh = true;
            const int h = at.hc / chunks, ch = at.hc - h * chunks;
            const bool whole = t_first == 0 && at.t == at.tiles - 1;
            const long long part = (long long)w * 2 + (t_first == 0 ? 1 : 0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float sum = l[nt][e];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                    const int j = nt * 8 + (lane & 3) * 2 + e;
                    if (ch * HEADS + j >= a.group) continue;
                    const int d0 = lane >> 2;
                    if (whole) {
                        const long long row = (long long)at.b * a.hq + h * a.group + ch * HEADS + j;
                        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
                        uint16_t *dst = a.out + row * D + d0;
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            dst[ks * 16] = round16<FP16>(o[ks][nt][e] * inv);
                            dst[ks * 16 + 8] = round16<FP16>(o[ks][nt][2 + e] * inv);
                        }
                        if (d0 == 0) {
                            a.row_ml[row] = make_float2(m[nt][e], inv);
                            if (a.lse) a.lse[row] = m[nt][e] * a.scale + logf(FP16 ? sum * 0x1p-14f : sum);
                        }
                    } else {
                        float *dst = a.part_o + (part * HEADS + j) * D + d0;
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            dst[ks * 16] = o[ks][nt][e];
                            dst[ks * 16 + 8] = o[ks][nt][2 + e];
                        }
                        if (d0 == 0) a.part_ml[part * HEADS + j] = make_float2(m[nt][e], sum);
                    }
                }
        }
        at.next(first, B, HC);
    }
}

constexpr int DJ_THREADS = 256;

// Joins what several warps left of one (sequence, query head): out = sum_w f_w o_w / sum_w f_w l_w, f_w = exp(scale (m_w - max)).
// Sequences without a slot get zeros.  Also where the table's pages and the lengths are looked at.
template <bool FP16, int D, int NT>
__global__ void __launch_bounds__(DJ_THREADS) k_decode_join(const DecodeArgs a) {
    constexpr int HEADS = 8 * NT, L4 = D / 4, G = DJ_THREADS / L4;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float red[2][DJ_THREADS / 32];
    __shared__ float4 sum_o[DJ_THREADS];
    const int B = a.kv.B, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int *first = reinterpret_cast<int *>(smem), *len = first + B + 1;
    float *fac = reinterpret_cast<float *>(len + B);
    pdl_launch();
    tile_lists(a, first, len);
    pdl_wait();
    const int chunks = (a.group + HEADS - 1) / HEADS, HC = a.kv.hkv * chunks;
    const int units = first[B] * HC, workers = workers_of(a, units);
    const float c = a.scale * 1.4426950408889634f;
    for (int b = blockIdx.x; b < B; b += gridDim.x) {
        const int add = a.k_new ? 1 : 0, raw = a.kv.lens[b];
        if (tid == 0 && (raw < 0 || raw > a.kv.cap - add)) latch_error(a.status, DEV_BAD_POSITION);
        const int pages = (len[b] + a.kv.page_size - 1) / a.kv.page_size;
        bool bad = false;
        for (int i = tid; i < pages; i += DJ_THREADS)
            bad |= (unsigned)a.kv.table[(long long)b * a.kv.max_pages + i] >= (unsigned)a.kv.n_pages;
        if (bad) latch_error(a.status, DEV_BAD_PAGE);
    }
    for (int row = blockIdx.x; row < B * a.hq; row += gridDim.x) {
        const int b = row / a.hq, hq = row - b * a.hq, h = hq / a.group, g = hq - h * a.group;
        const int ch = g / HEADS, j = g - ch * HEADS, tiles = first[b + 1] - first[b];
        if (tiles == 0) {
            for (int d = tid; d < D; d += DJ_THREADS) a.out[(long long)row * D + d] = 0;
            if (tid == 0 && a.lse) a.lse[row] = -INFINITY;
            continue;
        }
        const long long u0 = (long long)first[b] * HC + (long long)(h * chunks + ch) * tiles, u1 = u0 + tiles;
        // the worker that holds unit u is the last whose first unit is not behind it
        const int w0 = (int)(((u0 + 1) * workers - 1) / units), w1 = (int)((u1 * workers - 1) / units);
        if (w0 == w1) continue;  // one warp did it all
        const int nw = w1 - w0 + 1;
        float mx = -INFINITY;
        for (int i = tid; i < nw; i += DJ_THREADS) {
            const long long part = ((long long)(w0 + i) * 2 + (i == 0)) * HEADS + j;
            mx = fmaxf(mx, a.part_ml[part].x);
        }
        for (int s = 16; s; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
        __syncthreads();  // (red, fac and sum_o of the row before have been read)
        if (lane == 0) red[0][warp] = mx;
        __syncthreads();
        mx = red[0][0];
        for (int i = 1; i < DJ_THREADS / 32; ++i) mx = fmaxf(mx, red[0][i]);
        const float mu = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f;
        for (int i = tid; i < nw; i += DJ_THREADS) {
            const long long part = ((long long)(w0 + i) * 2 + (i == 0)) * HEADS + j;
            const float2 ml = a.part_ml[part];
            const float f = ex2((ml.x - mu) * c);
            fac[i] = f;
            sum += f * ml.y;
        }
        for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        if (lane == 0) red[1][warp] = sum;
        __syncthreads();
        sum = 0.f;
        for (int i = 0; i < DJ_THREADS / 32; ++i) sum += red[1][i];
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const int d4 = tid % L4, grp = tid / L4;
#pragma unroll 4
        for (int i = grp; i < nw; i += G) {
            const long long part = ((long long)(w0 + i) * 2 + (i == 0)) * HEADS + j;
            const float4 x = *reinterpret_cast<const float4 *>(a.part_o + part * D + d4 * 4);
            const float f = fac[i];
            acc.x += f * x.x;
            acc.y += f * x.y;
            acc.z += f * x.z;
            acc.w += f * x.w;
        }
        sum_o[tid] = acc;
        __syncthreads();
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
        if (tid < L4) {
            for (int i = 1; i < G; ++i) {
                const float4 x = sum_o[i * L4 + tid];
                acc.x += x.x;
                acc.y += x.y;
                acc.z += x.z;
                acc.w += x.w;
            }
            uint2 r;
            r.x = pack2<FP16>(acc.x * inv, acc.y * inv);
            r.y = pack2<FP16>(acc.z * inv, acc.w * inv);
            *reinterpret_cast<uint2 *>(a.out + (long long)row * D + tid * 4) = r;
        }
        if (tid == 0) {
            a.row_ml[row] = make_float2(mx, inv);
            if (a.lse) a.lse[row] = mx * a.scale + logf(FP16 ? sum * 0x1p-14f : sum);
        }
    }
}

constexpr int DW_THREADS = 256;

// weights[b][h][slot] += the weights that the heads of h's group give the slot; the new token's slot starts at 0.
template <bool FP16>
__global__ void __launch_bounds__(DW_THREADS) k_decode_weights(const DecodeArgs a) {
    extern __shared__ __align__(128) uint8_t smem[];
    float2 *ml = reinterpret_cast<float2 *>(smem);
    const int h = blockIdx.x % a.kv.hkv, b = blockIdx.x / a.kv.hkv;
    const float c = a.scale * 1.4426950408889634f, shift = FP16 ? 14.f : 0.f;
    pdl_wait();
    const int n = attended(a, b);
    const long long row = (long long)b * a.hq + h * a.group;
    for (int i = threadIdx.x; i < a.group; i += DW_THREADS) ml[i] = a.row_ml[row + i];
    __syncthreads();
    float *wt = a.kv.weights + ((long long)b * a.kv.hkv + h) * a.kv.cap;
    const int fresh = a.k_new ? n - 1 : -1;
    for (int slot = blockIdx.y * DW_THREADS + threadIdx.x; slot < n; slot += gridDim.y * DW_THREADS) {
        const float *s = a.scores + row * a.score_pitch + slot;
        float sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < a.group; ++i) {
            const float mu = ml[i].x == -INFINITY ? 0.f : ml[i].x;
            sum += ex2((s[i * a.score_pitch] - mu) * c + shift) * ml[i].y;
        }
        wt[slot] = slot == fresh ? sum : wt[slot] + sum;
    }
}

template <bool FP16, int D, int NT>
cudaError_t launch(DecodeArgs &a, cudaStream_t st) {
    using S = DaShape<D>;
    const size_t lists = (2 * (size_t)a.kv.B + 1) * 4, smem = S::RING + lists;
    static thread_local int configured = -1;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && configured != dev) {
        e = cudaFuncSetAttribute(k_decode_split<FP16, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 S::RING + (2 * KV_MAX_BATCH + 1) * 4);
        if (e == cudaSuccess) configured = dev;
    }
    if (e != cudaSuccess) return e;
    const int grid = gemm_ctas() * S::CTAS;
    a.workers = std::min(grid * DA_WARPS, KV_MAX_WORKERS);
    k_decode_split<FP16, D, NT><<<grid, DA_WARPS * 32, smem, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const size_t jsmem = lists + (size_t)a.workers * 4;
    e = launch_pdl(k_decode_join<FP16, D, NT>, std::min(a.kv.B * a.hq, gemm_ctas() * 4), DJ_THREADS, jsmem, st, a);
    if (e != cudaSuccess || !a.accumulate) return e;
    cudaLaunchConfig_t cfg = {};
    const int rows = a.kv.B * a.kv.hkv;
    const long long most = (a.kv.cap + DW_THREADS - 1) / DW_THREADS;
    cfg.gridDim = dim3((unsigned)rows, (unsigned)std::max(1ll, std::min(most, (long long)(gemm_ctas() * 8 + rows - 1) / rows)));
    cfg.blockDim = dim3(DW_THREADS);
    cfg.dynamicSmemBytes = (size_t)a.group * sizeof(float2);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_decode_weights<FP16>, static_cast<const DecodeArgs>(a));
}

template <bool FP16, int D>
cudaError_t launch_d(DecodeArgs &a, cudaStream_t st) {
    return a.group <= 8 ? launch<FP16, D, 1>(a, st) : launch<FP16, D, 2>(a, st);
}

template <bool FP16>
cudaError_t launch_t(DecodeArgs &a, cudaStream_t st) {
    return a.kv.d == 64 ? launch_d<FP16, 64>(a, st) : a.kv.d == 128 ? launch_d<FP16, 128>(a, st) : launch_d<FP16, 256>(a, st);
}

}  // namespace

bool decode_plan(const KvView &kv, int hq, bool accumulate, DecodePlan *p) {
    const int group = hq / kv.hkv, heads = group <= 8 ? 8 : 16;
    size_t off = 1024;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = (off + bytes + 1023) / 1024 * 1024;
        return o;
    };
    p->part_o = take((size_t)KV_MAX_WORKERS * 2 * heads * kv.d * sizeof(float));
    p->part_ml = take((size_t)KV_MAX_WORKERS * 2 * heads * sizeof(float2));
    p->row_ml = take((size_t)kv.B * hq * sizeof(float2));
    p->score_pitch = (kv.cap + DA_SLOTS - 1) / DA_SLOTS * DA_SLOTS;
    p->scores = take(accumulate ? (size_t)kv.B * hq * p->score_pitch * sizeof(float) : 0);
    p->total = off;
    // units are counted in 32 bits
    return (long long)kv.B * ((kv.cap + DA_SLOTS - 1) / DA_SLOTS) * kv.hkv * ((group + heads - 1) / heads) < (1ll << 31);
}

cudaError_t launch_decode_attention(DecodeArgs &a, cudaStream_t st) {
    return a.fp16 ? launch_t<true>(a, st) : launch_t<false>(a, st);
}

}  // namespace pbd
