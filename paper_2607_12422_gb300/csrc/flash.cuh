// flash.cuh -- what the tensor-core attention kernels of packed rows (prompt_attn.cu, tree_attn.cu) share: one pass over blocks
// of 128 keys for tiles of 128 rows, with a running maximum and sum a row.
//
//     S = Q K^T (tcgen05.mma from shared memory), P = 2^(c S - c m) (a thread a row, from tensor memory and back),
//     O += P V (P as the A operand in tensor memory)
//
// Tensor memory, 512 columns: S of tile i at 128 i, P over the first half of the S that it came from, O of tile i at 256 + D i.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace pbd {
namespace flash {

constexpr int ROWS = 128, KEYS = 128;  // of a tile, of a block
constexpr int SUB = 128 * 128;         // bytes of 128 rows x 64 dims in the 128-byte swizzle
// log2 of factors: P may grow so far beyond 1 before O is rescaled; P in fp16 is held so much larger, so that what is
// far below the maximum keeps its bits (2^14 at most)
constexpr float SLACK = 4.f, FP16_SHIFT = 10.f;
constexpr uint32_t TM_O = 256, TM_COLS = 512;

template <int D>
struct Shape {
    static constexpr int TILES = D == 256 ? 1 : 2;  // of a CTA: as many as tensor memory holds
    static constexpr int DU = D < 128 ? D : 128;    // dims of a ring unit
    static constexpr int UNITS = D / DU;            // of a block of K or V
    static constexpr int UNIT = DU / 64 * SUB;      // bytes
    static constexpr int QT = D / 64 * SUB;         // of a tile of queries
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (FP16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    return pack_bf162(lo, hi);
}

// Bits 15 and 31: whether the halves of w are infinite or NaN (exponents of all ones carry into them).
template <bool FP16>
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {
    return FP16 ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// instruction descriptors: 128 x N, bf16 or fp16 operands
template <bool FP16>
__host__ __device__ constexpr uint32_t idesc(int N) {
    return FP16 ? idesc_bf16_f32(128, N) & ~((1u << 7) | (1u << 10)) : idesc_bf16_f32(128, N);
}

// S of one tile from one ring unit of K (dims u * DU of them); issued by one thread.
template <int D, bool FP16>
__device__ __forceinline__ void mma_scores(uint32_t s, const uint8_t *q, const uint8_t *k, int u) {
    using L = Shape<D>;
    const uint64_t qd = sw128_kmajor_desc(q + u * L::UNIT), kd = sw128_kmajor_desc(k);
#pragma unroll
    for (int ks = 0; ks < L::DU / 16; ++ks) {
        const uint64_t off = (uint64_t)((ks >> 2) * (SUB / 16) + 2 * (ks & 3));
        mma_bf16_ss(s, qd + off, kd + off, idesc<FP16>(KEYS), (u | ks) != 0);
    }
}
// O of one tile += P V of one ring unit of V, the first `steps` 16 keys.
template <int D, bool FP16>
__device__ __forceinline__ void mma_values(uint32_t o, uint32_t p, const uint8_t *v, int u, int steps, bool first) {
    using L = Shape<D>;
    const uint64_t vd = sw128_mnmajor_desc(v, SUB);
#pragma unroll
    for (int ks = 0; ks < KEYS / 16; ++ks)
        if (ks < steps) mma_bf16_ts(o + u * L::DU, p + 8 * ks, vd + (uint64_t)(ks * (16 * 128 / 16)), idesc<FP16>(L::DU) | IDESC_B_MN, !first || ks != 0);
}

// One row's softmax: a thread's state.
struct Row {
    float m, l;  // largest score so far (as far as it has been followed), sum of P
};

// The scores s of one block, masked ones -inf, become P in tensor memory at `tp`; O at `to` is rescaled where the maximum has moved
// on.  c: the factor to exponents of 2.  Whole warp.
template <int D, bool FP16>
__device__ __forceinline__ void softmax_block(Row &r, uint32_t (&s)[KEYS], float c, bool first, uint32_t tp, uint32_t to) {
    float mx[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) mx[i] = fmaxf(__uint_as_float(s[i]), __uint_as_float(s[i + 4]));
#pragma unroll
    for (int i = 8; i < KEYS; i += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) mx[j] = fmaxf(mx[j], fmaxf(__uint_as_float(s[i + j]), __uint_as_float(s[i + j + 4])));
    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    if (first) {
        r.m = top;
        r.l = 0.f;
    } else {
        const float m = fmaxf(r.m, top);
        if (__any_sync(0xffffffffu, (m - r.m) * c > SLACK)) {
            const float f = m == r.m ? 1.f : ex2((r.m - m) * c);
            r.m = m;
            r.l *= f;
#pragma unroll 1
            for (int i = 0; i < D; i += 32) {
                uint32_t o[32];
                tmem_ld_32cols(to + i, o);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tmem_st_32cols(to + i, o);
            }
            tmem_st_wait();
        }
    }
    const float base = (r.m == -INFINITY ? 0.f : -r.m * c) + (FP16 ? FP16_SHIFT : 0.f);
    const F2 c2 = f2(c, c), b2 = f2(base, base);
    F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
    for (int i = 0; i < KEYS; i += 32) {
        uint32_t p[16];
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float2 x = unpack2(fma2(f2(__uint_as_float(s[i + j]), __uint_as_float(s[i + j + 1])), c2, b2));
            const float e0 = ex2(x.x), e1 = ex2(x.y);
            sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], f2(e0, e1));
            p[j >> 1] = pack16<FP16>(e0, e1);
        }
        tmem_st_16cols(tp + i / 2, p);
    }
    const float2 t = unpack2(add2(sum[0], sum[1]));
    r.l += t.x + t.y;
    tmem_st_wait();
}

// ln of the sum of exp(scale s) and the factor of O.
template <bool FP16>
__device__ __forceinline__ float row_lse(const Row &r, float scale) {
    return r.l == 0.f ? -INFINITY : r.m * scale + (logf(r.l) - (FP16 ? FP16_SHIFT * 0.69314718055994531f : 0.f));
}
__device__ __forceinline__ float row_factor(const Row &r) { return r.l == 0.f ? 0.f : 1.f / r.l; }

}  // namespace flash
}  // namespace pbd
