// flash.cuh -- what the tensor-core attention kernels of packed rows (prompt_attn.cu, tree_attn.cu) share: one pass over blocks
// of 128 keys for tiles of 128 rows, with a running maximum and sum a row.
//
//     S = Q K^T (tcgen05.mma from shared memory), P = 2^(c S - c m) (from tensor memory and back), O += P V (P as the A operand in
//     tensor memory)
//
// Two threads share a row, in warps w and w + 4 of a tile's eight: each takes 64 of a block's keys and half of the row's outputs.  P is
// made with the maximum m of the blocks before, which both know; only if the block's own is above m by more than SLACK do the two
// exchange it and rescale O.  P comes in two parts (32 keys of each thread), so that P V begins while the second is made.
// (One thread a row and P in one part: 1450 cycles from scores to P, during which this tile's MMAs wait; the MMAs of a tile and block
// take 1072.)
//
// P is rounded to one 16-bit value a key for P V: of a sum of p_j v_j each term is off by half a step at most, and outputs by 2.0e-3 to 2.3e-3 of their
// norm in bf16 (1.6e-3 is their own rounding alone), 2.1e-4 to 2.4e-4 in fp16 (2.0e-4).  A second 16-bit part of P, as attention of one token over a paged
// cache has it, makes P V twice as long and rows' work longer by as many registers as they do not have: 64 nodes behind 131071 slots 187 us instead of
// 106, 64 ragged trees of heads of 64 100 instead of 71, 17 nodes behind 512 slots 20 instead of 15.
//
// Tensor memory, 512 columns: S at 128 i, P over the S that it came from (keys 0-63 in columns 0-31, keys 64-127 in columns 64-95, so that
// no thread writes where another reads), O of tile i at 256 + D i.  With two tiles S i is tile i's: S of a tile's next block
// follows P V of this one, and the tensor core has the other tile's while P is made.  With one tile the two take turns: S of the next block
// goes before P V of this one.
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
constexpr int ROW_WARPS = 16;          // two tiles' rows
constexpr int THREADS = 32 * ROW_WARPS + 128;
// registers: the launch has 5 x 128 x 96; the rows' four warpgroups take 104, the last one keeps 64
constexpr int ROW_REGS = 104, OTHER_REGS = 64;
static_assert(4 * ROW_REGS + OTHER_REGS <= 5 * 96, "registers");

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

__device__ __forceinline__ float max3(float x, float y, float z) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
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

// Where the 64-dim halves of a ring unit lie: SUB apart, each with its 128 rows, or beside one another, eight rows at a time (pages'
// rows come so in half as many copies).
template <int D, bool BESIDE>
struct Layout {
    static constexpr int HALF = BESIDE ? 1024 : SUB;                            // bytes to the next 64 dims
    static constexpr int EIGHT = BESIDE ? Shape<D>::DU / 64 * 1024 : 1024;      // to the next eight rows
    // row r, 16-byte piece p of it
    static __device__ __forceinline__ uint32_t at(int r, int p) { return (uint32_t)((p >> 3) * HALF + (r >> 3) * EIGHT + (r & 7) * 128 + (((p & 7) ^ (r & 7)) << 4)); }
};

// S of one tile from one ring unit of K (dims u * DU of them); issued by one thread.
template <int D, bool FP16, bool BESIDE = false>
__device__ __forceinline__ void mma_scores(uint32_t s, const uint8_t *q, const uint8_t *k, int u) {
    using L = Shape<D>;
    using Y = Layout<D, BESIDE>;
    const uint64_t qd = sw128_kmajor_desc(q + u * L::UNIT), kd = sw128_desc(k, 16, Y::EIGHT);
#pragma unroll
    for (int ks = 0; ks < L::DU / 16; ++ks)
        mma_bf16_ss(s, qd + (uint64_t)((ks >> 2) * (SUB / 16) + 2 * (ks & 3)), kd + (uint64_t)((ks >> 2) * (Y::HALF / 16) + 2 * (ks & 3)), idesc<FP16>(KEYS),
                    (u | ks) != 0);
}
// O of one tile += P V of one ring unit of V, one part of P (keys 0-31 and 64-95, or 32-63 and 96-127), of the first `steps` 16 keys.
template <int D, bool FP16, bool BESIDE = false>
__device__ __forceinline__ void mma_values(uint32_t o, uint32_t p, const uint8_t *v, int u, int part, int steps, bool first) {
    using L = Shape<D>;
    using Y = Layout<D, BESIDE>;
    const uint64_t vd = sw128_desc(v, Y::HALF, Y::EIGHT);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int ks = (x >> 1) * 4 + part * 2 + (x & 1);
        if (ks < steps)
            mma_bf16_ts(o + u * L::DU, p + (ks >> 2) * 64 + (ks & 3) * 8, vd + (uint64_t)(ks * (2 * Y::EIGHT / 16)), idesc<FP16>(L::DU) | IDESC_B_MN,
                        !first || part != 0 || x != 0);
    }
}

// The ring's order, in blocks' K and V of a pass over nb blocks: K 0, V 0, K 1, V 1 .. for two tiles, K 0, K 1, V 0, K 2, V 1 ..
// for one.
__device__ __forceinline__ int k_place(int j, bool two) { return two || j == 0 ? 2 * j : 2 * j - 1; }
__device__ __forceinline__ int v_place(int j, int nb, bool two) { return two ? 2 * j + 1 : min(2 * j + 2, 2 * nb - 1); }
// Block at place n, negative (one's complement) for V.
__device__ __forceinline__ int at_place(int n, int nb, bool two) {
    if (two) return n & 1 ? ~(n >> 1) : n >> 1;
    if (n == 0) return 0;
    return n & 1 ? (n + 1 < 2 * nb ? (n + 1) >> 1 : ~(nb - 1)) : ~(n / 2 - 1);
}

// Whether any of the two warps that share 32 rows says so.  (Named barriers 1-8.  Every warp comes to every one of them, after waits that
// have a limit.)
__device__ __forceinline__ bool pair_any(int id, bool p) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred q, r;\n\tsetp.ne.u32 q, %2, 0;\n\tbarrier.cta.red.or.pred r, %1, 64, q;\n\tselp.u32 %0, 1, 0, r;\n\t}"
        : "=r"(r)
        : "r"(id), "r"((uint32_t)p)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ void pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }

// 32 bytes to global memory, a whole sector.
__device__ __forceinline__ void st_global_32(void *p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
// This thread's half of a finished row, in tensor memory at o_at, f its factor, to `out` (wide: 32-byte aligned, else 16); with
// careful, drop(d): whether dimension d of the half is NaN.  Returns whether a value is not finite.
template <int D, bool FP16, typename Drop>
__device__ __forceinline__ bool store_half(uint32_t o_at, float f, uint16_t *out, bool real, bool wide, bool careful, Drop &&drop) {
    uint32_t odd = 0;
#pragma unroll 1
    for (int x = 0; x < D / 2; x += 16) {
        uint32_t o[16], v[8];
        tmem_ld_16cols(o_at + x, o);
        tmem_ld_wait();
        if (careful)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (drop(x + e)) o[e] = 0x7fffffffu;
        if (!real) continue;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
            v[y] = pack16<FP16>(__uint_as_float(o[2 * y]) * f, __uint_as_float(o[2 * y + 1]) * f);
            odd |= odd_halves<FP16>(v[y]);
        }
        if (wide) {
            st_global_32(out + x, v);
        } else {
            *reinterpret_cast<uint4 *>(out + x) = make_uint4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<uint4 *>(out + x + 8) = make_uint4(v[4], v[5], v[6], v[7]);
        }
    }
    return odd != 0;
}

// A thread's half of a row.
struct Row {
    float m, l;  // largest score so far (as far as it has been followed; the row's), sum of P (of this half)
};

// The scores s of this half of a block, masked ones -inf, become P at tp.  ok: whether they are there at all; false if not for both
// threads.  to: this thread's half of O; places: the tile's maxima [2][128] in shared memory; c: the factor to exponents of 2.
// o_ready(): waits until O has all blocks before; there(part): this warp's P of a part is there.
template <int D, bool FP16, typename Ready, typename There>
__device__ __forceinline__ bool softmax_half(Row &r, const uint32_t (&s)[64], bool ok, float c, bool first, uint32_t tp, uint32_t to, int id, float *places,
                                             int half, int row, Ready &&o_ready, There &&there) {
    const F2 c2 = f2(c, c);
    F2 b2, sum[2];
    uint32_t p[16];
    auto make = [&](int part) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float2 x = unpack2(fma2(f2(__uint_as_float(s[32 * part + j]), __uint_as_float(s[32 * part + j + 1])), c2, b2));
            const float e0 = ex2(x.x), e1 = ex2(x.y);
            sum[(j >> 1) & 1] = j < 4 && part == 0 ? f2(e0, e1) : add2(sum[(j >> 1) & 1], f2(e0, e1));
            p[j >> 1] = pack16<FP16>(e0, e1);
        }
    };
    // the first part with the maximum so far, while the block's is looked for; once more if that was too low
#pragma unroll 1
    for (bool done = false;; done = true) {
        const float base = (r.m == -INFINITY ? 0.f : -r.m * c) + (FP16 ? FP16_SHIFT : 0.f);
        b2 = f2(base, base);
        make(0);
        if (done) break;
        float mx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[i] = max3(__uint_as_float(s[i]), __uint_as_float(s[i + 4]), __uint_as_float(s[i + 8]));
#pragma unroll
        for (int i = 12; i + 8 <= 64; i += 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx[j] = max3(mx[j], __uint_as_float(s[i + j]), __uint_as_float(s[i + j + 4]));
#pragma unroll
        for (int j = 0; j < 4; ++j) mx[j] = fmaxf(mx[j], __uint_as_float(s[60 + j]));
        const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        if (!pair_any(id, !ok || first || (top - r.m) * c > SLACK)) break;
        if (pair_any(id, !ok)) return false;
        places[half * ROWS + row] = top;
        pair_sync(id);
        const float both = fmaxf(top, places[(half ^ 1) * ROWS + row]);
        if (first) {
            r.m = both;
            r.l = 0.f;
        } else {
            const float m = fmaxf(r.m, both), f = m == r.m ? 1.f : ex2((r.m - m) * c);
            if (pair_any(id, !o_ready())) return false;
            r.m = m;
            r.l *= f;
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < D / 2; i += 16) {
                uint32_t o[16];
                tmem_ld_16cols(to + i, o);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tmem_st_16cols(to + i, o);
            }
        }
    }
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        if (part) make(1);
        tmem_st_16cols(tp + 16 * part, p);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        there(part);
    }
    const float2 t = unpack2(add2(sum[0], sum[1]));
    r.l += t.x + t.y;
    return true;
}

// ln of the sum of exp(scale s), and the factor of O; of the whole row.
template <bool FP16>
__device__ __forceinline__ float row_lse(const Row &r, float scale) {
    return r.l == 0.f ? -INFINITY : r.m * scale + (logf(r.l) - (FP16 ? FP16_SHIFT * 0.69314718055994531f : 0.f));
}
__device__ __forceinline__ float row_factor(const Row &r) { return r.l == 0.f ? 0.f : 1.f / r.l; }

}  // namespace flash
}  // namespace pbd
