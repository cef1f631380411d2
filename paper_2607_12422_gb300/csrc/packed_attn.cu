// packed_attn.cu -- attention of packed rows: whole prompts, causal (pbd_op_prompt_attention), and drafted trees over a paged
// cache (pbd_op_tree_attention).
//
// For query head h of KV head h / group and the keys j that row i sees:
//     s_ij = q_i . k_j,   p_ij = exp(scale (s_ij - max_j s_ij)),   l_i = sum_j p_ij,   out_i = sum_j p_ij v_j / l_i
//     lse_i = scale max_j s_ij + ln l_i
// A warp takes a row and query head, its lanes parts of the head's dimensions; one pass over the keys with a running maximum.
#include <algorithm>
#include <cuda_fp16.h>

#include "packed_ops.h"

namespace pbd {

namespace {

constexpr int PA_WARPS = 8;

template <bool FP16>
__device__ __forceinline__ float widen(uint16_t x) {
    return FP16 ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}
template <bool FP16>
__device__ __forceinline__ uint16_t narrow(float x) {
    return FP16 ? __half_as_ushort(__float2half_rn(x)) : __bfloat16_as_ushort(f2bf(x));
}

__device__ __forceinline__ bool bounds_ok(const PackedArgs &a, int b, bool tree) {
    const int s = a.starts[b], e = a.starts[b + 1];
    if (s < 0 || e < s || e > a.T) return false;
    if (!tree) return true;
    const int n = e - s, len = a.kv.lens[b];
    return n <= TREE_NODES && len >= 0 && len + (long long)n <= a.kv.cap;
}

__device__ __forceinline__ int page_at(const PackedArgs &a, int b, int slot) {
    return a.kv.table[(long long)b * a.kv.max_pages + page_index(a.kv, slot)];
}
__device__ __forceinline__ long long row_at(const PackedArgs &a, int page, int slot, int h) {
    return page * a.kv.stride_page + h * a.kv.stride_head + (slot - page_index(a.kv, slot) * a.kv.page_size) * a.kv.stride_slot;
}

template <bool FP16, int D, bool TREE>
__global__ void __launch_bounds__(32 * PA_WARPS) k_rows(const __grid_constant__ PackedArgs a) {
    constexpr int PER = D / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = blockIdx.x;
    if (t == a.T) {  // what the call's status says
        int code = DEV_OK;
        for (int b = threadIdx.x; b < a.B; b += blockDim.x)
            if (!bounds_ok(a, b, TREE)) code = DEV_BAD_POSITION;
        if (!TREE && a.kv.k)
            for (int i = threadIdx.x; i < a.T; i += blockDim.x)
                if (a.slots[i] >= (long long)a.kv.n_pages * a.kv.page_size) code = DEV_BAD_PAGE;
        if (TREE)
            for (int b = 0; b < a.B; ++b) {
                if (!bounds_ok(a, b, true)) continue;
                const int s = a.starts[b], n = a.starts[b + 1] - s;
                if (n == 0) continue;
                const int pages = page_index(a.kv, a.kv.lens[b] + n - 1) + 1;
                for (int i = threadIdx.x; i < pages; i += blockDim.x)
                    if ((unsigned)a.kv.table[(long long)b * a.kv.max_pages + i] >= (unsigned)a.kv.n_pages) code = DEV_BAD_PAGE;
                for (int i = threadIdx.x; i < n && a.parents; i += blockDim.x)
                    if (a.parents[s + i] < -1 || a.parents[s + i] >= i) code = DEV_BAD_TREE;
            }
        const int c5 = __syncthreads_or(code == DEV_BAD_POSITION), c7 = __syncthreads_or(code == DEV_BAD_PAGE), c9 = __syncthreads_or(code == DEV_BAD_TREE);
        if (threadIdx.x == 0) *a.status = c5 ? DEV_BAD_POSITION : c7 ? DEV_BAD_PAGE : c9 ? DEV_BAD_TREE : DEV_OK;
        return;
    }
    int b = -1;
    for (int b0 = 0; b < 0 && b0 < a.B; b0 += 32) {
        const int x = b0 + lane;
        const unsigned m = __ballot_sync(0xffffffffu, x < a.B && a.starts[x] <= t && t < a.starts[x + 1] && bounds_ok(a, x, TREE));
        if (m) b = b0 + __ffs(m) - 1;
    }
    if (b < 0) return;
    const int start = a.starts[b], i = t - start;
    const int len = TREE ? a.kv.lens[b] : 0;
    auto parent = [&](int x) {
        if (!a.parents) return x - 1;
        const int p = a.parents[start + x];
        return p >= -1 && p < x ? p : -1;
    };
    // the new rows of a tree are in nobody's way: they are read from k and v
    uint64_t sees = 0;
    if (TREE)
        for (int x = i; x >= 0; x = parent(x)) {
            const int page = page_at(a, b, len + x);
            if ((unsigned)page < (unsigned)a.kv.n_pages) sees |= 1ull << x;
        }
    for (int h = warp; h < a.hq; h += PA_WARPS) {
        const int g = h / a.group;
        float q[PER], o[PER], m = -INFINITY, l = 0.f;
        for (int j = 0; j < PER; ++j) q[j] = widen<FP16>(a.q[t * a.q_stride + h * D + lane + 32 * j]), o[j] = 0.f;
        auto key = [&](const uint16_t *kr, const uint16_t *vr) {
            float s = 0.f;
            for (int j = 0; j < PER; ++j) s += q[j] * widen<FP16>(kr[lane + 32 * j]);
            for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            s *= a.scale;
            const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
            const float c = expf(m - base), p = expf(s - base);
            m = mn;
            l = l * c + p;
            for (int j = 0; j < PER; ++j) o[j] = o[j] * c + p * widen<FP16>(vr[lane + 32 * j]);
        };
        for (int j = 0; j < len; ++j) {
            const int page = page_at(a, b, j);
            if ((unsigned)page >= (unsigned)a.kv.n_pages) continue;
            const long long r = row_at(a, page, j, g);
            key(a.kv.k + r, a.kv.v + r);
        }
        for (int j = 0; j <= i; ++j) {
            if (TREE && !(sees >> j & 1)) continue;
            const long long r = (long long)(start + j) * a.kv_stride + g * D;
            key(a.k + r, a.v + r);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        for (int j = 0; j < PER; ++j) a.out[((long long)t * a.hq + h) * D + lane + 32 * j] = narrow<FP16>(o[j] * inv);
        if (a.lse && lane == 0) a.lse[(long long)t * a.hq + h] = m + logf(l);
    }
    if (!a.kv.k) return;
    for (int g = warp; g < a.hkv; g += PA_WARPS) {
        long long r = -1;
        if (TREE) {
            const int page = page_at(a, b, len + i);
            if ((unsigned)page < (unsigned)a.kv.n_pages) r = row_at(a, page, len + i, g);
            if (lane == 0 && r >= 0 && a.new_pos && a.kv.positions) a.kv.positions[((long long)b * a.hkv + g) * a.kv.cap + len + i] = a.new_pos[t];
        } else {
            const long long slot = a.slots[t], page = slot / a.kv.page_size;
            if (slot >= 0 && page < a.kv.n_pages)
                r = page * a.kv.stride_page + g * a.kv.stride_head + (slot - page * a.kv.page_size) * a.kv.stride_slot;
        }
        if (r < 0) continue;
        for (int j = 0; j < PER; ++j) {
            const long long src = t * a.kv_stride + g * D + lane + 32 * j;
            const_cast<uint16_t *>(a.kv.k)[r + lane + 32 * j] = a.k[src];
            const_cast<uint16_t *>(a.kv.v)[r + lane + 32 * j] = a.v[src];
        }
    }
}

template <bool TREE>
cudaError_t launch(const PackedArgs &a, cudaStream_t st) {
    auto go = [&](auto kernel) {
        kernel<<<a.T + 1, 32 * PA_WARPS, 0, st>>>(a);
        return cudaGetLastError();
    };
    if (a.fp16) return a.d == 64 ? go(k_rows<true, 64, TREE>) : a.d == 128 ? go(k_rows<true, 128, TREE>) : go(k_rows<true, 256, TREE>);
    return a.d == 64 ? go(k_rows<false, 64, TREE>) : a.d == 128 ? go(k_rows<false, 128, TREE>) : go(k_rows<false, 256, TREE>);
}

}  // namespace

cudaError_t launch_tree_attention(const PackedArgs &a, cudaStream_t st) { return launch<true>(a, st); }

}  // namespace pbd
