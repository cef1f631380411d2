// prompt_attn.cu -- causal attention over packed whole prompts (pbd_op_prompt_attention).
//
// For query head h of KV head h / group and row i of a sequence:
//     s_ij = q_i . k_j (j <= i),  p_ij = exp(scale (s_ij - max_j s_ij)),  l_i = sum_j p_ij,  out_i = sum_j p_ij v_j / l_i
// in one pass over the keys (flash.cuh).  The tensor core bounds it: 4 D operations a (row, key).
//
// A tile's 128 rows are 128 / P tokens of P heads of one KV head, P the power of two in the group (16 at most), so that
// tiles waste no rows and a block of K and V serves the whole group.  A CTA takes two tiles, of consecutive tokens (heads of 256: one), over
// blocks of 128 keys up to its last token.  While the threads of one tile turn scores into P, the tensor core works on the other's.
//
// Warps 0-7: the tiles' rows, a thread each.  Warp 8: TMA.  Warp 9: MMAs.  Warps 10 and 11 look after values of V that not all rows
// of the CTA see (those of its last one or two blocks): 0 x NaN would be NaN in rows that do not.  Rows behind the sequence's end become zero;
// of the others, infinite and NaN values do, and the first row that sees one is noted for each dimension: from that row on the
// result is NaN there.
#include <algorithm>

#include "flash.cuh"
#include "packed_ops.h"

namespace pbd {

using namespace flash;

namespace {

constexpr int PA_THREADS = 384;
constexpr int PA_MASKED = 2;  // blocks that not all rows of a CTA see, at most

template <int D>
struct PromptShape : Shape<D> {
    using S = Shape<D>;
    static constexpr int STAGES = D == 64 ? 8 : 4;
    static constexpr int SMEM = S::TILES * S::QT + STAGES * S::UNIT + 1024;
};

template <int D>
struct PromptState {
    uint64_t full[PromptShape<D>::STAGES], empty[PromptShape<D>::STAGES], q_full, s_full[2], p_full[2], o_full[2], drain;
    uint64_t v_full[PA_MASKED], v_fixed[PA_MASKED];
    uint32_t tmem;
    int abort, odd;
    int first_odd[D];  // the first row that sees an infinite or NaN value in this dimension
    int start[KV_MAX_BATCH], tiles[KV_MAX_BATCH];
};

// What a CTA works on: tokens from q0 of a sequence, heads ch * P .. of the group of KV head h.
struct PromptItem {
    int b, start, len, q0, h, ch;
};

// Items with the most keys come first: by token tile, the last ones before, then by sequence; the heads of one innermost.  A warp.
__device__ __forceinline__ bool find_item(const PackedArgs &a, const int *start, const int *tiles, int heads, int chunks, int tokens, PromptItem &it) {
    const int lane = threadIdx.x & 31;
    const int o = blockIdx.x / heads, hc = blockIdx.x - o * heads;
    // items of token tiles t and above
    auto count = [&](int t) {
        int n = 0;
        for (int b = lane; b < a.B; b += 32) n += max(tiles[b] - t, 0);
        return __reduce_add_sync(0xffffffffu, n);
    };
    int most = 0;
    for (int b = lane; b < a.B; b += 32) most = max(most, tiles[b]);
    int lo = 0, hi = __reduce_max_sync(0xffffffffu, most);  // count(hi) <= o < count(lo)
    if (o >= count(0)) return false;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (count(mid) <= o)
            hi = mid;
        else
            lo = mid;
    }
    int r = o - count(lo + 1);  // which of the sequences with a token tile lo
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane;
        const unsigned m = __ballot_sync(0xffffffffu, b < a.B && tiles[b] > lo);
        const int n = __popc(m);
        if (r < n) {
            it.b = b0 + (int)__fns(m, 0, r + 1);
            break;
        }
        r -= n;
    }
    it.start = start[it.b];
    it.len = a.starts[it.b + 1] - it.start;
    it.q0 = lo * tokens;
    it.h = hc / chunks;
    it.ch = hc - it.h * chunks;
    return true;
}

// The call's status, by two warps: bounds and slots.
__device__ __forceinline__ void check_call(const PackedArgs &a, int t) {
    int code = DEV_OK;
    for (int b = t; b < a.B; b += 64) {
        const int s = a.starts[b], e = a.starts[b + 1];
        if (s < 0 || e < s || e > a.T) code = DEV_BAD_POSITION;
    }
    if (a.kv.k) {
        const long long slots = (long long)a.kv.n_pages * a.kv.page_size;
#pragma unroll 8
        for (int i = t; i < a.T; i += 64)
            if (a.slots[i] >= slots) code = code ? code : DEV_BAD_PAGE;
    }
    // (one of the two codes where both occur)
    if (code != DEV_OK) latch_error(a.status, code);
}

// K and V of `n` tokens from t0 on (of the packed rows) into the cache: 128 threads.
template <int D>
__device__ __forceinline__ void store_rows(const PackedArgs &a, int t0, int n, int h, int t) {
    constexpr int CPR = D / 8, U = 8;  // 16-byte pieces of a row; loads on their way together
    const long long slots = (long long)a.kv.n_pages * a.kv.page_size;
    for (int i0 = t; i0 < n * CPR; i0 += U * 128) {
        uint4 k[U], v[U];
        long long slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * 128, r = i / CPR, c = i % CPR;
            slot[u] = -1;
            if (i >= n * CPR) continue;
            slot[u] = a.slots[t0 + r];
            const long long src = (long long)(t0 + r) * a.kv_stride + h * D + c * 8;
            k[u] = *reinterpret_cast<const uint4 *>(a.k + src);
            v[u] = *reinterpret_cast<const uint4 *>(a.v + src);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0 || slot[u] >= slots) continue;
            const int c = (i0 + u * 128) % CPR;
            const long long page = slot[u] >> 32 ? slot[u] / a.kv.page_size : (long long)((uint32_t)slot[u] / (uint32_t)a.kv.page_size);
            const long long dst = page * a.kv.stride_page + h * a.kv.stride_head + (slot[u] - page * a.kv.page_size) * a.kv.stride_slot + c * 8;
            *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.k) + dst) = k[u];
            *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.v) + dst) = v[u];
        }
    }
}

template <int D, bool FP16>
__global__ void __launch_bounds__(PA_THREADS, 1)
    k_prompt(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
             const __grid_constant__ PackedArgs a, int log_p) {
    using L = PromptShape<D>;
    constexpr int TILES = L::TILES, UNITS = L::UNITS, STAGES = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sq = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *ring = sq + TILES * L::QT;
    __shared__ PromptState<D> S;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int P = 1 << log_p, tile_tokens = ROWS >> log_p, tokens = TILES * tile_tokens;
    const int chunks = a.group >> log_p, heads = a.hkv * chunks;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&S.full[i], 1);
            mbar_init(&S.empty[i], 1);
        }
        mbar_init(&S.q_full, 1);
        mbar_init(&S.drain, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&S.s_full[i], 1);
            mbar_init(&S.p_full[i], 4);
            mbar_init(&S.o_full[i], 1);
        }
        for (int i = 0; i < PA_MASKED; ++i) {
            mbar_init(&S.v_full[i], 1);
            mbar_init(&S.v_fixed[i], 2);
        }
        S.abort = S.odd = 0;
        fence_mbarrier_init();
        prefetch_tensormap(&qmap);
        prefetch_tensormap(&kmap);
        prefetch_tensormap(&vmap);
        if (blockIdx.x == 0) *a.status = DEV_OK;  // (before any thread of this CTA reports; a wait runs out a second later)
    }
    for (int i = threadIdx.x; i < D; i += PA_THREADS) S.first_odd[i] = 0x7fffffff;
    for (int b = threadIdx.x; b < a.B; b += PA_THREADS) {
        const int s = a.starts[b], e = a.starts[b + 1];
        S.start[b] = s;
        S.tiles[b] = s < 0 || e < s || e > a.T ? 0 : (e - s + tokens - 1) / tokens;
    }
    if (warp == 8) tmem_alloc(&S.tmem, TM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S.tmem;
    PromptItem it = {};
    const bool has = find_item(a, S.start, S.tiles, heads, chunks, tokens, it);  // (the same in every warp)
    // a tile's blocks, and those that all rows see
    auto blocks = [&](int tile) {
        const int first = it.q0 + tile * tile_tokens;
        return !has || first >= it.len ? 0 : min(first + tile_tokens - 1, it.len - 1) / KEYS + 1;
    };
    const int nb0 = blocks(0), nb1 = TILES == 2 ? blocks(1) : 0, nmax = max(nb0, nb1), masked = has ? (it.q0 + 1) / KEYS : 0;

    // registers: of the launch's 3 x 128 x 168 the last warpgroup keeps 128 x 72, the others take 128 x 216 each
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 8) {
            if (has && elect_one()) {
                // ---- TMA: the queries, then K 0, V 0, K 1, V 1, ...
                int issued = 0;
                mbar_arrive_expect_tx(&S.q_full, (uint32_t)(TILES * L::QT));
                for (int i = 0; i < TILES; ++i)
                    for (int c = 0; c < D / 64; ++c)
                        tma_load_4d(sq + i * L::QT + c * SUB, &qmap, c * 64, 0, it.h * chunks + it.ch, it.start + it.q0 + i * tile_tokens, &S.q_full);
                bool ok = true;
                for (int j = 0; ok && j < 2 * nmax; ++j)
                    for (int u = 0; u < UNITS; ++u) {
                        const int slot = issued % STAGES;
                        if (!mbar_wait(&S.empty[slot], ((issued / STAGES) & 1) ^ 1, a.status, DEV_TIMEOUT_SLOT, &S.abort)) {
                            ok = false;
                            break;
                        }
                        ++issued;
                        const int kb = j >> 1;
                        uint64_t *bar = &S.full[slot];
                        if ((j & 1) && kb >= masked) {  // V that is looked at first
                            mbarrier_arrive_one(bar);
                            bar = &S.v_full[kb - masked];
                            if (u == 0) mbar_arrive_expect_tx(bar, (uint32_t)(UNITS * L::UNIT));
                        } else {
                            mbar_arrive_expect_tx(bar, (uint32_t)L::UNIT);
                        }
                        for (int c = 0; c < L::DU / 64; ++c)
                            tma_load_3d(ring + slot * L::UNIT + c * SUB, (j & 1) ? &vmap : &kmap, u * L::DU + c * 64, it.h, it.start + kb * KEYS, bar);
                    }
                if (*(volatile int *)&S.abort) {  // error path: the copies in flight get a bounded chance to land
                    bool landed = mbar_wait(&S.q_full, 0, nullptr, 0, nullptr);
                    for (int h = issued > STAGES ? issued - STAGES : 0; landed && h < issued; ++h)
                        landed = mbar_wait(&S.full[h % STAGES], (h / STAGES) & 1, nullptr, 0, nullptr);
                    for (int k = 0; landed && k < PA_MASKED; ++k)
                        if (issued > ((masked + k) * 2 + 2) * UNITS - 1) landed = mbar_wait(&S.v_full[k], 0, nullptr, 0, nullptr);
                }
            }
        } else if (warp == 9) {
            if (has && elect_one()) {
                // ---- MMAs: for every block, tile after tile, O += P V of the block before, then S
                int pos = 0;
                bool ok = mbar_wait(&S.q_full, 0, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                auto landed = [&](int at) {
                    ok = ok && mbar_wait(&S.full[at % STAGES], (at / STAGES) & 1, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                };
                for (int j = 0; ok && j <= nmax; ++j) {
                    const int vp = pos, kp = pos + (j ? UNITS : 0);
                    pos = kp + UNITS;
                    for (int i = 0; ok && i < TILES; ++i) {
                        const int nb = i ? nb1 : nb0;
                        if (j > 0 && j <= nb) {
                            ok = mbar_wait(&S.p_full[i], (j - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
                            // (the last block's keys behind the sequence's end are not multiplied, to 16)
                            const int steps = min(KEYS, it.len - (j - 1) * KEYS + 15) / 16;
                            for (int u = 0; ok && u < UNITS; ++u) {
                                landed(vp + u);
                                if (j - 1 >= masked) ok = ok && mbar_wait(&S.v_fixed[j - 1 - masked], 0, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                                if (!ok) break;
                                tc_fence_after();
                                mma_values<D, FP16>(tmem + TM_O + i * D, tmem + i * KEYS, ring + ((vp + u) % STAGES) * L::UNIT, u, steps, j == 1);
                            }
                            if (ok && j == nb) mma_commit(&S.o_full[i]);
                        }
                        if (ok && j > 0 && i == TILES - 1)
                            for (int u = 0; u < UNITS; ++u) {
                                landed(vp + u);
                                mma_commit(&S.empty[(vp + u) % STAGES]);
                            }
                        if (ok && j < nb) {
                            for (int u = 0; ok && u < UNITS; ++u) {
                                landed(kp + u);
                                if (!ok) break;
                                tc_fence_after();
                                mma_scores<D, FP16>(tmem + i * KEYS, sq + i * L::QT, ring + ((kp + u) % STAGES) * L::UNIT, u);
                            }
                            if (ok) mma_commit(&S.s_full[i]);
                        }
                    }
                    if (ok && j < nmax)
                        for (int u = 0; u < UNITS; ++u) mma_commit(&S.empty[(kp + u) % STAGES]);
                }
                if (!ok) {  // every MMA issued completes before TMEM is released
                    mma_commit(&S.drain);
                    mbar_wait(&S.drain, 0, nullptr, 0, nullptr);
                }
            }
        } else {
            const int t = (warp - 10) * 32 + lane;
            // ---- V of the blocks that not all rows see
            bool ok = true;
            for (int j = masked; ok && j < nmax; ++j) {
                ok = mbar_wait(&S.v_full[j - masked], 0, a.status, DEV_TIMEOUT_LOAD, &S.abort);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                for (int u = 0; u < UNITS; ++u) {
                    const int slot = ((2 * j + 1) * UNITS + u) % STAGES;
                    const uint32_t at = smem_u32(ring + slot * L::UNIT);
#pragma unroll 4
                    for (int i = t; i < L::UNIT / 16; i += 64) {
                        const int r = (i >> 3) & 127, key = j * KEYS + r;
                        uint4 x = ld_shared_u4(at + i * 16);
                        if (key >= it.len) {
                            if (key < ((it.len + 15) & ~15)) st_shared_u4(at + i * 16, make_uint4(0, 0, 0, 0));
                            continue;
                        }
                        uint32_t w[4] = {x.x, x.y, x.z, x.w};
                        if (!(odd_halves<FP16>(w[0]) | odd_halves<FP16>(w[1]) | odd_halves<FP16>(w[2]) | odd_halves<FP16>(w[3]))) continue;
                        const int d0 = u * L::DU + (i >> 10) * 64 + (((i & 7) ^ (r & 7)) << 3);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t half = 0xffffu << (16 * (e & 1));
                            if (odd_halves<FP16>(w[e >> 1]) & half) {
                                w[e >> 1] &= ~half;
                                atomicMin(&S.first_odd[d0 + e], key);
                            }
                        }
                        st_shared_u4(at + i * 16, make_uint4(w[0], w[1], w[2], w[3]));
                        S.odd = 1;
                    }
                }
                fence_proxy_async_shared();
                __syncwarp();
                if (lane == 0) mbarrier_arrive_one(&S.v_fixed[j - masked]);
            }
            if (blockIdx.x == 0) check_call(a, t);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- softmax: thread r of tile i the row of token first + r / P, head r % P
        const int i = warp >> 2, w = warp & 3, nb = i ? nb1 : nb0, row = w * 32 + lane;
        const int first = it.q0 + i * tile_tokens, token = first + (row >> log_p);
        if (nb > 0) {
            if (a.kv.k && it.ch == 0) store_rows<D>(a, it.start + first, min(tile_tokens, it.len - first), it.h, row);
            const uint32_t lanes = (uint32_t)(w * 32) << 16, ts = tmem + lanes + i * KEYS, to = tmem + lanes + TM_O + i * D;
            const float c = a.scale * 1.4426950408889634f;
            Row r;
            bool ok = true;
            for (int j = 0; j < nb; ++j) {
                ok = mbar_wait(&S.s_full[i], j & 1, a.status, DEV_TIMEOUT_MMA, &S.abort);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                tc_fence_after();
                uint32_t s[KEYS];
#pragma unroll
                for (int x = 0; x < KEYS; x += 32) tmem_ld_32cols(ts + x, *reinterpret_cast<uint32_t(*)[32]>(&s[x]));
                tmem_ld_wait();
                if (j * KEYS + KEYS - 1 > first) {
                    const int last = token - j * KEYS;
#pragma unroll
                    for (int x = 0; x < KEYS; ++x)
                        if (x > last) s[x] = __float_as_uint(-INFINITY);
                }
                softmax_block<D, FP16>(r, s, c, j == 0, ts, to);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive_one(&S.p_full[i]);
            }
            if (ok) ok = mbar_wait(&S.o_full[i], 0, a.status, DEV_TIMEOUT_MMA, &S.abort);
            for (int k = 0; ok && masked + k < nmax; ++k) ok = mbar_wait(&S.v_fixed[k], 0, a.status, DEV_TIMEOUT_LOAD, &S.abort);
            if (__all_sync(0xffffffffu, ok)) {
                // rows go out through the queries' place (all scores of the tile are there), a row's pieces by neighbouring lanes
                tc_fence_after();
                const float f = row_factor(r);
                const bool odd = *(volatile int *)&S.odd;
                const uint32_t stage = smem_u32(sq + i * L::QT) + w * 32 * (D * 2);
#pragma unroll 1
                for (int x = 0; x < D; x += 32) {
                    uint32_t o[32];
                    tmem_ld_32cols(to + x, o);
                    tmem_ld_wait();
                    if (odd)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (S.first_odd[x + e] <= token) o[e] = 0x7fffffffu;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t v[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            v[y] = pack16<FP16>(__uint_as_float(o[e + 2 * y]) * f, __uint_as_float(o[e + 2 * y + 1]) * f);
                        st_shared_u4(stage + lane * (D * 2) + ((((x + e) >> 3) ^ (lane & 7)) << 4), make_uint4(v[0], v[1], v[2], v[3]));
                    }
                }
                __syncwarp();
                constexpr int CPR = D / 8, RPI = 32 / CPR;  // pieces of a row, rows of a step
                const int piece = lane % CPR, head = it.h * a.group + it.ch * P;
#pragma unroll 4
                for (int x = 0; x < 32; x += RPI) {
                    const int rr = x + lane / CPR, tk = first + ((w * 32 + rr) >> log_p);
                    if (tk >= it.len) continue;
                    const uint4 v = ld_shared_u4(stage + rr * (D * 2) + ((piece ^ (rr & 7)) << 4));
                    *reinterpret_cast<uint4 *>(a.out + ((long long)(it.start + tk) * a.hq + head + ((w * 32 + rr) & (P - 1))) * D + piece * 8) = v;
                }
                if (a.lse && token < it.len)
                    a.lse[(long long)(it.start + token) * a.hq + head + (row & (P - 1))] = row_lse<FP16>(r, a.scale);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, TM_COLS);
}

template <int D, bool FP16>
cudaError_t launch(const PackedArgs &a, cudaStream_t st) {
    using L = PromptShape<D>;
    static_assert(L::SMEM + sizeof(PromptState<D>) <= 227 * 1024, "shared memory");
    const cudaError_t e = cudaFuncSetAttribute(k_prompt<D, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
    if (e != cudaSuccess) return e;
    int log_p = 0;
    while (log_p < 4 && a.group % (2 << log_p) == 0) ++log_p;
    const int P = 1 << log_p, tokens = L::TILES * (ROWS / P), heads = a.hq / P;
    const long long tiles = std::min<long long>(a.T / tokens + a.B, a.T), grid = tiles * heads;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    CUtensorMap qm, km, vm;
    const uint64_t qs = (uint64_t)a.q_stride * 2, ks = (uint64_t)a.kv_stride * 2;
    const uint64_t qd[4] = {(uint64_t)D, (uint64_t)P, (uint64_t)heads, (uint64_t)a.T}, qst[3] = {D * 2, (uint64_t)P * D * 2, qs};
    const uint32_t qb[4] = {64, (uint32_t)P, 1, (uint32_t)(ROWS / P)};
    const uint64_t kd[3] = {(uint64_t)D, (uint64_t)a.hkv, (uint64_t)a.T}, kst[2] = {D * 2, ks};
    const uint32_t kb[3] = {64, 1, KEYS};
    if (!encode_map_16(&qm, a.q, 4, qd, qst, qb) || !encode_map_16(&km, a.k, 3, kd, kst, kb) || !encode_map_16(&vm, a.v, 3, kd, kst, kb))
        return cudaErrorInvalidValue;
    k_prompt<D, FP16><<<(unsigned)grid, PA_THREADS, L::SMEM, st>>>(qm, km, vm, a, log_p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_prompt_attention(const PackedArgs &a, cudaStream_t st) {
    if (a.fp16) return a.d == 64 ? launch<64, true>(a, st) : a.d == 128 ? launch<128, true>(a, st) : launch<256, true>(a, st);
    return a.d == 64 ? launch<64, false>(a, st) : a.d == 128 ? launch<128, false>(a, st) : launch<256, false>(a, st);
}

}  // namespace pbd
