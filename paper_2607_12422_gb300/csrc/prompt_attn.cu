// prompt_attn.cu -- causal attention over packed whole prompts (pbd_op_prompt_attention).
//
// For query head h of KV head h / group and row i of a sequence:
//     s_ij = q_i . k_j (j <= i),  p_ij = exp(scale (s_ij - max_j s_ij)),  l_i = sum_j p_ij,  out_i = sum_j p_ij v_j / l_i
// in one pass over the keys (flash.cuh).  The tensor core bounds it: 4 D operations a (row, key).
//
// A tile's 128 rows are 128 / P tokens of P heads of one KV head, P a divisor of the group for which few rows are left over, so that
// a block of K and V serves the whole group and short sequences fill tiles.  A CTA takes two tiles, of consecutive tokens (heads of 256: one),
// over blocks of 128 keys up to its last token.
//
// Each CTA works on a list of such items, with its tensor core on the next one's first blocks while the rows of one leave.
//
// 0 x NaN is NaN: an infinite or NaN value of V among the keys that a row's mask hides would reach it (and so would the rows of
// the packed neighbour in a sequence's last block).  Looking for such values first costs 4000 cycles an item.  Instead the rows look at
// their results, and an item with one that is not finite is done again, carefully: in the one or two blocks that not all of its rows see,
// rows of V behind the sequence's end become zero, infinite and NaN values too, and the first row that sees one is noted for each dimension; from
// that row on the result is NaN there.
//
// 16384 tokens, 16 heads of 128 on 8 KV heads, stored: 680-727 us, 1.5 to 1.6 PFLOP/s, the tensor core busy 70 % of the time and waiting for the chain
// scores, softmax, P V of two tiles (1400 cycles a tile and block, 1050 of them products).  Eight ragged prompts of 420 to 1757: 54 us, 36 blocks of a tile a
// CTA on average and 44 in the fullest; 32 ragged ones, groups of seven heads of 64: 81 us.  The first scores are there 4 (512 tokens) to 7 us after a
// CTA's start.  Heads of 256, one tile a CTA: the eight 106 us, 8192 tokens 380-398 us (1.4 PFLOP/s).
//
// Warps 0-15: the tiles' rows.  Warp 16: TMA.  Warps 17 and 18: the tiles' MMAs (one thread for both spent more on issuing and waiting
// than the tensor core on multiplying: 16384 tokens 916 us).  Warp 19: the list, and V of items done again.
#include <algorithm>

#include "flash.cuh"
#include "packed_ops.h"

namespace pbd {

using namespace flash;

namespace {

constexpr int PA_MASKED = 2;  // blocks that not all rows of a CTA see, at most

template <int D>
struct PromptShape : Shape<D> {
    using S = Shape<D>;
    static constexpr int STAGES = D == 64 ? 8 : 4;
    static constexpr int AHEAD = D == 64 ? 8 : 4;  // items that are told of, and notes of their values of V: more than the ring can be ahead of the rows
    static constexpr int SMEM = S::TILES * S::QT + STAGES * S::UNIT + 1024;
};

// What a CTA works on: tokens from q0 of a sequence of `len`, heads ch * P .. of the group of KV head h.  len 0: nothing more.
struct PromptItem {
    int start, len, q0, h, ch;
    int nb[2], masked;  // the tiles' blocks; those that all rows of both see
    int careful;        // done again
};

template <int D>
struct PromptState {
    using L = PromptShape<D>;
    uint64_t full[L::STAGES], empty[L::STAGES], q_full, q_free, s_full[2], p_full[2][2], o_done[2], o_free[2], turn[2], drain[2];
    uint64_t v_full[L::AHEAD][PA_MASKED], v_fixed[L::AHEAD][PA_MASKED], item_full[L::AHEAD], item_free[L::AHEAD];
    uint32_t tmem;
    uint32_t patience;  // mbar_wait_short
    int bad;  // bounds of a sequence
    PromptItem item[L::AHEAD];
    float top[2][2][ROWS];    // what the two threads of a row tell each other
    int odd[L::AHEAD];  // whether a result is not finite
    int first_odd[L::AHEAD][D];  // done again: the first row that sees an infinite or NaN value in this dimension
    int start[KV_MAX_BATCH], tiles[KV_MAX_BATCH];
};

// Item o of all.  Those with the most keys come first: by token tile, the last ones before, then by sequence; the heads of one
// innermost.  A warp; `most`: the largest number of token tiles.
__device__ __forceinline__ bool find_item(const PackedArgs &a, const int *start, const int *tiles, long long x, int total, int most, int heads, int chunks,
                                          int tokens, int tile_tokens, bool two, PromptItem &it) {
    const int lane = threadIdx.x & 31;
    if (x >= (long long)total * heads) return false;
    const int o = (int)(x / heads), hc = (int)(x - (long long)o * heads);
    // items of token tiles t and above
    auto count = [&](int t) {
        int n = 0;
        for (int b = lane; b < a.B; b += 32) n += max(tiles[b] - t, 0);
        return __reduce_add_sync(0xffffffffu, n);
    };
    int lo = 0, hi = most, above = 0;  // count(hi) = above <= o < count(lo)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1, n = count(mid);
        if (n <= o)
            hi = mid, above = n;
        else
            lo = mid;
    }
    int r = o - above, b = 0;  // which of the sequences with a token tile lo
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const bool in = b0 + lane < a.B && tiles[b0 + lane] > lo;
        const unsigned m = __ballot_sync(0xffffffffu, in);
        const int n = __popc(m);
        if (r < n) {
            const int before = __popc(m & ((1u << lane) - 1));
            b = b0 + __ffs(__ballot_sync(0xffffffffu, in && before == r)) - 1;
            break;
        }
        r -= n;
    }
    it.start = start[b];
    it.len = a.starts[b + 1] - it.start;
    it.q0 = lo * tokens;
    it.h = hc / chunks;
    it.ch = hc - it.h * chunks;
    for (int i = 0; i < 2; ++i) {
        const int first = it.q0 + i * tile_tokens;
        it.nb[i] = first >= it.len || (i && !two) ? 0 : min(first + tile_tokens - 1, it.len - 1) / KEYS + 1;
    }
    it.masked = (it.q0 + 1) / KEYS;
    it.careful = 0;
    return true;
}

// Stores K and V into the cache, beside k_prompt: a warp a row.  Its CTAs fit an SM together with k_prompt's, whose registers leave 4096.  (By
// k_prompt's own threads, before an item's first scores, it costs them registers that they lack.)  Beside k_prompt's warps its own fetch their code
// anew for every row, and that bounds it: a short loop without divisions and unrolling, the next row's slot on its way (1000 prompts of 40
// tokens, 8 KV heads of 128: 215 us, 211 alone, k_prompt alone 192; 295 before; two warps a CTA with all of a row's loads on their way: 857).
constexpr int PS_WARPS = 4;
__global__ void __launch_bounds__(32 * PS_WARPS, 16) k_prompt_store(const __grid_constant__ PackedArgs a) {
    __shared__ int start[KV_MAX_BATCH], end[KV_MAX_BATCH];
    bool descends = false;
    for (int b = threadIdx.x; b < a.B; b += 32 * PS_WARPS) {
        const int s = a.starts[b], e = a.starts[b + 1];
        start[b] = s;
        end[b] = s < 0 || e > a.T ? s : e;  // (between bounds that descend there is no row)
        descends |= e < s;
    }
    if (__syncthreads_or(descends)) {
        for (int b = threadIdx.x; b < a.B; b += 32 * PS_WARPS)
            if (!behind_all(a.starts, b)) end[b] = start[b];
        __syncthreads();
    }
    const int lane = threadIdx.x & 31;
    const long long slots = (long long)a.kv.n_pages * a.kv.page_size;
    const int log_per = 28 - __clz(a.d), pieces = a.hkv << log_per;  // 16-byte pieces of a head, of a row
    bool bad = false;
    int t = blockIdx.x * PS_WARPS + (threadIdx.x >> 5);
    long long next = t < a.T ? a.slots[t] : -1;
    for (; t < a.T; t += gridDim.x * PS_WARPS) {
        const long long slot = next;
        if (a.T - t > gridDim.x * PS_WARPS) next = a.slots[t + gridDim.x * PS_WARPS];
        bool mine = false;
        for (int b = lane; b < a.B; b += 32) mine |= start[b] <= t && t < end[b];
        if (!__any_sync(0xffffffffu, mine)) continue;
        bad |= slot >= slots;
        if (slot < 0 || slot >= slots) continue;
        const long long page = slot >> 32 ? slot / a.kv.page_size : (long long)((uint32_t)slot / (uint32_t)a.kv.page_size);
        const long long dst = page * a.kv.stride_page + (slot - page * a.kv.page_size) * a.kv.stride_slot, src = (long long)t * a.kv_stride;
#pragma unroll 1
        for (int i = lane; i < pieces; i += 32) {
            const long long to = dst + (i >> log_per) * a.kv.stride_head + (i & ((1 << log_per) - 1)) * 8;
            const uint4 k = *reinterpret_cast<const uint4 *>(a.k + src + i * 8), v = *reinterpret_cast<const uint4 *>(a.v + src + i * 8);
            *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.k) + to) = k;
            *reinterpret_cast<uint4 *>(const_cast<uint16_t *>(a.kv.v) + to) = v;
        }
    }
    pdl_wait();  // (k_prompt has cleared the status, and said what it found: that goes first)
    if (__syncthreads_or(bad) && threadIdx.x == 0) latch_error(a.status, DEV_BAD_PAGE);
}

template <int D, bool FP16>
__global__ void __launch_bounds__(THREADS, 1)
    k_prompt(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
             const __grid_constant__ PackedArgs a, int P, uint32_t inv_p) {
    using L = PromptShape<D>;
    constexpr int TILES = L::TILES, UNITS = L::UNITS, STAGES = L::STAGES, AHEAD = L::AHEAD;
    constexpr bool TWO = TILES == 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sq = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *ring = sq + TILES * L::QT;
    __shared__ PromptState<D> S;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int tile_tokens = ROWS * inv_p >> 16, tokens = TILES * tile_tokens;  // (inv_p: 1 / P in 16 bits, exact for what it is used for)
    const int chunks = a.group * inv_p >> 16, heads = a.hkv * chunks;
    pdl_launch();
    if (warp == 16) tmem_alloc(&S.tmem, TM_COLS);
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&S.full[i], 1);
            mbar_init(&S.empty[i], TILES);
        }
        mbar_init(&S.q_full, 1);
        mbar_init(&S.q_free, TILES);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&S.s_full[i], 1);
            mbar_init(&S.p_full[i][0], 8);
            mbar_init(&S.p_full[i][1], 8);
            mbar_init(&S.o_done[i], 1);
            mbar_init(&S.o_free[i], 8);
            mbar_init(&S.turn[i], 1);
            mbar_init(&S.drain[i], 1);
        }
        for (int i = 0; i < AHEAD; ++i) {
            for (int k = 0; k < PA_MASKED; ++k) {
                mbar_init(&S.v_full[i][k], 1);
                mbar_init(&S.v_fixed[i][k], 1);
            }
            mbar_init(&S.item_full[i], 1);
            mbar_init(&S.item_free[i], ROW_WARPS + 1 + TILES);
        }
        S.patience = a.patience;
        S.bad = 0;
        fence_mbarrier_init();
        if (blockIdx.x == 0) *a.status = DEV_OK;  // (a wait runs out a second later)
    }
    __syncthreads();
    // rows of no token stay zero
    for (int x = tile_tokens * P * 8 + threadIdx.x; x < ROWS * 8; x += THREADS)
        for (int c = 0; c < TILES * (D / 64); ++c) st_shared_u4(smem_u32(sq) + c * SUB + x * 16, make_uint4(0, 0, 0, 0));
    fence_proxy_async_shared();
    if (threadIdx.x == 32) {
        prefetch_tensormap(&qmap);
        prefetch_tensormap(&kmap);
        prefetch_tensormap(&vmap);
    }
    for (int b = threadIdx.x; b < a.B; b += THREADS) {
        const int s = a.starts[b], e = a.starts[b + 1];
        S.start[b] = s;
        const bool ok = bounds_ok(a, s, e);
        S.tiles[b] = ok ? (e - s + tokens - 1) / tokens : 0;
        if (!ok) S.bad = 1;
    }
    tc_fence_before();
    __syncthreads();
    if (S.bad) {
        for (int b = threadIdx.x; b < a.B; b += THREADS)
            if (!behind_all(a.starts, b)) S.tiles[b] = 0;
        __syncthreads();
    }
    tc_fence_after();
    const uint32_t tmem = S.tmem;
    // Whether there is an n-th item: S.item[n % AHEAD].
    auto item_there = [&](int n) {
        return mbar_wait_short(&S.item_full[n % AHEAD], (n / AHEAD) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience) && *(volatile int *)&S.item[n % AHEAD].len > 0;
    };

    if (warp >= ROW_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
        if (warp == 16) {
            if (elect_one()) {
                // ---- TMA: an item's queries, then K and V in the ring's order
                int issued = 0, n = 0;
                bool ok = true;
                for (; ok; ++n) {
                    if (!item_there(n)) break;
                    const int s = n % AHEAD;
                    const PromptItem it = S.item[s];
                    mbarrier_arrive_one(&S.item_free[s]);
                    const int nmax = max(it.nb[0], it.nb[1]);
                    if (n > 0 && !mbar_wait_short(&S.q_free, (n - 1) & 1, a.status, DEV_TIMEOUT_SLOT, &S.patience)) break;
                    mbar_arrive_expect_tx(&S.q_full, (uint32_t)(TILES * (D / 64) * 128 * tile_tokens * P));
                    for (int i = 0; i < TILES; ++i)
                        for (int c = 0; c < D / 64; ++c)
                            tma_load_4d(sq + i * L::QT + c * SUB, &qmap, c * 64, 0, it.h * chunks + it.ch, it.start + it.q0 + i * tile_tokens, &S.q_full);
                    for (int k = it.careful ? nmax - it.masked : 0; k < PA_MASKED; ++k) mbarrier_arrive_one(&S.v_full[s][k]);
                    for (int x = 0; ok && x < 2 * nmax; ++x) {
                        const int y = at_place(x, nmax, TWO), kb = y < 0 ? ~y : y;
                        for (int u = 0; u < UNITS; ++u) {
                            const int slot = issued % STAGES;
                            if (!mbar_wait_short(&S.empty[slot], ((issued / STAGES) & 1) ^ 1, a.status, DEV_TIMEOUT_SLOT, &S.patience)) {
                                ok = false;
                                break;
                            }
                            ++issued;
                            uint64_t *bar = &S.full[slot];
                            if (y < 0 && it.careful && kb >= it.masked) {  // V that is looked at first
                                mbarrier_arrive_one(bar);
                                bar = &S.v_full[s][kb - it.masked];
                                if (u == 0) mbar_arrive_expect_tx(bar, (uint32_t)(UNITS * L::UNIT));
                            } else {
                                mbar_arrive_expect_tx(bar, (uint32_t)L::UNIT);
                            }
                            for (int c = 0; c < L::DU / 64; ++c)
                                tma_load_3d(ring + slot * L::UNIT + c * SUB, y < 0 ? &vmap : &kmap, u * L::DU + c * 64, it.h, it.start + kb * KEYS, bar);
                        }
                    }
                }
                if (*(volatile uint32_t *)&S.patience == 0) {  // error path: the copies in flight get a bounded chance to land
                    const uint64_t t0 = globaltimer_ns();
                    while (globaltimer_ns() - t0 < WAIT_LIMIT_NS / 100) __nanosleep(1000);
                }
            }
        } else if (warp < 17 + TILES) {
            if (elect_one()) {
                // ---- MMAs of tile i
                const int i = warp - 17;
                const uint8_t *q = sq + i * L::QT;
                const uint32_t o = tmem + TM_O + i * D;
                bool ok = true;
                int pos = 0, step = 0, used = 0, used_o = 0;  // blocks' K and V, sections, blocks and items of the tile so far
                auto wait = [&](uint64_t *bar, int phase, int code) { ok = ok && mbar_wait_short(bar, phase & 1, a.status, code, &S.patience); };
                auto landed = [&](int place) {
                    for (int u = 0; u < UNITS; ++u) wait(&S.full[(place * UNITS + u) % STAGES], (place * UNITS + u) / STAGES, DEV_TIMEOUT_LOAD);
                };
                auto unit = [&](int place, int u) { return ring + ((place * UNITS + u) % STAGES) * L::UNIT; };
                auto scores = [&](int buf, int place) {
                    for (int u = 0; u < UNITS; ++u) mma_scores<D, FP16>(tmem + buf * KEYS, q, unit(place, u), u);
                    mma_commit(&S.s_full[buf]);
                };
                // (K and V that a tile has seen are given back by its rows, when they see S and O: each commit here costs 200 cycles)
                auto skip = [&](int place) {
                    for (int u = 0; u < UNITS; ++u) mbarrier_arrive_one(&S.empty[(place * UNITS + u) % STAGES]);
                };
                for (int n = 0; ok; ++n) {
                    if (!item_there(n)) break;
                    const PromptItem *it = &S.item[n % AHEAD];
                    const int nb = it->nb[i], nmax = max(it->nb[0], it->nb[1]), len = it->len, masked = it->careful ? it->masked : nmax;
                    mbarrier_arrive_one(&S.item_free[n % AHEAD]);
                    // P V of block j from the first part of P on
                    auto values = [&](int buf, int j, int place, int phase) {
                        // (the last block's keys behind the sequence's end are not multiplied, to 16)
                        const int steps = min(KEYS, len - j * KEYS + 15) / 16;
                        for (int u = 0; u < UNITS; ++u) mma_values<D, FP16>(o, tmem + buf * KEYS, unit(place, u), u, 0, steps, j == 0);
                        wait(&S.p_full[buf][1], phase, DEV_TIMEOUT_MMA);
                        if (!ok) return;
                        tc_fence_after();
                        for (int u = 0; u < UNITS; ++u) mma_values<D, FP16>(o, tmem + buf * KEYS, unit(place, u), u, 1, steps, j == 0);
                    };
                    auto values_ready = [&](int j, int place) {
                        landed(place);
                        if (j >= masked) wait(&S.v_fixed[n % AHEAD][j - masked], n / AHEAD, DEV_TIMEOUT_LOAD);
                        if (j == 0 && used_o > 0 && nb > 0) wait(&S.o_free[i], used_o - 1, DEV_TIMEOUT_MMA);
                    };
                    wait(&S.q_full, n, DEV_TIMEOUT_LOAD);
                    if (TWO) {  // for every block O += P V of the one before, then S; the tiles in turns
#pragma unroll 1
                        for (int j = 0; ok && j <= nmax; ++j, ++step) {
                            const int vp = pos + v_place(j - 1, nmax, true), kp = pos + k_place(j, true);
                            if (j > 0) values_ready(j - 1, vp);
                            if (j < nmax) landed(kp);
                            if (i + step > 0) wait(&S.turn[i], step + i - 1, DEV_TIMEOUT_MMA);
                            if (j > 0 && j <= nb) wait(&S.p_full[i][0], used + j - 1, DEV_TIMEOUT_MMA);
                            if (!ok) break;
                            tc_fence_after();
                            if (j > 0 && j <= nb) values(i, j - 1, vp, used + j - 1);
                            if (ok && j < nb) scores(i, kp);
                            mbarrier_arrive_one(&S.turn[i ^ 1]);
                            if (j > 0 && j == nb) mma_commit(&S.o_done[i]);
                            if (j == max(nb, 1) - 1) mma_commit(&S.q_free);
                            if (j > nb) skip(vp);  // (blocks that only the other tile sees)
                            if (j >= nb && j < nmax) skip(kp);
                        }
                    } else {  // S of the next block, then O += P V of this one
                        landed(pos);
                        if (ok) {
                            tc_fence_after();
                            scores(used & 1, pos);
                            if (nmax == 1) mma_commit(&S.q_free);
                        }
#pragma unroll 1
                        for (int j = 0; ok && j < nmax; ++j) {
                            const int vp = pos + v_place(j, nmax, false), kp = pos + k_place(j + 1, false), x = used + j;
                            if (j + 1 < nmax) {
                                landed(kp);
                                if (!ok) break;
                                tc_fence_after();
                                scores((x + 1) & 1, kp);
                                if (j + 2 == nmax) mma_commit(&S.q_free);
                            }
                            values_ready(j, vp);
                            wait(&S.p_full[x & 1][0], x >> 1, DEV_TIMEOUT_MMA);
                            if (!ok) break;
                            tc_fence_after();
                            values(x & 1, j, vp, x >> 1);
                            mma_commit(&S.o_done[0]);
                        }
                    }
                    pos += 2 * nmax;
                    used += nb;
                    used_o += nb > 0;
                }
                mma_commit(&S.drain[i]);  // every MMA issued completes before TMEM is released
                mbar_wait_short(&S.drain[i], 0, nullptr, 0, nullptr);
            }
        } else if (warp == 19) {
            // ---- the list, one item ahead; V of items done again
            int total = 0, most = 0, pos = 0, given = 0;  // given: items of the CTA's share so far
            for (int b = lane; b < a.B; b += 32) total += S.tiles[b], most = max(most, S.tiles[b]);
            total = __reduce_add_sync(0xffffffffu, total);
            most = __reduce_max_sync(0xffffffffu, most);
            bool ok = true;
            auto next_item = [&]() {  // there and back over the CTAs: each gets long and short ones
                PromptItem it{};
                const long long x = (long long)given * gridDim.x + (given & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
                ++given;
                if (!find_item(a, S.start, S.tiles, x, total, most, heads, chunks, tokens, tile_tokens, TWO, it)) it.len = 0;
                return it;
            };
            auto publish = [&](int n, const PromptItem &it) {
                const int s = n % AHEAD;
                if (it.careful)
                    for (int d = lane; d < D; d += 32) S.first_odd[s][d] = 0x7fffffff;
                __syncwarp();
                if (lane == 0) {
                    S.item[s] = it;
                    S.odd[s] = 0;
                    mbarrier_arrive_one(&S.item_full[s]);
                }
                __syncwarp();
                return it.len > 0;
            };
            int told = 0;  // items that the others have been told of, one ahead where there is one
            if (publish(told++, next_item())) {
                const PromptItem next = next_item();
                if (next.len > 0) publish(told++, next);
            }
            for (int n = 0; ok && S.item[n % AHEAD].len > 0; ++n) {
                const int s = n % AHEAD;
                const PromptItem it = S.item[s];
                const int nmax = max(it.nb[0], it.nb[1]);
                for (int k = 0; ok && k < PA_MASKED; ++k) {
                    const int j = it.masked + k;
                    if (it.careful) ok = mbar_wait_short(&S.v_full[s][k], (n / AHEAD) & 1, a.status, DEV_TIMEOUT_LOAD, &S.patience);
                    if (!(ok = __all_sync(0xffffffffu, ok))) break;
                    for (int u = 0; it.careful && j < nmax && u < UNITS; ++u) {
                        const int slot = ((pos + v_place(j, nmax, TWO)) * UNITS + u) % STAGES;
                        const uint32_t at = smem_u32(ring + slot * L::UNIT);
                        const int all = it.len - j * KEYS;  // keys of the block
                        for (int r = all + (lane >> 3); r < KEYS; r += 4)
                            for (int c = 0; c < L::DU / 64; ++c) st_shared_u4(at + c * SUB + r * 128 + (lane & 7) * 16, make_uint4(0, 0, 0, 0));
                        __syncwarp();
                        // (loads of many rows on their way together: one after the other they took 8000 cycles)
                        constexpr int U = 8;
#pragma unroll 1
                        for (int x0 = lane; x0 < L::UNIT / 16; x0 += 32 * U) {
                            uint4 v[U];
                            uint32_t any = 0;
#pragma unroll
                            for (int y = 0; y < U; ++y) v[y] = ld_shared_u4(at + (x0 + 32 * y) * 16);
#pragma unroll
                            for (int y = 0; y < U; ++y)
                                any |= odd_halves<FP16>(v[y].x) | odd_halves<FP16>(v[y].y) | odd_halves<FP16>(v[y].z) | odd_halves<FP16>(v[y].w);
                            if (any == 0) continue;
#pragma unroll 1
                            for (int e = 0; e < 8 * U; ++e) {  // (value by value: this is rare)
                                const int x = x0 + 32 * (e >> 3), r = (x >> 3) & 127;
                                const uint32_t to = at + x * 16 + 2 * (e & 7);
                                uint16_t y;
                                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(to) : "memory");
                                if (!odd_halves<FP16>(y)) continue;
                                asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"((uint16_t)0) : "memory");
                                atomicMin(&S.first_odd[s][u * L::DU + (x >> 10) * 64 + (((x & 7) ^ (r & 7)) << 3) + (e & 7)], j * KEYS + r);
                            }
                        }
                    }
                    fence_proxy_async_shared();
                    __syncwarp();
                    if (lane == 0) mbarrier_arrive_one(&S.v_fixed[s][k]);
                }
                pos += 2 * nmax;
                // when everybody is through with it: the next one, or this one again
                ok = ok && mbar_wait_short(&S.item_free[s], (n / AHEAD) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                PromptItem next = it;
                next.careful = 1;
                if (it.careful || !*(volatile int *)&S.odd[s]) next = next_item();
                if (next.len > 0 || told == n + 1) publish(told++, next);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ROW_REGS));
        // ---- rows: row r of tile i is token first + r / P, head r % P
        const int i = warp >> 3, half = (warp >> 2) & 1, w = warp & 3, row = w * 32 + lane, id = 1 + i * 4 + w;
        const uint32_t lanes = (uint32_t)(w * 32) << 16, ts = tmem + lanes + 64 * half, to = tmem + lanes + TM_O + i * D + half * (D / 2);
        const float c = a.scale * 1.4426950408889634f;
        const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
        float *top = S.top[i][0];
        Row r{0.f, 0.f};
        bool ok = true;
        int used = 0, used_o = 0, pos = 0;  // blocks and items of the tile so far, blocks' K and V of the CTA
        auto release = [&](int place) {
            if (w == 0 && half == 0 && lane == 0)
                for (int u = 0; u < UNITS; ++u) mbarrier_arrive_one(&S.empty[(place * UNITS + u) % STAGES]);
        };
        for (int n = 0; ok; ++n) {
            const int s = n % AHEAD;
            const volatile PromptItem &it = S.item[s];  // (read again at the end, to spare registers)
            if (pair_any(id, !mbar_wait_short(&S.item_full[s], (n / AHEAD) & 1, a.status, DEV_TIMEOUT_DEP, &S.patience))) break;
            const int nb = it.nb[i], first = it.q0 + i * tile_tokens;
            if (it.len == 0) break;
            const int nmax = max(it.nb[0], it.nb[1]);
            if (nb == 0) {
                pos += 2 * nmax;
                if (lane == 0) mbarrier_arrive_one(&S.item_free[s]);
                continue;
            }
            for (int j = 0; ok && j < nb; ++j, ++used) {
                const int buf = TWO ? i : used & 1;
                bool there = mbar_wait_short(&S.s_full[buf], (TWO ? used : used >> 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.patience), o_waited = TWO || j == 0;
                there = __all_sync(0xffffffffu, there);
                release(pos + k_place(j, TWO));
                if (TWO && j > 0) release(pos + v_place(j - 1, nmax, TWO));
                tc_fence_after();
                uint32_t s[64];
#pragma unroll
                for (int x = 0; x < 64; x += 32) tmem_ld_32cols(ts + buf * KEYS + x, *reinterpret_cast<uint32_t(*)[32]>(&s[x]));
                tmem_ld_wait();
                if (j * KEYS + KEYS - 1 > first) {
                    const int last = first + (int)(row * inv_p >> 16) - j * KEYS - 64 * half;
#pragma unroll
                    for (int x = 0; x < 64; ++x)
                        if (x > last) s[x] = __float_as_uint(-INFINITY);
                }
                auto o_ready = [&]() {  // (with two tiles S of this block has come after O of the one before)
                    bool o = true;
                    if (!o_waited) {
                        o = mbar_wait_short(&S.o_done[0], (used - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.patience);
                        release(pos + v_place(j - 1, nmax, TWO));
                    }
                    o_waited = true;
                    return __all_sync(0xffffffffu, o) != 0;
                };
                ok = softmax_half<D, FP16>(r, s, there, c, j == 0, ts + buf * KEYS, to, id, top, half, row, o_ready, [&](int part) {
                    if (!TWO && part == 1) o_ready();  // (every phase is waited for)
                    if (lane == 0) mbarrier_arrive_one(&S.p_full[buf][part]);
                });
            }
            bool there = mbar_wait_short(&S.o_done[i], (TWO ? used_o : used - 1) & 1, a.status, DEV_TIMEOUT_MMA, &S.patience);
            ++used_o;
            release(pos + v_place(nb - 1, nmax, TWO));
            pos += 2 * nmax;
            const bool careful = it.careful != 0;
            for (int k = 0; careful && there && k < PA_MASKED; ++k) there = mbar_wait_short(&S.v_fixed[s][k], (n / AHEAD) & 1, a.status, DEV_TIMEOUT_LOAD, &S.patience);
            if (!ok || pair_any(id, !there)) break;
            top[half * ROWS + row] = r.l;
            pair_sync(id);
            r.l += top[(half ^ 1) * ROWS + row];
            tc_fence_after();
            const int place = row * inv_p >> 16, head = it.h * a.group + it.ch * P + row - place * P, token = first + place;
            const bool real = token < it.len && place < tile_tokens;
            const long long out_row = (long long)(it.start + token) * a.hq + head;
            const bool odd = store_half<D, FP16>(to, row_factor(r), a.out + out_row * D + half * (D / 2), real, wide, careful,
                                                 [&](int d) { return S.first_odd[s][half * (D / 2) + d] <= token; });
            tc_fence_before();
            if (__any_sync(0xffffffffu, odd) && lane == 0) *(volatile int *)&S.odd[s] = 1;
            __syncwarp();
            if (lane == 0) {
                mbarrier_arrive_one(&S.o_free[i]);
                mbarrier_arrive_one(&S.item_free[s]);
            }
            if (a.lse && half == 0 && real) a.lse[out_row] = row_lse<FP16>(r, a.scale);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 16) tmem_dealloc(tmem, TM_COLS);
    if (blockIdx.x == 0 && threadIdx.x == 0 && S.bad) latch_error(a.status, DEV_BAD_POSITION);
}

template <int D, bool FP16>
cudaError_t launch(const PackedArgs &a, cudaStream_t st) {
    using L = PromptShape<D>;
    static_assert(L::SMEM + sizeof(PromptState<D>) <= 227 * 1024, "shared memory");
    static std::atomic<uint64_t> set{0};
    const cudaError_t e = once_per_device(set, [] {
        const cudaError_t x = cudaFuncSetAttribute(k_prompt<D, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
        // (an SM divides its memory into cache and shared one kernel's way at a time: without this the two do not share an SM)
        return x != cudaSuccess ? x : cudaFuncSetAttribute(k_prompt_store, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    });
    if (e != cudaSuccess) return e;
    // the largest divisor of the group up to 16 that leaves at most 8 rows over.  (One head a tile instead: 1000 prompts of 40 tokens 392 us instead of
    // 216, 32 ragged ones in groups of seven 95.5 instead of 81, eight in groups of 16 53.8 instead of 50.3, of 32 98 instead of 90.6.  Up to 8 or 32:
    // within 1 %.  No row left over: groups of seven have one head a tile then.  Up to 16 rows: a group of 13 has 13 heads a tile, 49.1 us
    // instead of 48.8: K and V come from the L2 when each head reads them.)
    int P = std::min(a.group, 16);
    while (a.group % P || ROWS % P > 8) --P;
    const uint32_t inv_p = 65536 / P + 1;
    const int tokens = L::TILES * (ROWS / P), heads = a.hq / P;
    const long long items = std::min<long long>(a.T / tokens + a.B, a.T) * heads;
    const int grid = (int)std::min<long long>(items, gemm_ctas());
    if (grid < 1) return cudaErrorInvalidDevice;
    CUtensorMap qm, km, vm;
    const uint64_t qs = (uint64_t)a.q_stride * 2, ks = (uint64_t)a.kv_stride * 2;
    const uint64_t qd[4] = {(uint64_t)D, (uint64_t)P, (uint64_t)heads, (uint64_t)a.T}, qst[3] = {D * 2, (uint64_t)P * D * 2, qs};
    const uint32_t qb[4] = {64, (uint32_t)P, 1, (uint32_t)(ROWS / P)};
    const uint64_t kd[3] = {(uint64_t)D, (uint64_t)a.hkv, (uint64_t)a.T}, kst[2] = {D * 2, ks};
    const uint32_t kb[3] = {64, 1, KEYS};
    if (!encode_map_16(&qm, a.q, 4, qd, qst, qb) || !encode_map_16(&km, a.k, 3, kd, kst, kb) || !encode_map_16(&vm, a.v, 3, kd, kst, kb))
        return cudaErrorInvalidValue;
    k_prompt<D, FP16><<<grid, THREADS, L::SMEM, st>>>(qm, km, vm, a, P, inv_p);
    const cudaError_t c = cudaGetLastError();
    // (the store as the second of the two, not the first, which k_prompt's CTAs would wait for: 512 tokens 15.5 us instead of 16.2)
    return c != cudaSuccess || !a.kv.k ? c : launch_pdl(k_prompt_store, std::min((a.T + PS_WARPS - 1) / PS_WARPS, gemm_ctas()), 32 * PS_WARPS, 0, st, a);
}

}  // namespace

cudaError_t launch_prompt_attention(PackedArgs &a, cudaStream_t st) {
    a.patience = prompt_patience(a.T);
    if (a.fp16) return a.d == 64 ? launch<64, true>(a, st) : a.d == 128 ? launch<128, true>(a, st) : launch<256, true>(a, st);
    return a.d == 64 ? launch<64, false>(a, st) : a.d == 128 ? launch<128, false>(a, st) : launch<256, false>(a, st);
}

}  // namespace pbd
