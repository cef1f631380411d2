// kv_attn.cu -- attention of one new token a sequence over a caller's paged cache (pbd_op_decode_attention).
//
// For query head h of KV head h / group and cached slot j:
//     s_hj = q_h . k_j,   p_hj = exp(scale (s_hj - max_j s_hj)),   l_h = sum_j p_hj,   out_h = sum_j p_hj v_j / l_h
// in one pass over K and V with a running maximum and sum.  Every cached byte is read once and used for the few
// query heads of its group, so memory bounds it.
//
// Work is cut into tiles of 16 slots of one (sequence, KV head).  A warp attends to a stretch of tiles with a ring of its own
// in shared memory, filled by 16-byte asynchronous copies, and waits for no other warp until it is done.
//
// Two ways to share the tiles out:
// - Small calls (launch): one cluster a (sequence, KV head), whose warps take a row's tiles in equal parts and join through
//   distributed shared memory.  One launch.
// - All others: the tiles of the whole batch form one list, [sequence][KV head][tile], and each warp takes one contiguous
//   stretch of it, all of about the same cost: how ragged the lengths are does not matter, and the host need not know
//   them.  Where a stretch begins or ends inside a (sequence, KV head) the warp leaves maximum, sum and unnormalised output in
//   scratch, and k_decode_join joins them.
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
constexpr int DA_SLOTS = 16;      // slots of a tile
constexpr int DA_MIN_TILES = 2;   // of a warp's stretch
constexpr int DA_ROW_TILES = 2;   // what beginning and ending a (sequence, KV head) costs a warp, in tiles (64 ragged: 31.8 us, 35.0 with 1, 32.2 with 4)
constexpr float DA_FP16_SHIFT = 10.f, DA_SLACK = 4.f;  // log2 of factors: of P in fp16, of P beyond 1 (attend)
constexpr int DA_CLUSTER = 16;    // CTAs of a cluster at most
constexpr int DA_CLUSTER_TILES = 16;  // tiles of its warps at most

// stages of a warp's ring and CTAs that fit an SM's shared memory: 96 KB (d = 256: 192 KB) a CTA
template <int D>
struct DaShape {
    static constexpr int UNIT = DA_SLOTS * D * 2 * 2;  // bytes of a tile: K rows, then V rows
    static constexpr int STAGES = D == 64 ? 6 : 3;
    static constexpr int CTAS = D == 256 ? 1 : 2;
    static constexpr int RING = DA_WARPS * STAGES * UNIT;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ const uint4 zero_row[32] = {};  // what is copied for rows that are none

__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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

// Slots that the call attends to in sequence b: none where the length, which is reported, lies outside the table (nothing
// is stored there either).
__device__ __forceinline__ bool length_ok(const DecodeArgs &a, int n) { return n >= 0 && n <= a.kv.cap - (a.k_new ? 1 : 0); }
__device__ __forceinline__ int attended(const DecodeArgs &a, int b) {
    const int n = a.kv.lens[b];
    return length_ok(a, n) ? n + (a.k_new ? 1 : 0) : 0;
}

// The table's entry for a slot.
__device__ __forceinline__ int page_of(const DecodeArgs &a, int b, int slot) {
    return a.kv.table[(long long)b * a.kv.max_pages + page_index(a.kv, slot)];
}

// The list of all tiles.  A (sequence, KV head, chunk of its query heads) is a row; it counts as its tiles and ROW more in
// front, so that stretches with many short rows are shorter.  first[b]: the count of one row of each sequence
// before b; len[b]: slots attended to.  Whole CTA.
template <int ROW>
__device__ __forceinline__ int row_count(int n) { return n > 0 ? (n + DA_SLOTS - 1) / DA_SLOTS + ROW : 0; }
template <int ROW>
__device__ __forceinline__ void tile_lists(const DecodeArgs &a, int *first, int *len) {
    __shared__ int warp_sum[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < a.kv.B; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        const int n = b < a.kv.B ? attended(a, b) : 0;
        if (b < a.kv.B) len[b] = n;
        int x = row_count<ROW>(n);
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

// warps that share the list, the first place of one of them, and the one that has a place
__device__ __forceinline__ int workers_of(const DecodeArgs &a, int count) {
    return max(1, min(a.workers, (count + DA_MIN_TILES - 1) / DA_MIN_TILES));
}
__device__ __forceinline__ int first_of(int w, int count, int workers) { return (int)((long long)w * count / workers); }
__device__ __forceinline__ int worker_at(long long at, int count, int workers) { return (int)(((at + 1) * workers - 1) / count); }

// Tiles [t, t_end) of one row: what a warp works on before it leaves the row.
template <int ROW>
struct Segment {
    int b, h, ch, t, t_end, tiles, n;  // sequence, KV head, chunk of its query heads, the row's tiles and slots
    int at, end;                    // list place of the row, end of the warp's stretch
    __device__ __forceinline__ bool clip(const int *len) {
        n = len[b];
        tiles = (n + DA_SLOTS - 1) / DA_SLOTS;
        t_end = min(tiles, end - at - ROW);
        return t < t_end;
    }
    // The first segment of the stretch [u, end); false if it has none.
    __device__ __forceinline__ bool seek(int u, int u_end, const int *first, const int *len, int B, int hkv, int chunks) {
        const int HC = hkv * chunks;
        end = u_end;
        if (u >= end) return false;
        int lo = 0, hi = B;  // first[lo] * HC <= u < first[hi] * HC
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((long long)first[mid] * HC <= u)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
        const int per = first[b + 1] - first[b];
        const int hc = (u - first[b] * HC) / per;
        h = hc / chunks;
        ch = hc - h * chunks;
        at = first[b] * HC + hc * per;
        t = max(0, u - at - ROW);
        return clip(len) || next(first, len, B, hkv, chunks);
    }
    __device__ __forceinline__ bool next(const int *first, const int *len, int B, int hkv, int chunks) {
        at += first[b + 1] - first[b];
        if (++ch == chunks) {
            ch = 0;
            if (++h == hkv) {
                h = 0;
                do ++b;
                while (b < B && first[b + 1] == first[b]);
            }
        }
        t = 0;
        return b < B && at < end && clip(len);  // (where only a row's front is left the stretch is over)
    }
};

// What a warp keeps in shared memory beside its tiles.
template <int STAGES>
struct Rings {
    ulonglong2 row[2][DA_SLOTS];  // where the rows of a tile's K and V are: of the tile to be copied, and of the next
    struct {
        long long off;  // where a new token's row goes in K and V (-1: nowhere), and its position
        int pos;
    } fresh[STAGES + 1];
    int page[STAGES][DA_SLOTS];  // the table's entries
};

using Tiles = Segment<DA_ROW_TILES>;

// A warp's work on its segments: `next(segment)` makes the following one of it, `leave(segment, t0, m, l, o)` takes the
// results of tiles [t0, t_end) of a row: maxima and sums (a lane's own part of them) of heads 8 nt + 2 (lane % 4) + e, and outputs
// o[ks][nt]: dims 16 ks + lane / 4 (+ 8 in elements 2 and 3) of those heads.
// Returns whether a page was outside the cache.
template <bool FP16, int D, int NT, typename Next, typename Leave>
__device__ __forceinline__ bool attend(const DecodeArgs &a, uint32_t ring, Rings<DaShape<D>::STAGES> &rings, Tiles at, Next &&next,
                                       Leave &&leave) {
    using S = DaShape<D>;
    constexpr int HEADS = 8 * NT, KS = D / 16, CPR = D / 8;  // heads of a chunk, k steps, 16-byte pieces of a row
    constexpr bool Q_AHEAD = KS * NT <= 16;                  // a row's queries are asked for a row ahead, if registers allow
    const int lane = threadIdx.x & 31;
    const bool append = a.k_new != nullptr;
    const float c = a.scale * 1.4426950408889634f;
    // P's scale: weights of fp16 lie in 2^-24 .. 2^14, so that what is far below the maximum keeps its bits
    const float shift = FP16 ? DA_FP16_SHIFT : 0.f;
    const float slack = fminf(DA_SLACK / c, 1e30f);
    // Tile by tile, in three steps, each so far ahead of the next that nothing is waited for: the table's entries are
    // fetched, STAGES - 1 tiles before they are used; rows' addresses are made of them, by a lane a row; the rows are copied, STAGES - 1
    // tiles before they are multiplied.  (Warps are few, so a step's instructions and waits count: with addresses handed
    // round by shuffles and entries waited for, 64 ragged sequences of d = 64 took 40 us instead of 33.)
    Tiles rs = at, pg = at;  // the next tile whose addresses are made, and whose entries are fetched
    bool resolving = true, looking = true, bad = false;
    int page_in = 0, page_out = 0, buf = 0, fresh_in = 0, fresh_out = 0;
    auto turn = [](int &i, int n) { i = i + 1 == n ? 0 : i + 1; };
    auto step = [&](Tiles &g, bool &more) {
        if (++g.t == g.t_end) more = next(g);
    };
    auto entry = [&](const Tiles &g, int slot) { return a.kv.table + (long long)g.b * a.kv.max_pages + page_index(a.kv, slot); };
    auto look_up = [&]() {
        if (!looking) return;
        const int slot = pg.t * DA_SLOTS + lane;
        if (lane < DA_SLOTS && slot < pg.n) cp_async4(smem_u32(&rings.page[page_in][lane]), entry(pg, slot));
        turn(page_in, S::STAGES);
        step(pg, looking);
    };
    // Addresses of the tile at rs into row[to]; page: the entry of slot lane.
    auto resolve = [&](int page, int to) {
        const int slot = rs.t * DA_SLOTS + lane;
        const bool real = slot < rs.n, ok = real && (unsigned)page < (unsigned)a.kv.n_pages;
        if (lane < DA_SLOTS) {
            bad |= real && !ok;
            const long long off = page * a.kv.stride_page + rs.h * a.kv.stride_head +
                                  (slot - page_index(a.kv, slot) * a.kv.page_size) * a.kv.stride_slot;
            ulonglong2 at_row;
            at_row.x = reinterpret_cast<unsigned long long>(ok ? a.kv.k + off : reinterpret_cast<const uint16_t *>(zero_row));
            at_row.y = reinterpret_cast<unsigned long long>(ok ? a.kv.v + off : reinterpret_cast<const uint16_t *>(zero_row));
            if (append && slot == rs.n - 1) {
                const long long src = rs.b * a.new_stride + rs.h * D;
                at_row.x = reinterpret_cast<unsigned long long>(a.k_new + src);
                at_row.y = reinterpret_cast<unsigned long long>(a.v_new + src);
                rings.fresh[fresh_in].off = ok ? off : -1;
                if (a.new_pos) cp_async4(smem_u32(&rings.fresh[fresh_in].pos), a.new_pos + rs.b);
            }
            rings.row[to][lane] = at_row;
        }
        turn(fresh_in, S::STAGES + 1);
        step(rs, resolving);
    };
    // Copies the tile of row[from] into a stage: a lane takes 16-byte pieces `piece`, `piece` + LPR, ... of rows r0, r0 + 32 / LPR, ...
    // Eight lanes take a whole line together; rows of d = 64 have one, and four lanes spare instructions (64 ragged
    // sequences 31.9 us instead of 33.0; at d = 128 they make 128 x 1024 slower, 123 us instead of 93).
    constexpr int LPR = D == 64 ? 4 : 8, PIECES = CPR / LPR;
    const int piece = lane % LPR, r0 = lane / LPR;
    auto issue = [&](int from, int stage) {
        const uint32_t st = ring + stage * S::UNIT;
#pragma unroll
        for (int x = 0; x < DA_SLOTS * LPR / 32; ++x) {
            const int r = r0 + x * (32 / LPR);
            const ulonglong2 p = rings.row[from][r];
            const uint4 *ks = reinterpret_cast<const uint4 *>(p.x) + piece, *vs = reinterpret_cast<const uint4 *>(p.y) + piece;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const uint32_t dst = st + r * (D * 2) + (((i * LPR + piece) ^ (r & 7)) << 4);
                cp_async16_at(dst, ks + i * LPR);
                cp_async16_at(dst + DA_SLOTS * D * 2, vs + i * LPR);
            }
        }
    };
    // The new token's row joins the cache (nobody reads it there in this call), from the stage it was copied to.
    auto store_new = [&](const Tiles &g, int stage) {
        const long long o = rings.fresh[fresh_out].off;
        const int r = (g.n - 1) & 15;
        if (o >= 0)
            for (int i = lane; i < 2 * CPR; i += 32) {
                const int cc = i % CPR;
                uint16_t *to = const_cast<uint16_t *>(i < CPR ? a.kv.k : a.kv.v) + o + cc * 8;
                const uint32_t from = ring + stage * S::UNIT + (i < CPR ? 0 : DA_SLOTS * D * 2) + r * (D * 2) + ((cc ^ (r & 7)) << 4);
                *reinterpret_cast<float4 *>(to) = ld_shared_v4(from);
            }
        if (o >= 0 && lane == 0 && a.new_pos && a.kv.positions)
            a.kv.positions[((long long)g.b * a.kv.hkv + g.h) * a.kv.cap + g.n - 1] = rings.fresh[fresh_out].pos;
    };
    // Slots of pages outside the cache take no part (looked up again: an error path).
    auto mask_bad = [&](const Tiles &g, float (&s)[NT][4]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int slot = g.t * DA_SLOTS + (lane >> 2) + half * 8;
            if (slot >= g.n || (unsigned)page_of(a, g.b, slot) < (unsigned)a.kv.n_pages) continue;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][2 * half] = s[nt][2 * half + 1] = -INFINITY;
            if (!a.scores) continue;
            const int j = g.ch * HEADS + (lane & 3) * 2;
            float *dst = a.scores + ((long long)g.b * a.hq + g.h * a.group + j) * a.score_pitch + slot;
#pragma unroll 1
            for (int i = 0; i < 2 * NT; ++i)  // (heads 8 nt + e of the chunk)
                if (j + (i >> 1) * 8 + (i & 1) < a.group) dst[((i >> 1) * 8 + (i & 1)) * a.score_pitch] = -INFINITY;
        }
    };
    // a row's queries as B operands: head 8 nt + lane / 4, dims 16 ks + 2 (lane % 4) and the next, and 8 further on
    uint32_t qn[Q_AHEAD ? KS : 1][NT][2], qf[KS][NT][2];
    auto load_q = [&](const Tiles &g, auto &q_to) {
        const uint16_t *q = a.q + g.b * a.q_stride + (long long)(g.h * a.group + g.ch * HEADS) * D;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int j = nt * 8 + (lane >> 2);
            const bool real = g.ch * HEADS + j < a.group;
            const uint32_t *src = reinterpret_cast<const uint32_t *>(q + j * D + (lane & 3) * 2);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q_to[ks][nt][0] = real ? src[ks * 8] : 0u;
                q_to[ks][nt][1] = real ? src[ks * 8 + 4] : 0u;
            }
        }
    };

    // The first tiles' entries are fetched together, before any tile is copied.
    int to_issue = 0;  // tiles with addresses that have not been copied
    {
        int pages[S::STAGES];
#pragma unroll
        for (int s = 0; s < S::STAGES; ++s)
            if (looking) {
                const int slot = pg.t * DA_SLOTS + lane;
                pages[s] = lane < DA_SLOTS && slot < pg.n ? *entry(pg, slot) : -1;
                step(pg, looking);
            }
#pragma unroll
        for (int s = 0; s < S::STAGES; ++s) {
            if (resolving) {
                resolve(pages[s], s & 1);
                ++to_issue;
            }
            __syncwarp();
            if (s < S::STAGES - 1) {
                if (to_issue > 0) {
                    issue(s & 1, s);
                    --to_issue;
                }
                look_up();
                cp_async_commit();
            }
        }
    }
    buf = (S::STAGES - 1) & 1;
    int stage_in = S::STAGES - 1, stage = 0;
    if constexpr (Q_AHEAD) load_q(at, qn);

    float o[KS][NT][4], m[NT][2], l[NT][2];
    bool fresh = true;
    int t0 = 0;
    // lane constants of the fragments' addresses
    const int k_row = (lane & 7) + ((lane >> 3) & 1) * 8, k_c = lane >> 4;
    const int v_row = (lane & 7) + (lane >> 4) * 8, v_c = (lane >> 3) & 1;
    for (bool going = true; going;) {
        if (fresh) {
            fresh = false;
            t0 = at.t;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    o[ks][nt][0] = o[ks][nt][1] = o[ks][nt][2] = o[ks][nt][3] = 0.f;
                }
            }
            if constexpr (Q_AHEAD) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) qf[ks][nt][0] = qn[ks][nt][0], qf[ks][nt][1] = qn[ks][nt][1];
                Tiles after = at;
                if (next(after)) load_q(after, qn);
            } else {
                load_q(at, qf);
            }
        }
        cp_async_wait<S::STAGES - 2>();
        __syncwarp();  // everybody's copies are there, and everybody is done with the stage that is filled next
        if (to_issue > 0) {
            issue(buf, stage_in);
            turn(stage_in, S::STAGES);
            buf ^= 1;
            --to_issue;
        }
        if (resolving) {
            resolve(lane < DA_SLOTS ? rings.page[page_out][lane] : -1, buf);
            turn(page_out, S::STAGES);
            ++to_issue;
        }
        look_up();
        cp_async_commit();
        if (append && at.t == at.tiles - 1 && at.ch == 0) store_new(at, stage);
        turn(fresh_out, S::STAGES + 1);
        const uint32_t kst = ring + stage * S::UNIT, vst = kst + DA_SLOTS * D * 2;
        turn(stage, S::STAGES);

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
        if (slot >= at.n)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = -INFINITY;
        if (slot + 8 >= at.n)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][2] = s[nt][3] = -INFINITY;
        if (a.scores) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = at.ch * HEADS + nt * 8 + (lane & 3) * 2 + e;
                    if (j < a.group) {
                        float *dst = a.scores + ((long long)at.b * a.hq + at.h * a.group + j) * a.score_pitch + slot;
                        dst[0] = s[nt][e];
                        dst[8] = s[nt][2 + e];
                    }
                }
        }
        // m follows the maximum only where a score is above it by more than the slack: what p exceeds 1 by (a factor of 16)
        // fp32 sums and P's halves have room for, and tiles in which nothing has to be done need no exchange.
        bool grew = bad;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) grew |= s[nt][e] > m[nt][e & 1] + slack;
        if (__any_sync(0xffffffffu, grew)) {
            if (__any_sync(0xffffffffu, bad)) mask_bad(at, s);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(s[nt][e], s[nt][2 + e]);
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    x = fmaxf(x, m[nt][e]);
                    // (a maximum of -inf goes with a sum of 0: any finite factor will do)
                    const float f = x > m[nt][e] ? ex2((m[nt][e] - x) * c) : 1.f;
                    m[nt][e] = x;
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
        if (++at.t == at.t_end) {
            fresh = true;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
                }
            leave(at, t0, m, l, o);
            going = next(at);
        }
    }
    return __any_sync(0xffffffffu, bad);
}

// 1 / sum; 0 for a row without anything, NaN for NaN
__device__ __forceinline__ float inverse(float sum) { return sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum); }
// ln of the sum, whose terms carry the factor of P's scale
template <bool FP16>
__device__ __forceinline__ float log_sum(float sum) { return logf(FP16 ? sum * 0x1p-10f : sum); }

// The list, a stretch a warp.
template <bool FP16, int D, int NT>
__global__ void __launch_bounds__(DA_WARPS * 32) k_decode_split(const DecodeArgs a) {
    using S = DaShape<D>;
    constexpr int HEADS = 8 * NT, KS = D / 16;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) Rings<S::STAGES> rings[DA_WARPS];
    const int B = a.kv.B, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int *first = reinterpret_cast<int *>(smem + S::RING), *len = first + B + 1;
    pdl_launch();
    tile_lists<DA_ROW_TILES>(a, first, len);
    const int chunks = (a.group + HEADS - 1) / HEADS, HC = a.kv.hkv * chunks;
    const int count = first[B] * HC, workers = workers_of(a, count);
    const int w = warp * gridDim.x + blockIdx.x;  // neighbours in the list on different SMs
    if (count == 0 || w >= workers) return;
    Tiles at;
    if (!at.seek(first_of(w, count, workers), first_of(w + 1, count, workers), first, len, B, a.kv.hkv, chunks)) {
        if (lane == 0) a.worker_bad[w] = 0;
        return;
    }
    const bool bad = attend<FP16, D, NT>(
        a, smem_u32(smem) + warp * S::STAGES * S::UNIT, rings[warp], at,
        [&](Tiles &g) { return g.next(first, len, B, a.kv.hkv, chunks); },
        [&](const Tiles &g, int t0, const float (&m)[NT][2], const float (&l)[NT][2], const float (&o)[KS][NT][4]) {
            const int h = g.h, ch = g.ch, d0 = lane >> 2;
            const bool whole = t0 == 0 && g.t_end == g.tiles;
            const long long part = (long long)w * 2 + (t0 == 0 ? 1 : 0);  // (a stretch has one row begun before it, and one that goes on)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = nt * 8 + (lane & 3) * 2 + e;
                    if (ch * HEADS + j >= a.group) continue;
                    if (whole) {
                        const long long row = (long long)g.b * a.hq + h * a.group + ch * HEADS + j;
                        const float inv = inverse(l[nt][e]);
                        uint16_t *dst = a.out + row * D + d0;
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            dst[ks * 16] = round16<FP16>(o[ks][nt][e] * inv);
                            dst[ks * 16 + 8] = round16<FP16>(o[ks][nt][2 + e] * inv);
                        }
                        if (d0 == 0) {
                            a.row_ml[row] = make_float2(m[nt][e], inv);
                            if (a.lse) a.lse[row] = m[nt][e] * a.scale + log_sum<FP16>(l[nt][e]);
                        }
                    } else {
                        if (d0 == 0) a.part_ml[part * HEADS + j] = make_float2(m[nt][e], l[nt][e]);
                        float *dst = a.part_o + (part * HEADS + j) * D + d0;
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            dst[ks * 16] = o[ks][nt][e];
                            dst[ks * 16 + 8] = o[ks][nt][2 + e];
                        }
                    }
                }
        });
    if (lane == 0) a.worker_bad[w] = bad;  // (k_decode_join reports it: the status word has one writer)
}

// Lengths outside the table, over the whole CTA.
__device__ __forceinline__ bool bad_length(const DecodeArgs &a) {
    bool bad = false;
    for (int b = threadIdx.x; b < a.kv.B; b += blockDim.x) bad |= !length_ok(a, a.kv.lens[b]);
    return __syncthreads_or(bad);
}

// Small calls: a cluster of C CTAs a (sequence, KV head).  Its warps take the row's tiles in equal parts; each CTA joins its
// four warps' results in shared memory and hands maxima and sums to every CTA, and each piece of the outputs to the CTA
// that finishes it (stores into distributed shared memory, which nobody waits for, where loads from it would each take
// 0.8 us).  Last, warps add the weights of their own slots.  (Bound to the CTAs an SM that shared memory allows: left to itself ptxas takes
// 72 to 128 registers for d = 64 and 128, and 4 x 900 tokens of d = 64 take 7.6 us instead of 7.1, the ragged batch of 8 with weights 15.4 instead of 14.6.)
template <bool FP16, int D, int NT>
__global__ void __launch_bounds__(DA_WARPS * 32, DaShape<D>::CTAS) k_decode_cluster(const DecodeArgs a, int C) {
    using S = DaShape<D>;
    constexpr int HEADS = 8 * NT, KS = D / 16, PITCH = D + 4, THREADS = DA_WARPS * 32, D4 = D / 4;
    static_assert(HEADS * PITCH * 4 <= S::STAGES * S::UNIT, "a warp's results lie in its ring");
    static_assert(KV_MAX_BATCH * 4 <= S::RING, "the status word's CTA keeps a number a sequence in the rings' place");
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) Rings<S::STAGES> rings[DA_WARPS];
    __shared__ float2 warp_ml[DA_WARPS][HEADS], row_ml[HEADS];
    __shared__ __align__(8) float2 every[DA_CLUSTER][HEADS];  // maximum and sum of each CTA
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x % C, row = blockIdx.x / C;
    if (row == a.kv.B * a.kv.hkv) {  // one cluster more: the call's status word has one writer
        if (rank != 0) return;
        const bool length = bad_length(a);
        const bool page = any_bad_page<THREADS>(a.kv, reinterpret_cast<int *>(smem), [&](int s) { return attended(a, s); });
        if (tid == 0) *a.status = length ? DEV_BAD_POSITION : page ? DEV_BAD_PAGE : DEV_OK;
        return;
    }
    cluster_arrive();  // (this CTA runs: others may store into its shared memory)
    const int b = row / a.kv.hkv, h = row - b * a.kv.hkv, n = attended(a, b), G = a.group;
    const float c = a.scale * 1.4426950408889634f, shift = FP16 ? DA_FP16_SHIFT : 0.f;
    uint8_t *ring = smem + warp * S::STAGES * S::UNIT;
    float *mine = reinterpret_cast<float *>(ring), *got = reinterpret_cast<float *>(smem + S::RING);  // got[C][own pieces][4]
    Tiles at;
    at.b = b;
    at.h = h;
    at.ch = 0;
    at.n = n;
    at.tiles = (n + DA_SLOTS - 1) / DA_SLOTS;
    const int w = rank * DA_WARPS + warp, W = C * DA_WARPS;
    at.t = first_of(w, at.tiles, W);
    at.t_end = first_of(w + 1, at.tiles, W);
    const int slot0 = at.t * DA_SLOTS, slot1 = min(n, at.t_end * DA_SLOTS);
    float *wt = a.kv.weights + ((long long)b * a.kv.hkv + h) * a.kv.cap;
    if (a.accumulate && slot0 + lane * 32 < slot1) prefetch_l2(wt + slot0 + lane * 32);
    const int page_new = a.accumulate && a.k_new && n > 0 ? page_of(a, b, n - 1) : -1;  // (a new token's; used at the end)
    if (at.t < at.t_end) {
        attend<FP16, D, NT>(
            a, smem_u32(ring), rings[warp], at, [&](Tiles &) { return false; },
            [&](const Tiles &, int, const float (&m)[NT][2], const float (&l)[NT][2], const float (&o)[KS][NT][4]) {
                cp_async_wait_all();
                __syncwarp();  // (the ring is free)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int j = nt * 8 + (lane & 3) * 2 + e, d0 = lane >> 2;
                        if (d0 == 0) warp_ml[warp][j] = make_float2(m[nt][e], l[nt][e]);
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            mine[j * PITCH + ks * 16 + d0] = o[ks][nt][e];
                            mine[j * PITCH + ks * 16 + d0 + 8] = o[ks][nt][2 + e];
                        }
                    }
            });
    } else if (lane < HEADS) {
        warp_ml[warp][lane] = make_float2(-INFINITY, 0.f);
    }
    __syncthreads();
    auto add = [](float4 &acc, float f, const float4 &x) {
        acc.x += f * x.x;
        acc.y += f * x.y;
        acc.z += f * x.z;
        acc.w += f * x.w;
    };
    // Piece p (a head's four dims) is finished by CTA p % C, as its piece p / C of `own`.
    const int pieces = G * D4, own = (pieces + C - 1) / C;
    cluster_wait();
    // (a part whose sum is 0 has no outputs, or was never written)
    for (int p = tid; p < pieces; p += THREADS) {
        const int j = p / D4, d4 = p % D4;
        float mx = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < DA_WARPS; ++i) mx = fmaxf(mx, warp_ml[i][j].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const float mu = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int i = 0; i < DA_WARPS; ++i) {
            const float2 x = warp_ml[i][j];
            if (x.y == 0.f) continue;
            const float f = ex2((x.x - mu) * c);
            sum += f * x.y;
            add(acc, f, *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem + i * S::STAGES * S::UNIT) + j * PITCH + d4 * 4));
        }
        st_cluster_v4(map_cta(smem_u32(got + (rank * own + p / C) * 4), p % C), acc);
        if (d4 < C) st_cluster_v2(map_cta(smem_u32(&every[rank][j]), d4), mx, sum);
    }
    cluster_sync();
    if (tid < G) {
        float mx = -INFINITY, sum = 0.f;
        for (int i = 0; i < C; ++i) mx = fmaxf(mx, every[i][tid].x);
        const float mu = mx == -INFINITY ? 0.f : mx;
        for (int i = 0; i < C; ++i) {
            const float f = every[i][tid].y == 0.f ? 0.f : ex2((every[i][tid].x - mu) * c);
            sum += f * every[i][tid].y;
            every[i][tid].x = f;
        }
        row_ml[tid] = make_float2(mu, inverse(sum));
        if (rank == 0 && a.lse) a.lse[(long long)b * a.hq + h * G + tid] = mx * a.scale + log_sum<FP16>(sum);
    }
    __syncthreads();
    for (int q = tid; q * C + rank < pieces; q += THREADS) {
        const int p = q * C + rank, j = p / D4, d4 = p % D4;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = 0; i < C; ++i) add(acc, every[i][j].x, *reinterpret_cast<const float4 *>(got + (i * own + q) * 4));
        const float inv = row_ml[j].y;
        uint2 r;
        r.x = pack2<FP16>(acc.x * inv, acc.y * inv);
        r.y = pack2<FP16>(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(a.out + ((long long)b * a.hq + h * G + j) * D + d4 * 4) = r;
    }
    if (a.accumulate) {
        const float *sc = a.scores + ((long long)b * a.hq + h * G) * a.score_pitch;
        const int fresh = (unsigned)page_new < (unsigned)a.kv.n_pages ? n - 1 : -1;
        for (int slot = slot0 + lane; slot < slot1; slot += 32) {
            float sum = slot == fresh ? 0.f : wt[slot];
#pragma unroll 8
            for (int j = 0; j < G; ++j) sum += ex2((sc[j * a.score_pitch + slot] - row_ml[j].x) * c + shift) * row_ml[j].y;
            wt[slot] = sum;
        }
    }
}

constexpr int DJ_THREADS = 256, DJ_CTAS = 2;

// Joins what several warps left of a row: out = sum_w f_w o_w / sum_w f_w l_w, f_w = exp(scale (m_w - max)).  TEAM threads a
// query head: the CTA where many warps share a row, a warp where rows are many.  Sequences without a slot get
// zeros.  A CTA an SM finds room beside k_decode_split's, so that all that does not depend on it is done when it ends.
template <bool FP16, int D, int NT, int TEAM>
__global__ void __launch_bounds__(DJ_THREADS) k_decode_join(const DecodeArgs a) {
    constexpr int HEADS = 8 * NT, TEAMS = DJ_THREADS / TEAM, L = D / 4 < TEAM ? D / 4 : TEAM, V = D / 4 / L, G = TEAM / L;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float red[2][DJ_THREADS / 32];
    __shared__ float4 sum_o[TEAM > 32 ? DJ_THREADS : 1];
    const int B = a.kv.B, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int *first = reinterpret_cast<int *>(smem), *len = first + B + 1;
    float *fac = reinterpret_cast<float *>(len + B);  // [TEAMS][workers]
    pdl_launch();
    tile_lists<DA_ROW_TILES>(a, first, len);
    const int chunks = (a.group + HEADS - 1) / HEADS, HC = a.kv.hkv * chunks;
    const int count = first[B] * HC, workers = workers_of(a, count);
    const float c = a.scale * 1.4426950408889634f;
    // the warps that share a row, and where one of them left it
    auto span = [&](int b, int h, int ch, int *w0) {
        const int per = first[b + 1] - first[b], tiles = per - DA_ROW_TILES;
        const long long at = (long long)first[b] * HC + (long long)(h * chunks + ch) * per + DA_ROW_TILES;
        *w0 = worker_at(at, count, workers);
        return worker_at(at + tiles - 1, count, workers) - *w0 + 1;
    };
    auto part_at = [&](int w0, int i, int j) { return ((long long)(w0 + i) * 2 + (i == 0)) * HEADS + j; };

    const bool length = blockIdx.x == 0 && bad_length(a);
    pdl_wait();
    if (blockIdx.x == 0) {
        bool page = false;
        if (count > 0)
            for (int w = tid; w < workers; w += DJ_THREADS) page |= a.worker_bad[w] != 0;
        page = __syncthreads_or(page);
        if (tid == 0) *a.status = length ? DEV_BAD_POSITION : page ? DEV_BAD_PAGE : DEV_OK;
    }
    const int rows = B * a.hq, team = tid / TEAM, me = tid % TEAM;
    float *f_team = fac + team * a.workers;
    auto team_sync = [&]() {
        if (TEAM > 32)
            __syncthreads();
        else
            __syncwarp();
    };
    for (int row = blockIdx.x * TEAMS + team; row < rows; row += gridDim.x * TEAMS) {
        const int b = row / a.hq, hq = row - b * a.hq, h = hq / a.group, g = hq - h * a.group;
        const int ch = g / HEADS, j = g - ch * HEADS;
        if (len[b] == 0) {
            for (int d = me; d < D; d += TEAM) a.out[(long long)row * D + d] = 0;
            if (me == 0 && a.lse) a.lse[row] = -INFINITY;
            continue;
        }
        int w0;
        const int nw = span(b, h, ch, &w0);
        if (nw == 1) continue;  // one warp did it all
        // the first outputs are asked for before their factors are known
        constexpr int U = V == 1 ? 8 : 4;
        const int d4 = me % L, grp = me / L;
        float4 x[U][V];
        auto load = [&](int i0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * G < nw)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        x[u][v] = *reinterpret_cast<const float4 *>(a.part_o + part_at(w0, i0 + u * G, j) * D + (v * L + d4) * 4);
        };
        load(grp);
        const float2 own = me < nw ? a.part_ml[part_at(w0, me, j)] : make_float2(-INFINITY, 0.f);
        float mx = own.x;
        for (int i = me + TEAM; i < nw; i += TEAM) mx = fmaxf(mx, a.part_ml[part_at(w0, i, j)].x);
        for (int s = 16; s; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
        team_sync();  // (what the row before left in shared memory has been read)
        if (TEAM > 32) {
            if (lane == 0) red[0][warp] = mx;
            __syncthreads();
            for (int i = 0; i < DJ_THREADS / 32; ++i) mx = fmaxf(mx, red[0][i]);
        }
        const float mu = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f;
        for (int i = me; i < nw; i += TEAM) {
            const float2 ml = i == me ? own : a.part_ml[part_at(w0, i, j)];
            const float f = ex2((ml.x - mu) * c);
            f_team[i] = f;
            sum += f * ml.y;
        }
        for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        if (TEAM > 32 && lane == 0) red[1][warp] = sum;
        team_sync();
        if (TEAM > 32) {
            sum = 0.f;
            for (int i = 0; i < DJ_THREADS / 32; ++i) sum += red[1][i];
        }
        float4 acc[V];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i0 = grp; i0 < nw; i0 += G * U) {
            if (i0 != grp) load(i0);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * G < nw) {
                    const float f = f_team[i0 + u * G];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        acc[v].x += f * x[u][v].x;
                        acc[v].y += f * x[u][v].y;
                        acc[v].z += f * x[u][v].z;
                        acc[v].w += f * x[u][v].w;
                    }
                }
        }
        if (TEAM > 32) {
            sum_o[tid] = acc[0];  // (V is 1)
            __syncthreads();
            if (grp == 0)
                for (int i = 1; i < G; ++i) {
                    const float4 y = sum_o[i * L + d4];
                    acc[0].x += y.x;
                    acc[0].y += y.y;
                    acc[0].z += y.z;
                    acc[0].w += y.w;
                }
        } else {
            for (int s = L; s < TEAM; s <<= 1) {
                acc[0].x += __shfl_xor_sync(0xffffffffu, acc[0].x, s);
                acc[0].y += __shfl_xor_sync(0xffffffffu, acc[0].y, s);
                acc[0].z += __shfl_xor_sync(0xffffffffu, acc[0].z, s);
                acc[0].w += __shfl_xor_sync(0xffffffffu, acc[0].w, s);
            }
        }
        const float inv = inverse(sum);
        if (grp == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                uint2 r;
                r.x = pack2<FP16>(acc[v].x * inv, acc[v].y * inv);
                r.y = pack2<FP16>(acc[v].z * inv, acc[v].w * inv);
                *reinterpret_cast<uint2 *>(a.out + (long long)row * D + (v * L + d4) * 4) = r;
            }
        if (me == 0) {
            a.row_ml[row] = make_float2(mx, inv);
            if (a.lse) a.lse[row] = mx * a.scale + log_sum<FP16>(sum);
        }
    }
}

constexpr int DW_THREADS = 256, DW_CTAS = 4;
constexpr int DW_ROW_TILES = 16;  // what a row costs a warp here, in tiles
constexpr int DW_VECS = 2;        // float4 of a lane and head at a time

// weights[b][h][slot] += what the heads of h's group give the slot; the new token's slot starts at 0.  A warp a stretch of a
// list of [sequence][KV head][tile].  (CTAs of the join that took stretches and joined the maxima and sums themselves did
// not have to wait for it, which saved 1.7 us of 101 on 131072 tokens; but each row cost a whole CTA 3 us: four sequences of 100
// to 60000 took 83 us instead of 69, eight 128 instead of 107.)
template <bool FP16>
__global__ void __launch_bounds__(DW_THREADS) k_decode_weights(const DecodeArgs a) {
    extern __shared__ __align__(128) uint8_t smem[];
    const int B = a.kv.B, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int *first = reinterpret_cast<int *>(smem), *len = first + B + 1;
    tile_lists<DW_ROW_TILES>(a, first, len);
    const int all = first[B] * a.kv.hkv, warps = gridDim.x * (DW_THREADS / 32), w = warp * gridDim.x + blockIdx.x;
    const float c = a.scale * 1.4426950408889634f, shift = FP16 ? DA_FP16_SHIFT : 0.f;
    Segment<DW_ROW_TILES> at;
    if (all == 0 || !at.seek(first_of(w, all, warps), first_of(w + 1, all, warps), first, len, B, a.kv.hkv, 1)) {
        pdl_wait();  // (a kernel behind this one counts on the join's end as well)
        return;
    }
    constexpr int STEP = 128 * DW_VECS;
    float have[DW_VECS][4];
    auto load_weights = [&](int s0, int s1) {
        const float *wt = a.kv.weights + ((long long)at.b * a.kv.hkv + at.h) * a.kv.cap;
#pragma unroll
        for (int v = 0; v < DW_VECS; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = s0 + v * 128 + lane * 4 + i;
                have[v][i] = slot < s1 ? wt[slot] : 0.f;
            }
    };
    load_weights(at.t * DA_SLOTS, min(at.n, at.t_end * DA_SLOTS));  // (no kernel of this call has written them)
    pdl_wait();
    bool begun = true;
    do {
        const int s0 = at.t * DA_SLOTS, s1 = min(at.n, at.t_end * DA_SLOTS);
        float *wt = a.kv.weights + ((long long)at.b * a.kv.hkv + at.h) * a.kv.cap;
        const int page_new = a.k_new && s1 == at.n ? page_of(a, at.b, at.n - 1) : -1;  // (used when the sums are there)
        for (int g0 = 0; g0 < a.group; g0 += 32) {
            const int heads = min(32, a.group - g0);
            const long long row = (long long)at.b * a.hq + at.h * a.group + g0;
            float2 ml = make_float2(0.f, 0.f);  // maximum and inverse sum of head g0 + lane
            if (lane < heads) ml = a.row_ml[row + lane];
            if (ml.x == -INFINITY) ml.x = 0.f;
            for (int s = s0; s < s1; s += STEP) {
                if (!begun || s != s0 || g0 != 0) load_weights(s, s1);
                float sum[DW_VECS][4] = {};
#pragma unroll 4
                for (int g = 0; g < heads; ++g) {
                    const float *sc = a.scores + (row + g) * a.score_pitch;  // (16-byte aligned; whole tiles can be read)
                    const float m = __shfl_sync(0xffffffffu, ml.x, g), inv = __shfl_sync(0xffffffffu, ml.y, g);
#pragma unroll
                    for (int v = 0; v < DW_VECS; ++v) {
                        const int slot = s + v * 128 + lane * 4;
                        if (slot < s1) {
                            const float4 x = *reinterpret_cast<const float4 *>(sc + slot);
                            sum[v][0] += ex2((x.x - m) * c + shift) * inv;
                            sum[v][1] += ex2((x.y - m) * c + shift) * inv;
                            sum[v][2] += ex2((x.z - m) * c + shift) * inv;
                            sum[v][3] += ex2((x.w - m) * c + shift) * inv;
                        }
                    }
                }
                const int fresh = g0 == 0 && (unsigned)page_new < (unsigned)a.kv.n_pages ? at.n - 1 : -1;
#pragma unroll
                for (int v = 0; v < DW_VECS; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int slot = s + v * 128 + lane * 4 + i;
                        if (slot < s1) wt[slot] = (slot == fresh ? 0.f : have[v][i]) + sum[v][i];
                    }
            }
        }
        begun = false;
    } while (at.next(first, len, B, a.kv.hkv, 1));
}

// Kernel attributes, set for the current device before any launch there; *done is the device they were last set for.
template <typename K>
cudaError_t configure(K *kernel, size_t smem, int *done, int *most_cluster = nullptr) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || *done == dev) return e;
    const void *f = reinterpret_cast<const void *>(kernel);
    e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    // (kernels with another division of an SM's memory do not run beside each other)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess && most_cluster) {
        e = cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess) *most_cluster = largest_cluster(f, DA_WARPS * 32, smem, DA_CLUSTER) < DA_CLUSTER ? 8 : DA_CLUSTER;
    }
    if (e == cudaSuccess) *done = dev;
    return e;
}

template <bool FP16, int D, int NT, int TEAM>
cudaError_t launch_join(DecodeArgs &a, cudaStream_t st) {
    static thread_local int done = -1;
    const size_t lists = (2 * (size_t)a.kv.B + 1) * 4, most = (2 * KV_MAX_BATCH + 1 + (DJ_THREADS / TEAM) * KV_MAX_WORKERS) * 4;
    const size_t facs = (size_t)(DJ_THREADS / TEAM) * a.workers * 4;
    cudaError_t e = configure(k_decode_join<FP16, D, NT, TEAM>, most, &done);
    if (e != cudaSuccess) return e;
    const int teams = DJ_THREADS / TEAM, rows = a.kv.B * a.hq, sms = gemm_ctas();
    e = launch_pdl(k_decode_join<FP16, D, NT, TEAM>, std::min((rows + teams - 1) / teams, sms * DJ_CTAS), DJ_THREADS, lists + facs, st, a);
    if (e != cudaSuccess || !a.accumulate) return e;
    static thread_local int done_w = -1;
    if ((e = configure(k_decode_weights<FP16>, (2 * KV_MAX_BATCH + 1) * 4, &done_w)) != cudaSuccess) return e;
    return launch_pdl(k_decode_weights<FP16>, sms * DW_CTAS, DW_THREADS, lists, st, a);
}

// CTAs of a (sequence, KV head)'s cluster, or 0 where the list of tiles is the better way: clusters where all of them run at
// once and no warp has more than DA_CLUSTER_TILES tiles. (Clusters and list, 8 KV heads of d = 128: 1 x 2048 6.3 us and 9.0,
// 1 x 8192 11.8 and 14.0, 8 x 1757 13.9 and 16.8; a ragged batch of 8, where the longest row sets the time, 10.7 and 11.9, with
// weights 14.2 and 16.6; 4 x 900 of d = 64 with weights 7.1 and 13.3. Longer rows than the bound's spread better over the list.)
int pick_cluster(const DecodeArgs &a, int ctas, int most) {
    const long long rows = (long long)a.kv.B * a.kv.hkv, tiles = (a.kv.cap + DA_SLOTS - 1) / DA_SLOTS;
    if (a.group > 16 || rows > ctas) return 0;
    int C = 1;
    while (C < most && rows * C * 2 <= ctas && C * DA_WARPS * 2 <= tiles) C *= 2;
    return tiles <= (long long)C * DA_WARPS * DA_CLUSTER_TILES ? C : 0;
}

template <bool FP16, int D, int NT>
cudaError_t launch(DecodeArgs &a, cudaStream_t st) {
    using S = DaShape<D>;
    static thread_local int done_c = -1, most = 8;
    constexpr size_t C_SMEM = S::RING + 8 * NT * D * 4 + DA_CLUSTER * 16;  // (rings, pieces of outputs)
    cudaError_t e = configure(k_decode_cluster<FP16, D, NT>, C_SMEM, &done_c, &most);
    if (e != cudaSuccess) return e;
    if (const int C = pick_cluster(a, gemm_ctas() * S::CTAS, most)) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((a.kv.B * a.kv.hkv + 1) * C));
        cfg.blockDim = dim3(DA_WARPS * 32);
        cfg.dynamicSmemBytes = C_SMEM;
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)C;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, k_decode_cluster<FP16, D, NT>, static_cast<const DecodeArgs>(a), C);
    }
    const size_t lists = (2 * (size_t)a.kv.B + 1) * 4;
    static thread_local int done = -1;
    e = configure(k_decode_split<FP16, D, NT>, S::RING + (2 * KV_MAX_BATCH + 1) * 4, &done);
    if (e != cudaSuccess) return e;
    const int grid = gemm_ctas() * S::CTAS;
    a.workers = std::min(grid * DA_WARPS, KV_MAX_WORKERS);
    k_decode_split<FP16, D, NT><<<grid, DA_WARPS * 32, S::RING + lists, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    // Where a row is shared by many warps, a CTA joins it, else a warp (8 KV heads of d = 128: 1 x 131072 89 us and 99, 4 x 32768
    // 88 and 92, a ragged batch of 8 95 and 100, but 16 x 8192 both 89, 64 ragged rows of d = 64 40 and 32).
    const int rows = a.kv.B * a.kv.hkv * ((a.group + 8 * NT - 1) / (8 * NT));
    return rows * 16 <= a.workers ? launch_join<FP16, D, NT, DJ_THREADS>(a, st) : launch_join<FP16, D, NT, 32>(a, st);
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
    p->worker_bad = take((size_t)KV_MAX_WORKERS * sizeof(int));
    p->row_ml = take((size_t)kv.B * hq * sizeof(float2));
    p->score_pitch = (kv.cap + DA_SLOTS - 1) / DA_SLOTS * DA_SLOTS;
    p->scores = take(accumulate ? (size_t)kv.B * hq * p->score_pitch * sizeof(float) : 0);
    p->total = off;
    // places of the list are counted in 32 bits
    return (long long)kv.B * ((kv.cap + DA_SLOTS - 1) / DA_SLOTS + DW_ROW_TILES) * kv.hkv * ((group + heads - 1) / heads) < (1ll << 31);
}

cudaError_t launch_decode_attention(DecodeArgs &a, cudaStream_t st) {
    return a.fp16 ? launch_t<true>(a, st) : launch_t<false>(a, st);
}

}  // namespace pbd
