// pk_attend_chunk.cu -- attention of chunks of new tokens over the 4-bit pages of
// their requests, with or without a sliding window (pk_attend_chunk).
//
// out = v_scale sum_j p_j V_j / sum_j p_j over the keys j that a query sees, p_j =
// 2^(s_j - ref), s_j = scale k_scale log2(e) q . K_j; K and V are code * scale, which
// has six significant bits: exact in a half and in a bfloat16.  K takes the type of
// q, which the matrix instruction wants, V and the weights are halves for either.
// ref moves as in pk_attend_prompt.cu: only when a tile's weights of a row sum to
// more than 2^15.
//
// Keys are counted without the gap that a window leaves: of a tile of queries the
// granules (16 tokens) of the first tokens and those from the first query's window
// on are one list, cut into tiles of 128 keys.  In its places a query sees last and
// below, down to low, and those before `sinks`.
#include <cuda.h>
#include <cuda_runtime.h>
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "pk_attend.cuh"
#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"
#include "pk_tcgen05.cuh"
#include "pk_tma.cuh"

namespace {

constexpr int kRows = 128;      // (query token, head of the group) rows of a tile; an item is two tiles
constexpr int kKeys = 128;      // keys of a tile
constexpr int kThreads = 512;
constexpr float kTop = 32768.0f;     // a tile's weights of a row sum to no more, so each fits a half (65504)
constexpr float kBase = 4.0f;        // the largest weight when the reference moves: 2^kBase, so 128 stay below 2^11
constexpr float kFar = 16777216.0f;  // scores (times log2 e) from here on are further apart than a weight's exponents:
                                     // one 32-bit reference cannot lie kBase below one
constexpr int kPlanThreads = 1024;

struct Args {
    const uint8_t *pool;
    uint64_t page_bytes, n_slots, page_stride, positions;  // positions: that a request can hold
    uint32_t page_grans;  // granules of one head in a page
    const int64_t *q_off;
    const int32_t *kv_len;
    const uint32_t *pages;
    uint32_t R, q_heads, kv_heads, group;
    uint64_t n_q;
    uint32_t tile_tokens, tile_heads, chunks;  // of a tile; tiles that it takes for a group's heads
    uint32_t window, sinks, sink_grans;        // window 0: none
    float scale2, v_scale;                     // scale * k_scale * log2 e
    uint16_t *out;
    int64_t o_ts, o_hs;
    bool wide_out;  // every 16 values of out start on 32 bytes
    float *lse;
    // Keys of an item are cut into pieces of about `split` tiles, so that few rows over many keys fill the GPU.
    uint32_t target, least;  // pieces that a call is cut into, about (0: none is cut), and tiles of one at least
    uint64_t *plan;          // [0]: split; [1 + r]: items of one KV head in the requests before r
    bool listed;             // more than 32 requests: k_chunk_plan made the plan
    uint32_t most_items;     // no call has more
    float4 *part_ml;         // [item][2][128]: (ref, fine, sum) of a piece's rows
    float *part_o;           // [item][2][128][D]
    int32_t *status;
};

__device__ __forceinline__ bool bad_offsets(int64_t qa, int64_t qb, uint64_t n_q) {
    return qa < 0 || qb < qa || (uint64_t)qb > n_q;
}

// The length of a request, 0 when it is out of range.
__device__ __forceinline__ int32_t good_length(const Args &a, int32_t len) {
    return len < 0 || (uint64_t)len > a.positions ? 0 : len;
}

// Items of one KV head in a request of n queries, before they are cut.
__device__ __forceinline__ uint32_t units_of(const Args &a, int64_t n) {
    return ((uint32_t)n + 2 * a.tile_tokens - 1) / (2 * a.tile_tokens) * a.chunks;
}

// Key tiles of a request's last queries, or a few more.
__device__ __forceinline__ uint32_t tiles_of(const Args &a, int32_t len) {
    uint64_t grans = ((uint64_t)len + 15) / 16;
    if (a.window) grans = min(grans, (uint64_t)a.sink_grans + ((uint64_t)a.window + 2 * a.tile_tokens + 14) / 16 + 1);
    return (uint32_t)((grans + 7) / 8);
}

// Tiles of a piece, from the sum over the items of their requests' tiles; pieces of an item.
__device__ __forceinline__ uint32_t split_of(const Args &a, uint64_t total) {
    if (a.target == 0) return 0x7fffffff;
    return (uint32_t)max((total + a.target - 1) / a.target, (uint64_t)a.least);
}
__device__ __forceinline__ uint32_t pieces_of(uint32_t tiles, uint32_t split) {
    return tiles <= split ? 1 : (tiles + split - 1) / split;
}

// The plan of more than 32 requests; of no items where an offset is out of order or range.
__global__ void __launch_bounds__(kPlanThreads) k_chunk_plan(const Args a) {
    __shared__ uint64_t warp_sum[32];
    __shared__ uint32_t bad;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    if (tid == 0) bad = 0;
    const int64_t *q_off = a.q_off;
    const int32_t *kv_len = a.kv_len;
    uint64_t *plan = a.plan;
    pk::pdl_wait(q_off, kv_len, plan);
    pk::pdl_launch_dependents();
    __syncthreads();
    uint32_t split = 0x7fffffff;
    for (int pass = a.target ? 0 : 1; pass < 2; ++pass) {  // the sum of the tiles, then the items
        uint64_t base = 0;
        for (uint64_t r0 = 0; r0 < a.R; r0 += kPlanThreads) {
            const uint64_t r = r0 + tid;
            uint64_t n = 0;
            if (r < a.R) {
                const int64_t qa = __ldcg(q_off + r), qb = __ldcg(q_off + r + 1);
                const int32_t l = __ldcg(kv_len + r), len = good_length(a, l);
                if (pass && l != len) pk::set_status(a.status, PK_ERR_ARG);
                if (bad_offsets(qa, qb, a.n_q))
                    bad = 1;
                else
                    n = (uint64_t)units_of(a, qb - qa) * (pass ? pieces_of(tiles_of(a, len), split) : a.kv_heads * tiles_of(a, len));
            }
            uint64_t scan = n;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint64_t o = __shfl_up_sync(0xffffffffu, scan, d);
                if (lane >= (uint32_t)d) scan += o;
            }
            if (lane == 31) warp_sum[wid] = scan;
            __syncthreads();
            uint64_t before = base, total = 0;
            for (uint32_t w = 0; w < kPlanThreads / 32; ++w) {
                if (w < wid) before += warp_sum[w];
                total += warp_sum[w];
            }
            if (pass && r < a.R) plan[2 + r] = before + scan;
            base += total;
            __syncthreads();
        }
        if (pass == 0) split = split_of(a, base);
    }
    if (tid == 0) {
        plan[0] = split;
        plan[1] = 0;
    }
    if (bad) {
        for (uint64_t r = tid; r <= a.R; r += kPlanThreads) plan[1 + r] = 0;
        if (tid == 0) pk::set_status(a.status, PK_ERR_ARG);
    }
}

// Shared memory of a CTA, from a 1024-byte boundary: Q (two tiles), the ring of K and V tiles in 16 bits, the ring of
// granules as they lie in the pages, then Small.
template <int D>
struct Layout {
    static constexpr uint32_t kTile = 128 * D * 2;  // 128 rows; blocks of [128][64] values, 16 KB each
    static constexpr uint32_t kStages = D == 128 ? 3 : 8;
    static constexpr uint32_t kGran = pk::Granule<D>::kBytes;
    static constexpr uint32_t kGrans = D == 128 ? 28 : 32;
    static constexpr uint32_t kRing = 2 * kTile;
    static constexpr uint32_t kGranRing = kRing + kStages * kTile;
    static constexpr uint32_t kBytes = kGranRing + kGrans * kGran;
};

constexpr uint32_t kNotes = 8;       // key tiles whose notes are kept: they are read before the ring has gone round
constexpr uint32_t kMarked = 1, kLost = 2;
constexpr uint32_t kMakers = 6;      // warps that make tiles of granules

// A softmax warp's tile of the present item.
struct TileOf {
    int32_t causal, hides[2];  // from the first on some query does not see some key; between the others too
    int32_t off, base;         // position of the request's first query; what a position is more than its place in the piece
    int32_t sinks, tok0, row0, head0, n_all;
    int64_t part;              // where the piece's rows go; -1: the item is not cut
};

struct Small {
    uint64_t full[8], empty[8];             // ring stages: tile ready; no longer read
    uint64_t gran_full[32], gran_empty[32]; // the same of granules
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], p_ready[2], o_done[2];
    uint64_t over;                          // every product that was issued is done (a matrix warp that gave up)
    uint32_t tmem, abort;
    int32_t work[8][2];                     // by item with keys: key tiles of its two tiles, for the matrix warp; 0, 0 ends it
    uint8_t gran_lost[32];                  // what stands in a granule's place is another request's
    uint32_t split;
    alignas(2) uint8_t flags[kNotes][2];    // by key tile and half of its keys: kMarked, kLost
    uint8_t marked[kNotes][128];            // by key, where kMarked: blocks of V that are NaN (0 stands in the tile)
    uint32_t item_end[32];                  // up to 32 requests: items of one KV head in those up to each, and what they are
    int32_t q_start[32], q_len[32], len[32];
    TileOf tile[8];
};

// Up to 32 requests every CTA makes the plan itself, a lane a request, and keeps it in shared memory.
__device__ __forceinline__ void plan_here(const Args &a, Small &sm, const int64_t *q_off, const int32_t *kv_len) {
    const uint32_t lane = threadIdx.x & 31;
    int64_t qa = 0, qb = 0;
    int32_t len = 0;
    if (lane < a.R) {
        qa = __ldcg(q_off + lane), qb = __ldcg(q_off + lane + 1);
        const int32_t l = __ldcg(kv_len + lane);
        len = good_length(a, l);
        if (l != len) pk::set_status(a.status, PK_ERR_ARG);
    }
    const bool bad = __any_sync(0xffffffffu, bad_offsets(qa, qb, a.n_q));
    if (bad && lane == 0) pk::set_status(a.status, PK_ERR_ARG);
    const uint32_t units = bad ? 0 : units_of(a, qb - qa), tiles = tiles_of(a, len);
    uint64_t total = (uint64_t)units * a.kv_heads * tiles;
#pragma unroll
    for (int d = 16; d; d /= 2) total += __shfl_xor_sync(0xffffffffu, total, d);
    const uint32_t split = split_of(a, total);
    uint32_t scan = units * pieces_of(tiles, split);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    sm.item_end[lane] = scan;
    sm.q_start[lane] = (int32_t)qa;
    sm.q_len[lane] = (int32_t)(qb - qa);
    sm.len[lane] = len;
    if (lane == 0) sm.split = split;
    if (a.target && blockIdx.x == 0) {  // for k_chunk_join
        if (lane < a.R) a.plan[2 + lane] = scan;
        if (lane == 0) {
            a.plan[0] = split;
            a.plan[1] = 0;
        }
    }
}

// One item: 2 tiles of tile_tokens query tokens times tile_heads heads of one group, and a piece of their keys.
struct Item {
    uint32_t r, head, chunk, index, pieces;
    int32_t q0, lq, len, tok0;
    int32_t skip;         // tokens in the gap, a multiple of 16: place x is position x, or x + skip behind the first granules
    int32_t first;        // first key tile of the piece
    int32_t n_tiles[2], n_all;
    uint32_t n_gran;      // granules of the whole list
};

__device__ __forceinline__ bool find_item(const Args &a, const Small &sm, const uint64_t *plan, const int64_t *q_off,
                                          const int32_t *kv_len, uint32_t index, Item &it) {
    const uint32_t tile = index / a.kv_heads;
    it.index = index;
    it.head = index - tile * a.kv_heads;
    it.q0 = it.lq = it.len = 0;
    it.r = 0;
    uint32_t x = 0, split = 0;  // which of the request's items
    if (a.listed) {
        if (tile < __ldcg(plan + 1 + a.R)) {
            it.r = pk::warp_find_request(reinterpret_cast<const int64_t *>(plan + 1), a.R, (int64_t)tile);
            it.q0 = (int32_t)__ldcg(q_off + it.r);
            it.lq = (int32_t)__ldcg(q_off + it.r + 1) - it.q0;
            it.len = good_length(a, __ldcg(kv_len + it.r));
            x = (uint32_t)__ldcg(plan + 2 + it.r) - 1 - tile;
            split = (uint32_t)__ldcg(plan);
        }
    } else {
        const uint32_t lane = threadIdx.x & 31;
        it.r = __popc(__ballot_sync(0xffffffffu, sm.item_end[lane] <= tile));
        if (it.r < 32) {  // (requests past R repeat the total)
            it.q0 = sm.q_start[it.r];
            it.lq = sm.q_len[it.r];
            it.len = sm.len[it.r];
            x = sm.item_end[it.r] - 1 - tile;
            split = sm.split;
        }
    }
    // the last queries first: they have the most keys
    it.pieces = pieces_of(tiles_of(a, it.len), split);
    const uint32_t piece = x % it.pieces;
    x /= it.pieces;
    it.chunk = x % a.chunks;
    it.tok0 = (int32_t)(x / a.chunks) * 2 * (int32_t)a.tile_tokens;
    const int32_t off = it.len - it.lq;  // position of the request's first query
    const int64_t low = (int64_t)off + it.tok0 - a.window + 1;
    const uint32_t low_gran = a.window && low > 0 ? (uint32_t)(low / 16) : 0;
    it.skip = low_gran > a.sink_grans ? (int32_t)(low_gran - a.sink_grans) * 16 : 0;
    int32_t n[2];
    it.n_gran = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int32_t t0 = it.tok0 + t * (int32_t)a.tile_tokens, t1 = min(t0 + (int32_t)a.tile_tokens, it.lq);
        const int32_t last = t1 > t0 ? off + t1 - 1 - it.skip : -1;
        n[t] = last >= 0 ? last / kKeys + 1 : 0;
        if (last >= 0) it.n_gran = (uint32_t)last / 16 + 1;
    }
    const int32_t all = max(n[0], n[1]);
    it.first = (int32_t)((uint64_t)all * piece / it.pieces);
    const int32_t end = (int32_t)((uint64_t)all * (piece + 1) / it.pieces);
#pragma unroll
    for (int t = 0; t < 2; ++t) it.n_tiles[t] = max(min(n[t], end) - it.first, 0);
    it.n_all = max(it.n_tiles[0], it.n_tiles[1]);
    return it.lq > 0;
}

// Lowest position that the query `tok` of a request sees behind the first tokens; off: position of the request's first.
__device__ __forceinline__ int32_t low_of(const Args &a, int32_t off, int32_t tok) {
    return a.window ? (int32_t)max((int64_t)off + tok - a.window + 1, (int64_t)0) : 0;
}

// Registers move to the softmax warps: 256 * 176 + 256 * 80 = 512 * 128, the launch's own.
constexpr int kRegsSoftmax = 176, kRegsOther = 80;
constexpr uint32_t kWarpLoad = 8, kWarpMma = 9, kWarpNote = 10, kWarpUnpack = 12;  // warps 0-7: softmax

// Where a lane finds its codes and scales of K or V in a granule, and where it puts them as 16-bit values in a tile, in
// the 128-byte swizzle: 32 dimensions of a token, and the same of the token 8 further on for D = 128.  Eight lanes that
// store at once have two rows' (D = 128) or four rows' pieces: the upper half of the dimensions goes in another order,
// so that they lie in eight different 16-byte columns.
template <int D>
struct Unpack {
    static constexpr uint32_t kParts = D / 32, kRows = 32 / kParts;
    uint32_t row, codes[2], scales, pick[2], dst[4];

    __device__ __forceinline__ explicit Unpack(uint32_t lane) {
        const uint32_t part = lane % kParts, flip = part >= 2 ? 2 : 0;
        row = lane / kParts;
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            codes[i] = row * (D / 2) + part * 16 + ((2 * i) ^ flip) * 4;
            pick[i] = i ^ flip / 2 ? 0x3232 : 0x1010;
        }
        scales = row * (D / 16) + part * 2;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            dst[i] = part / 2 * 16384 + row * 128 + (((part % 2 * 4 + (i ^ flip)) ^ (row & 7)) << 4);
    }

    // A granule's 16 rows; `tile`: where the first of them lies.  Weights of 0 must not meet a NaN: of V (kClean) rows from
    // `valid` on, past the request's end, count as 0, and so do blocks marked NaN.
    template <bool kBf16, bool kClean>
    __device__ __forceinline__ void granule(const uint8_t *from, const uint8_t *from_scales, uint8_t *tile, int32_t valid) const {
#pragma unroll
        for (uint32_t r = 0; r < 16; r += kRows) {
            uint32_t two = *reinterpret_cast<const uint16_t *>(from_scales + scales + r * (D / 16));
            if (kClean) {
                if (((two & 0x7f7f) + 0x0101) & 0x8080) two &= ~__vcmpeq4(two & 0x7f7f, 0x7f7f);
                if ((int32_t)(row + r) >= valid) two = 0;
            }
            const uint32_t z = pk::e4m3_to_half2(two);
            uint32_t by[2];
            if (kBf16) {
                // a half's bits, three to the right, are 2^-112 times the value as a bfloat16; the scale makes up for it
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&z));
                by[0] = pk::Elem<PK_BF16>::from2(f.x * 0x1p112f, f.y * 0x1p112f);
                by[1] = __byte_perm(by[0], by[0], pick[1]);
                by[0] = __byte_perm(by[0], by[0], pick[0]);
            } else {
                by[0] = __byte_perm(z, z, pick[0]);
                by[1] = __byte_perm(z, z, pick[1]);
            }
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const uint2 u = *reinterpret_cast<const uint2 *>(from + codes[i / 2] + r * (D / 2));
                const uint32_t w[2] = {u.x, u.y};
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    uint32_t h[4];
                    pk::e2m1x8_to_half2(w[n], h);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (kBf16) {
                            const uint32_t b = (h[k] >> 3 & 0x0fff0fffu) | (h[k] & 0x80008000u);
                            asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(h[k]) : "r"(b), "r"(by[i / 2]));
                        } else {
                            asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(h[k]) : "r"(h[k]), "r"(by[i / 2]));
                        }
                    }
                    *reinterpret_cast<uint4 *>(tile + dst[i + n] + r * 128) = make_uint4(h[0], h[1], h[2], h[3]);
                }
            }
        }
    }
};

// One CTA an SM takes one item after another.  Warp roles: one copies Q tiles and
// granules, six make K and V tiles of granules, one issues the matrix products, and two warpgroups of four turn scores into weights, a thread a row,
// for one of the item's two tiles each: while one tile's scores are weighed the
// other's products run.  TMEM: scores of the tiles (128 columns each; the weights, two
// to a column, take the place of scores that have been read), then their outputs
// (D columns each).  Every counter of a barrier's use runs on over the items.
template <int D, uint32_t DT>
__global__ void __launch_bounds__(kThreads, 1) k_attend_chunk(const Args a, const __grid_constant__ CUtensorMap map_q) {
    using L = Layout<D>;
    using G = pk::Granule<D>;
    // all the shared memory that the kernel has, so that it starts on the swizzle's 1024 bytes
    extern __shared__ __align__(1024) uint8_t smem_c[];
    Small &sm = *reinterpret_cast<Small *>(smem_c + L::kBytes);
    const uint32_t smem = pk::smem_addr(smem_c);
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = pk::uniform(tid >> 5);
    if (smem & 1023) {
        if (tid == 0) pk::set_status(a.status, PK_ERR_CUDA);
        return;
    }

    if (tid == 0) {
        for (uint32_t i = 0; i < L::kStages; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.full[i]), kMakers);
            pk::mbar_init(pk::smem_addr(&sm.empty[i]), 1);
        }
        for (uint32_t i = 0; i < L::kGrans; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.gran_full[i]), 1);
            pk::mbar_init(pk::smem_addr(&sm.gran_empty[i]), kMakers);
        }
        for (int t = 0; t < 2; ++t) {
            pk::mbar_init(pk::smem_addr(&sm.q_full[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.q_empty[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.s_full[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.p_ready[t]), 4);
            pk::mbar_init(pk::smem_addr(&sm.o_done[t]), 1);
        }
        pk::mbar_init(pk::smem_addr(&sm.over), 1);
        pk::mbar_fence_init();
        sm.abort = 0;
    }
    if (warp == kWarpMma) pk::tmem_alloc(pk::smem_addr(&sm.tmem), 512);
    const uint64_t *plan = a.plan;
    const int64_t *q_off = a.q_off;
    const int32_t *kv_len = a.kv_len;
    const uint32_t *pages = a.pages;
    const uint8_t *pool = a.pool;
    pk::pdl_wait(plan, q_off, kv_len, pages, pool);
    pk::pdl_launch_dependents();
    if (warp == kWarpLoad && !a.listed) plan_here(a, sm, q_off, kv_len);
    pk::tmem_fence_before();
    __syncthreads();
    pk::tmem_fence_after();
    const uint32_t tmem = pk::uniform(sm.tmem);

    volatile uint32_t *abort = &sm.abort;
    auto give_up = [&]() {
        *abort = 1;
        pk::set_status(a.status, PK_ERR_TIMEOUT);
    };

    Item it;
    uint32_t turn = 0;  // items before the present one
    bool more = find_item(a, sm, plan, q_off, kv_len, blockIdx.x, it);
    // every other turn runs through the blocks backwards: one that got the heaviest item of a turn gets the lightest of
    // the next
    auto take_next = [&]() {
        ++turn;
        const uint64_t next = (uint64_t)turn * gridDim.x + (turn & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        more = next < a.most_items && find_item(a, sm, plan, q_off, kv_len, (uint32_t)next, it);
    };
    if (warp >= kWarpLoad) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kWarpLoad) {
            uint32_t count = 0, nq[2] = {0, 0};  // granules and Q tiles so far
            bool ok = true, sent = false;        // sent: a copy that `count` does not hold
            const uint32_t slot_shift = 31 - __clz(a.page_grans);
            const bool pow2 = (a.page_grans & (a.page_grans - 1)) == 0;
            pk::fence_proxy_async();  // pages written by an earlier kernel are read by the async proxy
            while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
                const uint32_t v0 = 8 * (uint32_t)it.first, v1 = min(8 * (uint32_t)(it.first + it.n_all), it.n_gran);
                const uint32_t *row = pages + (uint64_t)it.r * a.page_stride;
                uint64_t where = 0;  // lane l: address of the granule `base` + l of the list
                bool lost = false;   // slot 0's bytes stand in for a slot out of range
                auto find_granules = [&](uint32_t base) {
                    const uint32_t v = base + lane;
                    lost = false;
                    if (v < v1) {
                        const uint32_t gr = v >= a.sink_grans ? v + (uint32_t)it.skip / 16 : v;
                        const uint32_t page = pow2 ? gr >> slot_shift : gr / a.page_grans;
                        uint64_t slot = __ldcg(row + page);
                        if (slot >= a.n_slots) {
                            pk::set_status(a.status, PK_ERR_ARG);
                            slot = 0;
                            lost = true;
                        }
                        where = reinterpret_cast<uint64_t>(pool) + slot * a.page_bytes +
                                ((uint64_t)it.head * a.page_grans + (gr - page * a.page_grans)) * L::kGran;
                    }
                };
                for (uint32_t v = v0; ok && it.n_all > 0 && v < v1; v += 8) {
                    if (((v - v0) & 31) == 0) find_granules(v);
                    const uint32_t n = min(v1 - v, 8u), from = ((v - v0) & 31) + (lane & 7);
                    const uint64_t src = __shfl_sync(0xffffffffu, where, from);
                    const bool bad = __shfl_sync(0xffffffffu, (uint32_t)lost, from) != 0;
                    if (lane < n) {  // a lane a granule
                        const uint32_t c = count + lane, s = c % L::kGrans;
                        ok = c < L::kGrans || pk::mbar_wait(pk::smem_addr(&sm.gran_empty[s]), (c / L::kGrans + 1) & 1);
                        if (ok) {
                            sm.gran_lost[s] = bad;
                            pk::mbar_expect(pk::smem_addr(&sm.gran_full[s]), L::kGran);
                            pk::bulk_load(smem + L::kGranRing + s * L::kGran, reinterpret_cast<const void *>(src), L::kGran,
                                          pk::smem_addr(&sm.gran_full[s]));
                            sent = true;
                        }
                    }
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    sent = false;
                    count += n;
                    if (v == v0 && lane == 0) {  // Q behind the first tile
                        const uint32_t q_bytes = a.tile_tokens * a.tile_heads * 128 * (D / 64);
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (!ok || it.n_tiles[t] == 0) continue;
                            ok = nq[t] == 0 || pk::mbar_wait(pk::smem_addr(&sm.q_empty[t]), (nq[t] - 1) & 1);
                            if (!ok) break;
                            const uint32_t bar = pk::smem_addr(&sm.q_full[t]);
                            pk::mbar_expect(bar, q_bytes);
#pragma unroll
                            for (int b = 0; b < D / 64; ++b)
                                pk::tile_load3(smem + t * L::kTile + b * 16384, &map_q, b * 64,
                                               (int)(it.head * a.group + it.chunk * a.tile_heads),
                                               it.q0 + it.tok0 + t * (int)a.tile_tokens, bar);
                            ++nq[t];
                        }
                    }
                    ok = __all_sync(0xffffffffu, ok);
                }
                if (ok) take_next();
            }
            if (!ok && lane == 0) give_up();
            // no copy of its own stays in flight, each by the barrier that its own arrival completes, so that no wait
            // depends on a warp that gave up
            const uint32_t tail = count + (sent ? lane + 1 : 0);  // a lane of a turn that failed: its own copy too
            if (sent) pk::mbar_wait(pk::smem_addr(&sm.gran_full[(tail - 1) % L::kGrans]), ((tail - 1) / L::kGrans) & 1);
            if (lane < L::kGrans && lane < count) {
                const uint32_t c = count - 1 - lane;
                pk::mbar_wait(pk::smem_addr(&sm.gran_full[c % L::kGrans]), (c / L::kGrans) & 1);
            }
            if (lane == 0)
                for (int t = 0; t < 2; ++t)
                    if (nq[t]) pk::mbar_wait(pk::smem_addr(&sm.q_full[t]), (nq[t] - 1) & 1);
            __syncwarp();
        } else if (warp >= kWarpNote) {
            // Makers of K and V tiles: two warps look for what the softmax warps have to know of a tile, four unpack it.
            const uint32_t w = warp - kWarpUnpack, half = warp - kWarpNote;
            const bool notes = warp < kWarpUnpack;
            const Unpack<D> lanes(lane);
            uint32_t n = 0, count = 0, tiles = 0, items = 0;  // stages, granules, key tiles, items with keys so far
            bool ok = true;
            auto wait_empty = [&](uint32_t n) {
                return n < L::kStages ||
                       pk::mbar_wait_warp(pk::smem_addr(&sm.empty[n % L::kStages]), (n / L::kStages + 1) & 1);
            };
            while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
                if (it.n_all > 0) {
                    // its reader, at most four items behind, sees it by way of the first K tile's barrier
                    if (warp == kWarpNote && lane == 0) {
                        sm.work[items & 7][0] = it.n_tiles[0];
                        sm.work[items & 7][1] = it.n_tiles[1];
                    }
                    ++items;
                }
                for (int32_t j = 0; j < it.n_all; ++j) {
                    const uint32_t v0 = 8 * (uint32_t)(it.first + j), have = min(it.n_gran - v0, 8u);
                    // Every warp waits for all of the tile's granules, a lane each, and gives all of them back: a place's
                    // next user may be another warp, and one that has not seen a use of it, or sees it too late, would
                    // take one state of the barrier for another.
                    const uint32_t c = count + lane;
                    ok = lane >= have || pk::mbar_wait(pk::smem_addr(&sm.gran_full[c % L::kGrans]), (c / L::kGrans) & 1);
                    ok = __all_sync(0xffffffffu, ok) && wait_empty(n);
                    if (!ok) break;
                    auto place = [&](uint32_t g) { return smem_c + L::kGranRing + (count + g) % L::kGrans * L::kGran; };
                    // tokens of a granule before the request's end
                    auto valid = [&](uint32_t g) {
                        return it.len - (int32_t)(16 * (v0 + g)) - (v0 + g >= a.sink_grans ? it.skip : 0);
                    };
                    const uint32_t mine = have > 2 * w ? min(have - 2 * w, 2u) : 0;  // granules, of an unpacking warp
                    uint8_t *tile = smem_c + L::kRing + n % L::kStages * L::kTile + (notes ? 0 : 32 * w * 128);
                    if (notes) {  // blocks of V marked NaN, two tokens a lane
                        uint32_t bits[2] = {0, 0}, lost = 0;
#pragma unroll
                        for (uint32_t i = 0; i < 2; ++i) {
                            const uint32_t g = 4 * half + 2 * i + lane / 16, tok = lane % 16;
                            if (g >= have) continue;
                            const uint32_t *s = reinterpret_cast<const uint32_t *>(place(g) + G::kVs + tok * G::kScales);
                            lost |= sm.gran_lost[(count + g) % L::kGrans];
                            if ((int32_t)tok >= valid(g)) continue;
#pragma unroll
                            for (uint32_t k = 0; k < G::kScales / 4; ++k) {
                                const uint32_t m = __vcmpeq4(s[k] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                                bits[i] |= ((m & 1) | (m >> 7 & 2) | (m >> 14 & 4) | (m >> 21 & 8)) << (4 * k);
                            }
                        }
                        const bool marked = __any_sync(0xffffffffu, (bits[0] | bits[1]) != 0);
                        const bool gone = __any_sync(0xffffffffu, lost != 0);
                        if (marked) {
                            sm.marked[tiles % kNotes][64 * half + lane] = (uint8_t)bits[0];
                            sm.marked[tiles % kNotes][64 * half + 32 + lane] = (uint8_t)bits[1];
                        }
                        if (lane == 0) sm.flags[tiles % kNotes][half] = (marked ? kMarked : 0) | (gone ? kLost : 0);
                    } else {
#pragma unroll
                        for (uint32_t h = 0; h < 2; ++h)
                            if (h < mine)
                                lanes.template granule<DT == PK_BF16, false>(place(2 * w + h) + G::kK, place(2 * w + h) + G::kKs,
                                                                             tile + 16 * h * 128, 16);
                        pk::fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[n % L::kStages]));
                    ++n;
                    ok = wait_empty(n);
                    if (!ok) break;
                    if (!notes) {
                        tile = smem_c + L::kRing + n % L::kStages * L::kTile + 32 * w * 128;
#pragma unroll
                        for (uint32_t h = 0; h < 2; ++h)
                            if (h < mine)
                                lanes.template granule<false, true>(place(2 * w + h) + G::kV, place(2 * w + h) + G::kVs,
                                                                    tile + 16 * h * 128, valid(2 * w + h));
                        // rows behind the last granule: weights of 0 must not meet what lies there
                        for (uint32_t x = mine * 16 * (D / 8) + lane; x < 32 * (D / 8); x += 32)
                            *reinterpret_cast<uint4 *>(tile + x % (D / 8) / 8 * 16384 + x / (D / 8) * 128 + x % 8 * 16) =
                                make_uint4(0, 0, 0, 0);
                        pk::fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane < have) pk::mbar_arrive(pk::smem_addr(&sm.gran_empty[c % L::kGrans]));
                    if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[n % L::kStages]));
                    ++n;
                    count += have;
                    ++tiles;
                }
                if (ok) take_next();
            }
            ok = ok && wait_empty(n);
            if (ok) {  // the matrix warp's end: a stage without a tile
                if (lane == 0) {
                    if (warp == kWarpNote) sm.work[items & 7][0] = sm.work[items & 7][1] = 0;
                    pk::mbar_arrive(pk::smem_addr(&sm.full[n % L::kStages]));
                }
            } else if (lane == 0) {
                give_up();
            }
            __syncwarp();
        } else if (warp == kWarpMma) {
            const uint32_t qk_kind = pk::mma_idesc(DT == PK_BF16, 128, 128, false) |
                                     (a.scale2 < 0.0f ? 1u << 13 : 0u);  // a negative scale negates Q
            constexpr uint32_t kPv = pk::mma_idesc(false, 128, D, true);
            uint32_t ring = 0, use = 0;             // next ring stage, and how often the ring has been gone round
            uint32_t ni0 = 0, ni1 = 0, nq0 = 0, nq1 = 0;  // key tiles and Q tiles used so far, by tile
            bool ok = true;
            auto wait_full = [&](uint32_t st, uint32_t round) {
                return pk::mbar_wait_warp(pk::smem_addr(&sm.full[st]), round & 1);
            };
            auto advance = [&](uint32_t by) {
                ring += by;
                if (ring >= L::kStages) ring -= L::kStages, ++use;
            };
            auto qk = [&](int t, uint32_t st, bool last) {
                const uint32_t q = smem + t * L::kTile, k = smem + L::kRing + st * L::kTile;
                if (pk::elect_lane()) {
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        pk::mma_ss(tmem + 128 * t, pk::mma_desc(q + (s / 4) * 16384 + (s % 4) * 32, 16, 1024),
                                   pk::mma_desc(k + (s / 4) * 16384 + (s % 4) * 32, 16, 1024), qk_kind, s > 0);
                    pk::mma_commit(pk::smem_addr(&sm.s_full[t]));
                    if (last) pk::mma_commit(pk::smem_addr(&sm.q_empty[t]));
                }
                __syncwarp();
            };
            auto pv = [&](int t, uint32_t st, bool first) {
                const uint32_t v = smem + L::kRing + st * L::kTile;
                if (pk::elect_lane()) {
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        pk::mma_ts(tmem + 256 + D * t, tmem + 128 * t + 8 * s, pk::mma_desc(v + s * 2048, 16384, 1024),
                                   kPv, !first || s > 0);
                    pk::mma_commit(pk::smem_addr(&sm.o_done[t]));
                }
                __syncwarp();
            };
            auto release = [&](uint32_t st) {
                if (pk::elect_lane()) pk::mma_commit(pk::smem_addr(&sm.empty[st]));
                __syncwarp();
            };
            for (uint32_t items = 0; ok && !__any_sync(0xffffffffu, *abort != 0); ++items) {
                ok = wait_full(ring, use);
                if (!ok) break;
                const int32_t n0 = (int32_t)pk::uniform(sm.work[items & 7][0]);
                const int32_t n1 = (int32_t)pk::uniform(sm.work[items & 7][1]);
                const int32_t n_all = max(n0, n1);
                if (n_all == 0) break;
                if (n0 > 0 && (ok = pk::mbar_wait_warp(pk::smem_addr(&sm.q_full[0]), nq0++ & 1))) {
                    pk::tmem_fence_after();
                    qk(0, ring, n0 == 1);
                }
                if (ok && n1 > 0 && (ok = pk::mbar_wait_warp(pk::smem_addr(&sm.q_full[1]), nq1++ & 1))) {
                    pk::tmem_fence_after();
                    qk(1, ring, n1 == 1);
                }
                if (ok) release(ring);
                advance(1);
                for (int32_t j = 0; ok && j < n_all; ++j) {
                    const uint32_t sv = ring, uv = use;
                    advance(1);
                    const uint32_t sk = ring, uk = use;  // K of the next tile, where there is one
                    ok = wait_full(sv, uv);
                    if (ok && j < n0 && (ok = pk::mbar_wait_warp(pk::smem_addr(&sm.p_ready[0]), ni0++ & 1))) {
                        pk::tmem_fence_after();
                        pv(0, sv, j == 0);
                        if (j + 1 < n0 && (ok = wait_full(sk, uk))) qk(0, sk, j + 2 == n0);
                    }
                    if (ok && j < n1 && (ok = pk::mbar_wait_warp(pk::smem_addr(&sm.p_ready[1]), ni1++ & 1))) {
                        pk::tmem_fence_after();
                        pv(1, sv, j == 0);
                        release(sv);
                        if (j + 1 < n1 && (ok = wait_full(sk, uk))) qk(1, sk, j + 2 == n1);
                    } else if (ok) {
                        release(sv);
                    }
                    if (ok && j + 1 < n_all) {
                        release(sk);
                        advance(1);
                    }
                }
            }
            // The commits' arrivals come by themselves: none may be left to find the shared memory in another block's
            // hands, nor a product the TMEM.  So the last one on every barrier is waited for: a stage, two tiles' scores
            // and outputs, and their Q, were given back once a use.
            auto last_commit = [&](const uint64_t &bar, uint32_t commits) {
                if (commits) ok = pk::mbar_wait_warp(pk::smem_addr(&bar), (commits - 1) & 1) && ok;
            };
            if (ok) {
                const uint32_t freed = use * L::kStages + ring;
                for (uint32_t i = freed > L::kStages ? freed - L::kStages : 0; i < freed; ++i)
                    last_commit(sm.empty[i % L::kStages], i / L::kStages + 1);
                last_commit(sm.s_full[0], ni0);
                last_commit(sm.s_full[1], ni1);
                last_commit(sm.o_done[0], ni0);
                last_commit(sm.o_done[1], ni1);
                last_commit(sm.q_empty[0], nq0);
                last_commit(sm.q_empty[1], nq1);
            } else {  // it left somewhere between: behind this one all products are done
                if (pk::elect_lane()) pk::mma_commit(pk::smem_addr(&sm.over));
                __syncwarp();
                last_commit(sm.over, 1);
            }
            if (!ok && lane == 0) give_up();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const uint32_t t = warp >> 2;
        const int32_t row = tid & 127;  // TMEM lane
        const int32_t row_tok = row / (int32_t)a.tile_heads, row_head = row % (int32_t)a.tile_heads;
        const uint32_t ts = tmem + 128 * t + ((warp & 3) * 32 << 16), to = tmem + 256 + D * t + ((warp & 3) * 32 << 16);
        // a scale of 0 would make a masked -infinity NaN; the smallest normal one gives the same weights
        const float scale2 = fmaxf(fabsf(a.scale2), FLT_MIN);
        const uint64_t scale22 = pk::pack2(scale2, scale2);
        // What is not needed at every tile of the item lies in shared memory: in registers it would push others out.
        volatile TileOf *mine = &sm.tile[warp];
        uint32_t ni = 0, tiles = 0;  // key tiles weighed so far; key tiles of the CTA's items before the present one
        bool ok = true;
        while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
            const int32_t n_tiles = t ? it.n_tiles[1] : it.n_tiles[0];
            bool on;
            {
                const int32_t tok0 = it.tok0 + (int32_t)(t * a.tile_tokens), off = it.len - it.lq;
                const int32_t base = it.first * kKeys + it.skip;  // from positions to places behind the piece's first one
                const int32_t all_last = off + tok0 - base;
                const int32_t all_low = low_of(a, off, min(tok0 + (int32_t)a.tile_tokens, it.lq) - 1) - base;
                const int32_t sinks = (int32_t)a.sinks - it.first * kKeys, gh0 = (int32_t)(it.chunk * a.tile_heads);
                if (lane == 0) {
                    mine->causal = ((all_last - (kKeys - 1)) >> 7) + 1;
                    mine->hides[0] = sinks >> 7;
                    mine->hides[1] = a.window ? (all_low + kKeys - 1) >> 7 : 0;
                    mine->off = off;
                    mine->base = base;
                    mine->sinks = sinks;
                    mine->tok0 = tok0;
                    mine->row0 = it.q0 + tok0;
                    mine->head0 = it.head * a.group + gh0;
                    mine->part = it.pieces > 1 ? ((int64_t)it.index * 2 + t) * kRows : -1;
                    mine->n_all = it.n_all;
                }
                on = row_tok < (int32_t)a.tile_tokens && tok0 + row_tok < it.lq && gh0 + row_head < (int32_t)a.group;
                __syncwarp();
            }
            // a weight is 2^(score - ref + fine), and fine is 0 but for a reference of kFar and more
            float ref = -FLT_MAX, fine = 0.0f, sum = 0.0f;
            uint32_t marked = 0;  // blocks of 16 dimensions in which the row saw a NaN of V
            bool lost = false;    // it saw a token whose slot is out of range
#pragma unroll 1
            for (int32_t j = 0; ok && j < n_tiles; ++j, ++ni) {
                ok = pk::mbar_wait_warp(pk::smem_addr(&sm.s_full[t]), ni & 1);
                if (!ok) break;
                pk::tmem_fence_after();
                // the row sees the tile's keys up to `see` that are not below `from`, or are below `first`
                const bool edge = j >= mine->causal || (j >= mine->hides[0] && j < mine->hides[1]);
                int32_t see = kKeys, from = 0, first = 0;
                if (edge) {
                    const int32_t tok = mine->tok0 + row_tok, x0 = j * kKeys;
                    see = on ? mine->off + tok - mine->base - x0 : -1;
                    from = low_of(a, mine->off, tok) - mine->base - x0;
                    first = mine->sinks - x0;
                }
                auto hidden = [&](int32_t i) { return i > see || (i < from && i >= first); };
                const uint32_t note = (tiles + j) % kNotes;
                const uint32_t flags = *reinterpret_cast<const volatile uint16_t *>(sm.flags[note]);
                if (flags) {
                    lost |= (flags & 0x0101u * kLost) != 0;
#pragma unroll 1
                    for (int32_t i = 0; i < kKeys; ++i)
                        if ((flags >> (i / 64 * 8) & kMarked) && !hidden(i)) marked |= sm.marked[note][i];
                }
                uint32_t x[3][32];
                // Chunk c of the scores, 32 keys.  Loads run ahead (1 and 2 behind 0's use, 3 behind 1's).  Masked or
                // not is known at compile time.
                auto chunk = [&](int c, auto masked) -> uint32_t(&)[32] {
                    if (c == 0) pk::tmem_load32(ts, x[0]);
                    uint32_t(&y)[32] = x[c % 3];
                    if (c != 2) pk::tmem_wait_load(y);
                    if (c == 0) {
                        pk::tmem_load32(ts + 32, x[1]);
                        pk::tmem_load32(ts + 64, x[2]);
                    } else if (c == 1) {
                        pk::tmem_wait_load(x[2]);
                        pk::tmem_load32(ts + 96, x[0]);
                    }
                    if (decltype(masked)::value) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (hidden(32 * c + i)) y[i] = 0xff800000u;
                    }
                    return y;
                };
                auto largest = [&](auto masked) {
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t(&y)[32] = chunk(c, masked);
#pragma unroll
                        for (int i = 0; i < 32; ++i) m4[i & 3] = fmaxf(m4[i & 3], __uint_as_float(y[i]));
                    }
                    return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                };
                // The weights by the reference so far, and their sum.
                uint32_t p[2][32];
                auto weigh = [&](auto masked) {
                    const uint64_t ref2 = pk::pack2(-ref, -ref);
                    uint64_t sum2[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t(&y)[32] = chunk(c, masked);
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float2 z = pk::unpack2(
                                pk::fma2(pk::pack2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), scale22, ref2));
                            z.x = pk::ex2(z.x);
                            z.y = pk::ex2(z.y);
                            sum2[i / 2 & 1] = pk::add2(sum2[i / 2 & 1], pk::pack2(z.x, z.y));
                            p[c / 2][c % 2 * 16 + i / 2] = pk::Elem<PK_FP16>::from2(z.x, z.y);
                        }
                    }
                    const float2 s0 = pk::unpack2(sum2[0]), s1 = pk::unpack2(sum2[1]);
                    return (s0.x + s1.x) + (s0.y + s1.y);
                };
                // The same where a row of the warp has a far reference, which few calls have: by 16 scores, with `fine`.
                auto weigh_far = [&]() {
                    float s = 0.0f;
                    uint32_t(&y)[16] = reinterpret_cast<uint32_t(&)[16]>(x[0]);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        pk::tmem_load16(ts + 16 * c, y);
                        pk::tmem_wait_load(y);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float w[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const bool off = edge && hidden(16 * c + i + h);
                                w[h] = off ? 0.0f : pk::ex2(fmaf(__uint_as_float(y[i + h]), scale2, -ref) + fine);
                                s += w[h];
                            }
                            p[c / 4][c % 4 * 8 + i / 2] = pk::Elem<PK_FP16>::from2(w[0], w[1]);
                        }
                    }
                    return s;
                };
                auto weigh_any = [&]() {
                    if (__any_sync(0xffffffffu, fine != 0.0f)) return weigh_far();
                    return edge ? weigh(std::true_type{}) : weigh(std::false_type{});
                };
                // Moves the reference of the rows that `over` names to their largest score; their sum and output so
                // far are rescaled.  That score's weight is then a power of two, which rounding leaves as it is: a
                // row with one key, or one that outweighs the others, gets its value of V and no more error.
                auto move_ref = [&](bool over) {
                    const float top = edge ? largest(std::true_type{}) : largest(std::false_type{}), m = top * scale2;
                    const bool moves = over && m > -INFINITY, far = moves && fabsf(m) >= kFar;
                    const float next = !moves ? ref : far ? m : m - kBase;
                    // far: what m's rounding lost comes off again, so the largest weight is 2^kBase or, where kBase
                    // is lost beside that, 1; not a number where m overflowed
                    const float next_fine = !moves ? fine : far ? kBase - fmaf(top, scale2, -m) : 0.0f;
                    const float f = pk::ex2((ref - next) + (next_fine - fine));
                    ref = next;
                    fine = next_fine;
                    sum *= f;
                    if (j == 0) return;
                    ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (ni - 1) & 1);
                    if (!ok) return;
                    pk::tmem_fence_after();
#pragma unroll 1
                    for (int d = 0; d < D / 32; ++d) {
                        pk::tmem_load32(to + 32 * d, x[0]);
                        pk::tmem_wait_load(x[0]);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[0][i] = __float_as_uint(__uint_as_float(x[0][i]) * f);
                        pk::tmem_store32(to + 32 * d, x[0]);
                    }
                };
                if (j == 0) move_ref(on);
                // One pass over the scores takes the weights by the reference so far, with no look at the scores
                // first: a weight that has outgrown it shows in the sum, and only then the reference is moved and
                // the pass done again.  A row that saw no key yet (its window begins further on) has the lowest
                // reference, by which any weight is infinite.  Once does: behind a move no weight is above
                // 2^(kBase + 2).  Rows without a query have no say.
                float part_sum = weigh_any();
                if (__any_sync(0xffffffffu, on && part_sum > kTop)) {
                    move_ref(on && part_sum > kTop);
                    if (!ok) break;
                    part_sum = weigh_any();
                }
                if (!ok) break;
                sum += part_sum;
                pk::tmem_store32(ts, p[0]);  // over the scores, which every pass is done with
                pk::tmem_store32(ts + 32, p[1]);
                pk::tmem_wait_store();
                pk::tmem_fence_before();
                __syncwarp();
                if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.p_ready[t]));
            }
            tiles += (uint32_t)mine->n_all;
            take_next();  // while the last product runs
            if (ok && n_tiles > 0) ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (ni - 1) & 1);
            if (!ok) break;
            if (lost) sum = __int_as_float(0x7fffffff);
            const int64_t part = mine->part >= 0 ? mine->part + row : -1;
            const bool cut = part >= 0;
            const int64_t q_row = (int64_t)mine->row0 + row_tok;
            const uint32_t qh = (uint32_t)(mine->head0 + row_head);
            const float inv = cut ? 1.0f : sum == 0.0f ? 0.0f : a.v_scale / sum;
            if (on && cut) a.part_ml[part] = make_float4(ref, fine, sum, 0.0f);
            if (on && !cut && a.lse)
                a.lse[q_row * a.q_heads + qh] = sum == 0.0f ? -INFINITY : (ref - fine + log2f(sum)) * 0.69314718055994531f;
            uint16_t *dst = a.out + q_row * a.o_ts + (int64_t)qh * a.o_hs;
            pk::tmem_fence_after();
            // 16 columns of the output, the next ones on their way meanwhile
            uint32_t y[2][16];
            if (n_tiles > 0) pk::tmem_load16(to, y[0]);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {  // no load is left in flight over a loop's end
                uint32_t(&z)[16] = y[c & 1];
                if (n_tiles > 0) {  // else O was never written
                    __syncwarp();
                    pk::tmem_wait_load(z);
                    if (c + 1 < D / 16) pk::tmem_load16(to + 16 * (c + 1), y[(c + 1) & 1]);
                }
                if (!on) continue;
                const bool none = n_tiles == 0 || inv == 0.0f, nan = marked >> c & 1;
                float f[16];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    f[i] = nan ? __int_as_float(0x7fffffff) : none ? 0.0f : __uint_as_float(z[i]) * inv;
                uint32_t w[8];
                if (cut) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[8 * h + i]);
                        pk::store32(reinterpret_cast<uint16_t *>(a.part_o + part * D + 16 * c + 8 * h), true, w);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; i += 2) w[i / 2] = pk::Elem<DT>::from2(f[i], f[i + 1]);
                    pk::store32(dst + 16 * c, a.wide_out, w);
                }
            }
            __syncwarp();
        }
        if (!ok && lane == 0) give_up();
    }
    pk::tmem_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        pk::tmem_fence_after();
        pk::tmem_free(tmem, 512);
    }
}

// Joins the pieces of the rows whose keys were cut, a warp a row, in the order of the keys.
constexpr int kJoinThreads = 256;
template <int D, uint32_t DT>
__global__ void __launch_bounds__(kJoinThreads) k_chunk_join(const Args a) {
    const uint64_t *plan = a.plan;
    const int64_t *q_off = a.q_off;
    const int32_t *kv_len = a.kv_len;
    const float4 *ml = a.part_ml;
    const float *po = a.part_o;
    pk::pdl_wait(plan, q_off, kv_len, ml, po);
    pk::pdl_launch_dependents();
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t id = (uint64_t)blockIdx.x * (kJoinThreads / 32) + threadIdx.x / 32, token = id / a.q_heads;
    const uint32_t qh = (uint32_t)(id % a.q_heads);
    if (token >= a.n_q || __ldcg(plan + 1 + a.R) == 0) return;  // uniform; no items where an offset is bad
    const uint32_t r = pk::warp_find_request(q_off, a.R, (int64_t)token);
    const int64_t qa = __ldcg(q_off + r), qb = __ldcg(q_off + r + 1);
    if ((int64_t)token < qa || (int64_t)token >= qb) return;
    const uint32_t pieces = pieces_of(tiles_of(a, good_length(a, __ldcg(kv_len + r))), (uint32_t)__ldcg(plan));
    if (pieces == 1) return;  // the row is written
    const uint32_t tok = (uint32_t)((int64_t)token - qa), head = qh / a.group, gh = qh % a.group;
    const uint32_t t = tok / a.tile_tokens % 2;
    const uint32_t row = tok % a.tile_tokens * a.tile_heads + gh % a.tile_heads;
    const uint32_t x = (tok / (2 * a.tile_tokens) * a.chunks + gh / a.tile_heads) * pieces;
    const uint64_t end = __ldcg(plan + 2 + r);
    auto part_of = [&](uint32_t piece) {
        return (((end - 1 - (x + piece)) * a.kv_heads + head) * 2 + t) * (uint64_t)kRows + row;
    };
    // the exponent of a piece's weights is ref - fine, which 32 bits may not hold: differences are taken part by part
    float ref = -FLT_MAX, fine = 0.0f;
    for (uint32_t p = 0; p < pieces; ++p) {
        const float4 y = __ldcg(ml + part_of(p));
        if ((y.x - ref) - (y.y - fine) > 0.0f) ref = y.x, fine = y.y;
    }
    constexpr int kPer = D / 32;
    float sum = 0.0f, o[kPer] = {};
#pragma unroll 4
    for (uint32_t p = 0; p < pieces; ++p) {
        const uint64_t at = part_of(p);
        const float4 y = __ldcg(ml + at);
        float z[kPer];
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
            const float2 u = __ldcg(reinterpret_cast<const float2 *>(po + at * D + lane * kPer + i));
            z[i] = u.x, z[i + 1] = u.y;
        }
        if (y.z == 0.0f) continue;  // a piece without a key that the row sees
        const float f = pk::ex2((y.x - ref) - (y.y - fine));
        sum += f * y.z;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] += f * z[i];
    }
    const float inv = sum == 0.0f ? 0.0f : a.v_scale / sum;
#pragma unroll
    for (int i = 0; i < kPer; i += 2)
        *reinterpret_cast<uint32_t *>(a.out + (int64_t)token * a.o_ts + (int64_t)qh * a.o_hs + lane * kPer + i) =
            pk::Elem<DT>::from2(o[i] * inv, o[i + 1] * inv);
    if (lane == 0 && a.lse)
        a.lse[token * a.q_heads + qh] = sum == 0.0f ? -INFINITY : (ref - fine + log2f(sum)) * 0.69314718055994531f;
}

// How the call is cut: what the host knows are bounds, the kernels see the lengths.
struct Plan {
    uint64_t units, items;  // at most: before the keys are cut, and behind
    uint32_t target, least;
    uint64_t plan_bytes, ml_bytes, o_bytes;
};

constexpr uint64_t kSms = 152;
constexpr uint32_t kLeastTiles = 4;
Plan plan_of(const pk_kv_cache &kv, uint32_t R, uint64_t n_q, uint32_t q_heads, uint64_t page_stride, uint32_t window,
             uint32_t sinks) {
    Plan p;
    p.units = pk_attend_prompt_items(n_q, R, q_heads, kv.kv_heads);
    p.least = kLeastTiles;
    uint64_t grans = (page_stride * kv.page_tokens + 15) / 16;
    if (window) grans = std::min<uint64_t>(grans, ((uint64_t)sinks + 15) / 16 + ((uint64_t)window + 2 * kRows + 14) / 16 + 1);
    const uint64_t most = ((grans + 7) / 8 + p.least - 1) / p.least;  // pieces of an item
    p.target = p.units <= 2 * kSms && most > 1 ? 2 * kSms : 0;
    p.items = p.target ? std::min(p.units + p.target, p.units * most) : p.units;
    p.plan_bytes = (((uint64_t)R + 2) * 8 + 31) & ~31ull;
    p.ml_bytes = p.target ? p.items * 2 * kRows * 16 : 0;
    p.o_bytes = p.target ? p.items * 2 * kRows * kv.head_dim * 4 : 0;
    return p;
}

template <int D, uint32_t DT>
cudaError_t launch(const Args &a, unsigned grid, const CUtensorMap &mq, cudaStream_t s) {
    constexpr size_t smem = Layout<D>::kBytes + sizeof(Small);
    static_assert(smem <= 227 * 1024, "shared memory of a block");
    static std::atomic<uint64_t> seen{0};
    cudaError_t e = pk_allow_smem(k_attend_chunk<D, DT>, smem, seen);
    if (e == cudaSuccess) e = pk_launch_smem(k_attend_chunk<D, DT>, grid, kThreads, smem, s, a, mq);
    if (e == cudaSuccess && a.target)
        e = pk_launch(k_chunk_join<D, DT>, (unsigned)((a.n_q * a.q_heads + kJoinThreads / 32 - 1) / (kJoinThreads / 32)),
                      kJoinThreads, s, a);
    return e;
}

}  // namespace

uint64_t pk_attend_chunk_scratch_bytes_impl(const pk_kv_cache &kv, uint32_t R, uint64_t n_q, uint32_t q_heads,
                                            uint64_t page_stride, uint32_t window, uint32_t sinks) {
    const Plan p = plan_of(kv, R, n_q, q_heads, page_stride, window, sinks);
    if (p.items > 0x7fffffffull) return UINT64_MAX;
    return p.plan_bytes + p.ml_bytes + p.o_bytes;
}

cudaError_t pk_launch_attend_chunk(const pk_kv_cache &kv, uint32_t dtype, const pk_heads &q, const pk_heads &out,
                                   float *lse, uint64_t n_q, const int64_t *q_off, uint32_t R, uint32_t q_heads,
                                   float scale, uint32_t window, uint32_t sinks, const int32_t *kv_len,
                                   const uint32_t *pages, uint64_t page_stride, void *scratch, int32_t *status,
                                   cudaStream_t s) {
    const Plan p = plan_of(kv, R, n_q, q_heads, page_stride, window, sinks);
    Args a;
    a.pool = static_cast<const uint8_t *>(kv.pool_dev);
    a.page_bytes = pk_kv_page_bytes(kv.page_tokens, kv.kv_heads, kv.head_dim);
    a.n_slots = kv.n_slots;
    a.page_stride = page_stride;
    a.positions = page_stride * kv.page_tokens;
    a.page_grans = kv.page_tokens / 16;
    a.q_off = q_off;
    a.kv_len = kv_len;
    a.pages = pages;
    a.R = R;
    a.q_heads = q_heads;
    a.kv_heads = kv.kv_heads;
    a.group = q_heads / kv.kv_heads;
    a.n_q = n_q;
    a.tile_heads = std::min<uint32_t>(a.group, kRows);
    a.tile_tokens = kRows / a.tile_heads;
    a.chunks = (a.group + a.tile_heads - 1) / a.tile_heads;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.sink_grans = (a.sinks + 15) / 16;
    a.scale2 = (float)((double)scale * kv.k_scale * 1.4426950408889634);
    a.v_scale = kv.v_scale;
    a.out = static_cast<uint16_t *>(out.p);
    a.o_ts = out.tok_stride;
    a.o_hs = out.head_stride;
    a.wide_out = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && a.o_ts % 16 == 0 && a.o_hs % 16 == 0;
    a.lse = lse;
    a.target = p.target;
    a.least = p.least;
    a.listed = R > 32;
    a.most_items = (uint32_t)p.items;
    uint8_t *at = static_cast<uint8_t *>(scratch);
    a.plan = reinterpret_cast<uint64_t *>(at);
    a.part_ml = reinterpret_cast<float4 *>(at + p.plan_bytes);
    a.part_o = reinterpret_cast<float *>(at + p.plan_bytes + p.ml_bytes);
    a.status = status;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    CUtensorMap mq;
    if (e == cudaSuccess) e = map_of(&mq, q, n_q, q_heads, kv.head_dim, dtype, a.tile_tokens, a.tile_heads);
    if (e == cudaSuccess && a.listed) e = pk_launch(k_chunk_plan, 1, kPlanThreads, s, a);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)std::min<uint64_t>(p.items, (uint64_t)sms);
    if (kv.head_dim == 128)
        e = dtype == PK_BF16 ? launch<128, PK_BF16>(a, grid, mq, s) : launch<128, PK_FP16>(a, grid, mq, s);
    else
        e = dtype == PK_BF16 ? launch<64, PK_BF16>(a, grid, mq, s) : launch<64, PK_FP16>(a, grid, mq, s);
    return e != cudaSuccess ? e : cudaGetLastError();
}
