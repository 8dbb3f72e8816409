// pk_attend_prompt.cu -- causal attention over packed prompts with grouped
// heads (pk_attend_prompt).
//
// out = sum_j p_j v_j / sum_j p_j over the keys j that a query sees, p_j =
// 2^(s_j - ref), s_j = scale log2(e) q . k_j.  Any ref gives the same quotient:
// it stays as long as a tile's weights of a row sum to 2^15 at most, which is
// looked at after the weights are taken, not before.  So most tiles cost one
// pass over the scores and no rescaling of the output; lse = ln 2 (ref + log2 of
// the sum).  Scores, sums and outputs are 32 bits; the weights round to the
// operands' type for the second product, which takes no other.
//
// Arithmetic: 4 D products a (query, key, head) on the tensor pipe, one 2^x on a
// unit of 32 a clock.  A 128 x 128 tile of D = 128 is 1024 clocks of the first
// and 512 of the second; at D = 64 the two are even.  So both have to run at
// once: an item is two tiles, one's weights are taken while the other's products
// run.  Rows of a tile are (token, head of the group), so K and V are read once
// for a group.  Two tiles, because their scores (256 columns) and outputs
// (2 D) fill the TMEM at D = 128.  At D = 64 a third buffer of scores, made
// ahead, changed nothing (128 | 128 us), nor did halves of a tile to two
// warpgroups (675 | 776 us at D = 128, two prompts of 8192).
//
// Two prompts of 8192 (32 heads over 8, D = 128, bf16): 604 us, 1.5 PFLOP/s,
// tensor pipe 70% busy at 1.8 GHz under the power limit.  12 of 1500 behind 2048
// keys (12 over 4, D = 64): 121 us, 0.77 PFLOP/s: a tile's chain (scores, 2^x,
// product) and five items an SM.  8 of 512: 32 us, 3 short items an SM: the
// chain's latency.
#include <cuda.h>
#include <cuda_runtime.h>
#include <float.h>

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
constexpr int kThreads = 384;
constexpr float kTop = 32768.0f;  // a tile's weights of a row sum to no more, so each fits a half (65504)
constexpr float kBase = 4.0f;     // the largest weight when the reference moves: 2^kBase, so 128 stay below 2^11
constexpr float kFar = 16777216.0f;  // scores (times log2 e) from here on are further apart than a weight's exponents:
                                     // one 32-bit reference cannot lie kBase below one
constexpr int kPlanThreads = 1024;
constexpr uint64_t kLongKeys = 1280;  // keys a request, on average, from which blocks take their items as they come

struct Args {
    uint16_t *out;
    int64_t o_ts, o_hs;
    bool wide_out;  // every 16 values of out start on 32 bytes
    float *lse;
    const int64_t *q_off, *k_off;
    uint64_t *tile_off;  // [R + 1]: items of one KV head in the requests before r; NULL for up to 32 requests
    uint32_t R, q_heads, kv_heads, group;
    uint64_t n_q, n_k;
    uint32_t most_items;  // no call has more
    uint32_t tile_tokens, tile_heads, chunks;  // of a tile; tiles that it takes for a group's heads
    float scale2;  // scale * log2 e
    int32_t *status;
};

__device__ __forceinline__ bool bad_offsets(int64_t qa, int64_t qb, int64_t ka, int64_t kb, uint64_t n_q,
                                            uint64_t n_k) {
    return qa < 0 || qb < qa || (uint64_t)qb > n_q || ka < 0 || kb < ka || (uint64_t)kb > n_k;
}

// Items of one KV head in a request of n queries.
__device__ __forceinline__ uint32_t items_of(int64_t n, uint32_t item_tokens, uint32_t chunks) {
    return ((uint32_t)n + item_tokens - 1) / item_tokens * chunks;
}

// tile_off: how many items of one KV head the requests before each one have;
// all zero where an offset is out of order or range.
__global__ void __launch_bounds__(kPlanThreads)
k_prompt_tiles(const int64_t *q_off, const int64_t *k_off, uint32_t R, uint64_t n_q, uint64_t n_k,
               uint32_t item_tokens, uint32_t chunks, uint64_t *tile_off, int32_t *status) {
    __shared__ uint64_t warp_sum[32];
    __shared__ uint32_t bad;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    if (tid == 0) bad = 0;
    pk::pdl_wait(q_off, k_off, tile_off, status);
    pk::pdl_launch_dependents();
    __syncthreads();
    uint64_t base = 0;
    for (uint64_t r0 = 0; r0 < R; r0 += kPlanThreads) {
        const uint64_t r = r0 + tid;
        uint64_t n = 0;
        if (r < R) {
            const int64_t a = __ldcg(q_off + r), b = __ldcg(q_off + r + 1);
            const int64_t e = __ldcg(k_off + r), f = __ldcg(k_off + r + 1);
            if (bad_offsets(a, b, e, f, n_q, n_k))
                bad = 1;
            else
                n = items_of(b - a, item_tokens, chunks);
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
        if (r < R) tile_off[r + 1] = before + scan;
        base += total;
        __syncthreads();
    }
    if (tid == 0) tile_off[0] = 0;
    if (bad) {
        for (uint64_t r = tid; r <= R; r += kPlanThreads) tile_off[r] = 0;
        if (tid == 0) pk::set_status(status, PK_ERR_ARG);
    }
}

// Shared memory of a CTA, from a 1024-byte boundary: Q (two tiles), the ring of K and V tiles, then Small.
template <int D>
struct Layout {
    static constexpr uint32_t kTile = 128 * D * 2;  // 128 rows; blocks of [128][64] values, 16 KB each
    static constexpr uint32_t kStages = D == 128 ? 5 : 8;
    static constexpr uint32_t kRing = 2 * kTile;
    static constexpr uint32_t kBytes = kRing + kStages * kTile;
};

struct Small {
    uint64_t full[8], empty[8];    // ring stages: tile ready (loaded, and an edge tile's V made finite); no longer read
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], p_ready[2], o_done[2];
    uint64_t edge_v[4];            // an edge tile's V loaded, by edge tile
    uint64_t over;                 // every product that was issued is done (a matrix warp that gave up)
    uint64_t next_full[4], next_empty[4];  // an answer on the next item is there; its readers have it
    alignas(16) uint64_t next[4][2];       // the answers
    uint32_t tmem, abort;
    int32_t work[8][2];            // by item with keys: key tiles of its two tiles, for the matrix warp; 0, 0 ends it
    uint32_t epilogues[8];         // by softmax warp: items whose outputs it has written
    uint32_t any_bad[2][2];        // by item parity and half of the dimensions: bad_row holds something
    int32_t bad_row[2][128];       // first key of an edge tile whose V is not finite, by dimension
    uint32_t item_end[32];         // up to 32 requests: items of one KV head in those up to each, and where they lie
    int32_t q_start[32], k_start[32], q_len[32], k_len[32];
};

// Up to 32 requests every CTA counts the items itself, a lane a request, and keeps
// the list in shared memory: no launch of k_prompt_tiles, and no loads to wait for
// at each item.
__device__ __forceinline__ void count_items(const Args &a, Small &sm, const int64_t *q_off, const int64_t *k_off) {
    const uint32_t lane = threadIdx.x & 31;
    int64_t qa = 0, qb = 0, ka = 0, kb = 0;
    if (lane < a.R) {
        qa = __ldcg(q_off + lane), qb = __ldcg(q_off + lane + 1);
        ka = __ldcg(k_off + lane), kb = __ldcg(k_off + lane + 1);
    }
    const bool bad = __any_sync(0xffffffffu, bad_offsets(qa, qb, ka, kb, a.n_q, a.n_k));
    if (bad && lane == 0) pk::set_status(a.status, PK_ERR_ARG);
    uint32_t scan = bad ? 0 : items_of(qb - qa, 2 * a.tile_tokens, a.chunks);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    sm.item_end[lane] = scan;
    sm.q_start[lane] = (int32_t)qa;
    sm.k_start[lane] = (int32_t)ka;
    sm.q_len[lane] = (int32_t)(qb - qa);
    sm.k_len[lane] = (int32_t)(kb - ka);
}

// One item: 2 tiles of `tokens` query tokens times `heads` heads of one group.
struct Item {
    int32_t q0, k0, lq, lk, tok0, chunk, head;
    int32_t n_tiles[2], first_last[2], n_all, first_edge;
};

// Item `index` of the call's; false: there are not so many, or an offset is out of range.
__device__ __forceinline__ bool find_item(const Args &a, const Small &sm, const uint64_t *tile_off, const int64_t *q_off,
                                          const int64_t *k_off, uint32_t index, Item &it) {
    const uint32_t tile = index / a.kv_heads;
    it.head = (int32_t)(index - tile * a.kv_heads);
    it.q0 = it.k0 = it.lq = it.lk = 0;
    uint32_t x = 0;  // which of the request's items
    if (tile_off) {
        if (tile < __ldcg(tile_off + a.R)) {
            const uint32_t r = pk::warp_find_request(reinterpret_cast<const int64_t *>(tile_off), a.R, (int64_t)tile);
            it.q0 = (int32_t)__ldcg(q_off + r);
            it.k0 = (int32_t)__ldcg(k_off + r);
            it.lq = (int32_t)__ldcg(q_off + r + 1) - it.q0;
            it.lk = (int32_t)__ldcg(k_off + r + 1) - it.k0;
            x = (uint32_t)__ldcg(tile_off + r + 1) - 1 - tile;
        }
    } else {
        const uint32_t lane = threadIdx.x & 31;
        const uint32_t r = __popc(__ballot_sync(0xffffffffu, sm.item_end[lane] <= tile));
        if (r < 32) {  // (requests past R repeat the total)
            it.q0 = sm.q_start[r];
            it.k0 = sm.k_start[r];
            it.lq = sm.q_len[r];
            it.lk = sm.k_len[r];
            x = sm.item_end[r] - 1 - tile;
        }
    }
    // the last queries first: they have the most keys
    it.chunk = (int32_t)(x % a.chunks);
    it.tok0 = (int32_t)(x / a.chunks) * 2 * (int32_t)a.tile_tokens;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int32_t t0 = it.tok0 + t * (int32_t)a.tile_tokens, t1 = min(t0 + (int32_t)a.tile_tokens, it.lq);
        const int32_t keys = t1 > t0 ? t1 + it.lk - it.lq : 0;  // that some query of the tile sees
        it.n_tiles[t] = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
        it.first_last[t] = t0 + it.lk - it.lq;                  // last key of the tile's first query
    }
    it.n_all = max(it.n_tiles[0], it.n_tiles[1]);
    // From this key tile on, some query does not see some key: p = 0 there, which must not meet an infinity or NaN
    // of V.  At most three tiles, as an item has at most 256 queries.
    it.first_edge = it.first_last[0] + 1 >= kKeys ? (it.first_last[0] + 1) / kKeys : 0;
    return it.lq > 0;
}

// How a block gets to its next item.
// Fixed: the grid has a block an SM, and every other turn runs through the blocks backwards: one that got the heaviest
// item of a turn gets the lightest of the next.
// Else the grid has a block for every item, and a running one takes the place of the next that has not started, until
// none is left: the SM that is done first gets the next item.  Item n + 1 is asked for near the end of item n's loads.
// It evens out what is left over at the end, but the next block number takes time to come, a block that waits for it
// cannot look for its item early, and the next kernel starts later.  Fixed | taken, D = 128: 32 prompts of 512 103 |
// 117 us, 8 of 2048 105 | 94, two of 8192 616 | 604; D = 64: 40 of 700 behind 300 keys 89 | 100, 12 of 1500 behind 2048
// 130 | 118.  So the keys per request decide (kLongKeys).
__device__ __forceinline__ void ask_next(uint32_t answer, uint32_t bar) {
    pk::mbar_expect(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer),
                 "r"(bar)
                 : "memory");
}
// n-th answer; false: no block was left.  ok turns false when none came.
__device__ __forceinline__ bool next_taken(Small &sm, uint32_t n, bool reader, uint32_t &index, bool &ok) {
    ok = pk::mbar_wait_warp(pk::smem_addr(&sm.next_full[n & 3]), n >> 2 & 1);
    if (!ok) return false;
    const volatile uint64_t *answer = sm.next[n & 3];
    const uint64_t lo = answer[0], hi = answer[1];
    uint32_t got;
    asm volatile(
        "{\n .reg .pred p;\n .reg .b128 r;\n mov.b128 r, {%2, %3};\n"
        " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n"
        " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
        : "=r"(got), "=r"(index)
        : "l"(lo), "l"(hi));
    if (reader) {
        pk::fence_proxy_async();  // the slot's next answer comes by the async proxy
        __syncwarp();
        if ((threadIdx.x & 31) == 0) pk::mbar_arrive(pk::smem_addr(&sm.next_empty[n & 3]));
    }
    return got != 0;
}

// Registers move to the softmax warps, whose scores on their way and weights do not fit 168: 256 * 200 + 128 * 104 =
// 384 * 168, the launch's own.
constexpr int kRegsSoftmax = 200, kRegsOther = 104;
constexpr uint32_t kWarpLoad = 8, kWarpMma = 9, kWarpClean = 10;  // warps 0-7: softmax

// One CTA an SM takes one item after another.  Warp roles: one loads Q, K and V by TMA,
// one issues the matrix products, two look after V at the causal edge, and
// two warpgroups of four turn scores into weights, a thread a row, for one of
// the item's two tiles each: while one tile's scores are weighed the other's
// products run.  TMEM: scores of the tiles (128 columns each; the weights, two
// to a column, take the place of scores that have been read), then their outputs
// (D columns each).  Every counter of a barrier's use runs on over the items, so
// the next item's loads and first products run under this one's end.
template <int D, uint32_t DT, bool kFixed>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_prompt(const Args a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                const __grid_constant__ CUtensorMap map_v) {
    using L = Layout<D>;
    // all the shared memory that the kernel has, so that it starts on the swizzle's 1024 bytes
    extern __shared__ __align__(1024) uint8_t smem_p[];
    Small &sm = *reinterpret_cast<Small *>(smem_p + L::kBytes);
    const uint32_t smem = pk::smem_addr(smem_p);
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = pk::uniform(tid >> 5);
    if (smem & 1023) {
        if (tid == 0) pk::set_status(a.status, PK_ERR_CUDA);
        return;
    }

    if (tid == 0) {
        for (uint32_t i = 0; i < L::kStages; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.full[i]), 2);  // the loader twice, or the two cleaning warps
            pk::mbar_init(pk::smem_addr(&sm.empty[i]), 1);
        }
        for (int t = 0; t < 2; ++t) {
            pk::mbar_init(pk::smem_addr(&sm.q_full[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.q_empty[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.s_full[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.p_ready[t]), 4);
            pk::mbar_init(pk::smem_addr(&sm.o_done[t]), 1);
        }
        for (int i = 0; i < 4; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.edge_v[i]), 1);
            pk::mbar_init(pk::smem_addr(&sm.next_full[i]), 1);
            pk::mbar_init(pk::smem_addr(&sm.next_empty[i]), 10);  // cleaning and softmax warps
        }
        pk::mbar_init(pk::smem_addr(&sm.over), 1);
        pk::mbar_fence_init();
        sm.abort = 0;
        for (int i = 0; i < 8; ++i) sm.epilogues[i] = 0;
    }
    if (warp == kWarpMma) pk::tmem_alloc(pk::smem_addr(&sm.tmem), 512);
    const uint64_t *tile_off = a.tile_off;
    const int64_t *q_off = a.q_off, *k_off = a.k_off;
    pk::pdl_wait(tile_off, q_off, k_off);
    pk::pdl_launch_dependents();
    if (warp == kWarpLoad && !tile_off) count_items(a, sm, q_off, k_off);
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
    uint32_t turn = 0, index = blockIdx.x;  // items before the present one; its number
    auto next_index = [&](uint32_t n, bool reader, uint32_t &index, bool &ok) {
        if (!kFixed) return next_taken(sm, n, reader, index, ok);
        const uint64_t next = (uint64_t)(n + 1) * gridDim.x + (n & 1 ? blockIdx.x : gridDim.x - 1 - blockIdx.x);
        index = (uint32_t)next;  // less than 2^31 if it is one
        return next < a.most_items;
    };
    bool more = find_item(a, sm, tile_off, q_off, k_off, index, it);
    if (warp >= kWarpLoad) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kWarpLoad) {
            uint32_t n = 0, edges = 0, nq[2] = {0, 0}, items = 0;  // ring stages, edge tiles, Q tiles, items so far
            uint32_t asked = 0, dirty_last = 0;  // dirty_last: bit i is 1 where the stage i before the next one is an edge tile's
            bool ok = true;
            pk::fence_proxy_async();
            while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
                auto ask = [&]() {  // by lane 0, once an item
                    ok = ok && (turn < 4 || pk::mbar_wait(pk::smem_addr(&sm.next_empty[turn & 3]), (turn / 4 + 1) & 1));
                    if (ok) ask_next(pk::smem_addr(sm.next[turn & 3]), pk::smem_addr(&sm.next_full[turn & 3])), ++asked;
                };
                if (lane == 0 && !kFixed && it.n_all <= 3) ask();
                if (lane == 0 && it.n_all > 0) {
                    // its reader, at most four items behind, sees it by way of the first K tile's barrier
                    sm.work[items & 7][0] = it.n_tiles[0];
                    sm.work[items & 7][1] = it.n_tiles[1];
                    ++items;
                    const uint32_t q_bytes = a.tile_tokens * a.tile_heads * 128 * (D / 64);
                    for (int32_t j = 0; ok && j < it.n_all; ++j) {
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv) {
                            const uint32_t st = n % L::kStages;
                            const bool dirty = kv && j >= it.first_edge;
                            const uint32_t bar = pk::smem_addr(dirty ? &sm.edge_v[edges & 3] : &sm.full[st]);
                            ok = ok && (n < L::kStages ||
                                        pk::mbar_wait(pk::smem_addr(&sm.empty[st]), (n / L::kStages + 1) & 1));
                            if (!ok) break;
                            // only now: the barrier's earlier phase is over, as the stage was read
                            if (!dirty) pk::mbar_arrive(bar);
                            pk::mbar_expect(bar, L::kTile);
#pragma unroll
                            for (int b = 0; b < D / 64; ++b)
                                pk::tile_load3(smem + L::kRing + st * L::kTile + b * 16384, kv ? &map_v : &map_k, b * 64,
                                               it.head, it.k0 + j * kKeys, bar);
                            ++n;
                            edges += dirty;
                            dirty_last = dirty_last << 1 | (uint32_t)dirty;
                        }
                        if (j == 0) {  // Q behind the first tiles, which need not wait for the last item's Q
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
                                                   it.head * (int)a.group + it.chunk * (int)a.tile_heads,
                                                   it.q0 + it.tok0 + t * (int)a.tile_tokens, bar);
                                ++nq[t];
                            }
                        }
                        if (!kFixed && it.n_all > 3 && j == it.n_all - 3) ask();
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                more = next_index(turn, false, index, ok);
                ++turn;
                if (more) more = find_item(a, sm, tile_off, q_off, k_off, index, it);
            }
            if (lane == 0) {
                const uint32_t st = n % L::kStages;
                ok = ok && (n < L::kStages ||
                            pk::mbar_wait(pk::smem_addr(&sm.empty[st]), (n / L::kStages + 1) & 1));
                if (ok) {  // the matrix warp's end: a stage without a tile
                    sm.work[items & 7][0] = sm.work[items & 7][1] = 0;
                    pk::mbar_arrive(pk::smem_addr(&sm.full[st]));
                    pk::mbar_arrive(pk::smem_addr(&sm.full[st]));
                    ++n;
                    dirty_last <<= 1;
                }
                if (!ok) give_up();
                // no copy of its own stays in flight, and no answer on its way; each by the barrier that its own
                // arrivals complete, so that no wait depends on a warp that gave up
                if (asked > turn) pk::mbar_wait(pk::smem_addr(&sm.next_full[turn & 3]), turn >> 2 & 1);
                for (uint32_t i = n > L::kStages ? n - L::kStages : 0; i < n; ++i)
                    if (!(dirty_last >> (n - 1 - i) & 1))
                        pk::mbar_wait(pk::smem_addr(&sm.full[i % L::kStages]), (i / L::kStages) & 1);
                for (uint32_t i = edges > 4 ? edges - 4 : 0; i < edges; ++i)
                    pk::mbar_wait(pk::smem_addr(&sm.edge_v[i & 3]), (i >> 2) & 1);
                for (int t = 0; t < 2; ++t)
                    if (nq[t]) pk::mbar_wait(pk::smem_addr(&sm.q_full[t]), (nq[t] - 1) & 1);
            }
            __syncwarp();
        } else if (warp == kWarpMma) {
            const uint32_t qk_kind = pk::mma_idesc(DT == PK_BF16, 128, 128, false) |
                                     (a.scale2 < 0.0f ? 1u << 13 : 0u);  // a negative scale negates Q
            constexpr uint32_t kPv = pk::mma_idesc(DT == PK_BF16, 128, D, true);
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
        } else {
            // V of the tiles at the causal edge and at the request's end: rows past its last key become 0, and so do
            // infinities and NaN, which are noted for the queries that do attend them.  Each of the two warps has its
            // own half of the dimensions.
            constexpr uint32_t kChunks = D / 16;  // 16-byte chunks of a row that a warp looks at
            const uint32_t half = warp - kWarpClean;
            uint32_t base = 0, edges = 0, items = 0;
            bool ok = true;
            while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
                int32_t *bad_row = sm.bad_row[items & 1];
                if (it.first_edge < it.n_all) {
                    // the item before the last one shared these notes: its outputs must have been written
                    uint64_t t0 = 0, t1 = 0;
                    while (items >= 2) {
                        uint32_t done;
                        asm volatile("ld.acquire.cta.shared.u32 %0, [%1];" : "=r"(done) : "r"(pk::smem_addr(&sm.epilogues[lane & 7])) : "memory");
                        if (__all_sync(0xffffffffu, (int32_t)(done - (items - 1)) >= 0)) break;
                        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
                        t1 = __shfl_sync(0xffffffffu, t1, 0);
                        if (t0 == 0) t0 = t1;
                        if (t1 - t0 > pk::kMbarLimitNs) {
                            ok = false;
                            break;
                        }
                    }
                    for (uint32_t d = lane; d < D / 2; d += 32) bad_row[half * (D / 2) + d] = 0x7fffffff;
                    if (lane == 0) sm.any_bad[items & 1][half] = 0;
                    __syncwarp();
                }
                for (int32_t j = it.first_edge; ok && j < it.n_all; ++j, ++edges) {
                    const uint32_t st = (base + 2 * j + 1) % L::kStages;
                    ok = pk::mbar_wait_warp(pk::smem_addr(&sm.edge_v[edges & 3]), (edges >> 2) & 1);
                    if (!ok) break;
                    uint8_t *v = smem_p + L::kRing + st * L::kTile + (D == 128 ? half * 16384 : 0);
                    // eight 16-byte pieces of a lane at once: mostly there is nothing to do
                    auto piece = [&](uint32_t x) {
                        const uint32_t row = x / kChunks, chunk = x % kChunks + (D == 128 ? 0 : half * kChunks);
                        return reinterpret_cast<uint4 *>(v + row * 128 + ((chunk ^ (row & 7)) << 4));
                    };
                    constexpr uint32_t kInf = pk::Elem<DT>::kInfBits;
#pragma unroll 1
                    for (uint32_t x0 = lane; x0 < 128 * kChunks; x0 += 256) {
                        uint4 u[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) u[i] = *piece(x0 + 32 * i);
                        uint32_t m = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            m = __vmaxu2(m, __vmaxu2(u[i].x & 0x7fff7fffu, u[i].y & 0x7fff7fffu));
                            m = __vmaxu2(m, __vmaxu2(u[i].z & 0x7fff7fffu, u[i].w & 0x7fff7fffu));
                        }
                        const bool past = j * kKeys + (int32_t)((x0 + 224) / kChunks) >= it.lk;
                        if (!past && (m & 0xffffu) < kInf && m >> 16 < kInf) continue;
#pragma unroll 1
                        for (uint32_t x = x0; x < x0 + 256; x += 32) {
                            const uint32_t row = x / kChunks, chunk = x % kChunks + (D == 128 ? 0 : half * kChunks);
                            const int32_t key = j * kKeys + (int32_t)row;
                            if (key >= it.lk) {
                                *piece(x) = make_uint4(0, 0, 0, 0);
                                continue;
                            }
                            const uint4 y = *piece(x);
                            uint32_t w[4] = {y.x, y.y, y.z, y.w};
                            bool found = false;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t d = (D == 128 ? half * 64 : 0) + chunk * 8 + 2 * i;
                                if ((w[i] & 0x7fffu) >= kInf) {
                                    atomicMin(&bad_row[d], key);
                                    w[i] &= 0xffff0000u;
                                    found = true;
                                }
                                if ((w[i] >> 16 & 0x7fffu) >= kInf) {
                                    atomicMin(&bad_row[d + 1], key);
                                    w[i] &= 0xffffu;
                                    found = true;
                                }
                            }
                            if (found) {
                                *piece(x) = make_uint4(w[0], w[1], w[2], w[3]);
                                sm.any_bad[items & 1][half] = 1;
                            }
                        }
                    }
                    pk::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[st]));
                }
                base += 2 * it.n_all;
                ++items;
                if (!ok) break;
                more = next_index(turn, true, index, ok);
                ++turn;
                if (more) more = find_item(a, sm, tile_off, q_off, k_off, index, it);
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
        uint32_t ni = 0, items = 0;  // key tiles weighed so far
        bool ok = true;
        while (more && ok && !__any_sync(0xffffffffu, *abort != 0)) {
            const int32_t n_tiles = t ? it.n_tiles[1] : it.n_tiles[0];
            const int32_t first_last = t ? it.first_last[1] : it.first_last[0];
            const int32_t tok = it.tok0 + (int32_t)(t * a.tile_tokens) + row_tok;
            const int32_t gh = it.chunk * (int32_t)a.tile_heads + row_head;
            const bool on = row_tok < (int32_t)a.tile_tokens && tok < it.lq && gh < (int32_t)a.group;
            const int32_t last = on ? tok + it.lk - it.lq : -1;
            const int64_t q_row = it.q0 + tok;
            const uint32_t qh = it.head * a.group + gh;
            const bool notes = it.first_edge < n_tiles;  // only then are this item's notes sure to be there
            auto take_next = [&]() {
                if (ok) more = next_index(turn, true, index, ok);
                ++turn;
                if (more) more = find_item(a, sm, tile_off, q_off, k_off, index, it);
            };
            if (kFixed) take_next();
            // a weight is 2^(score - ref + fine), and fine is 0 but for a reference of kFar and more
            float ref = -FLT_MAX, fine = 0.0f, sum = 0.0f;
#pragma unroll 1
            for (int32_t j = 0; ok && j < n_tiles; ++j, ++ni) {
                ok = pk::mbar_wait_warp(pk::smem_addr(&sm.s_full[t]), ni & 1);
                if (!ok) break;
                pk::tmem_fence_after();
                const bool edge = j * kKeys + kKeys - 1 > first_last;
                const int32_t see = last - j * kKeys;  // columns up to here
                uint32_t x[3][32];
                // Chunk c of the scores, 32 keys.  Loads run ahead (1 and 2 behind 0's use, 3 behind 1's).  Masked or
                // not is known at compile time: as a branch around the masking it cost 170 of 1010 cycles a tile.
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
                            if (32 * c + i > see) y[i] = 0xff800000u;
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
                            p[c / 2][c % 2 * 16 + i / 2] = pk::Elem<DT>::from2(z.x, z.y);
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
                                const bool masked = edge && 16 * c + i + h > see;
                                w[h] = masked ? 0.0f : pk::ex2(fmaf(__uint_as_float(y[i + h]), scale2, -ref) + fine);
                                s += w[h];
                            }
                            p[c / 4][c % 4 * 8 + i / 2] = pk::Elem<DT>::from2(w[0], w[1]);
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
                // the pass done again.
                // Once does: behind a move no weight is above 2^(kBase + 2).  Rows without a query, of a tile's unused
                // rows too, which hold anything, have no say.
                float part = weigh_any();
                if (__any_sync(0xffffffffu, on && part > kTop)) {
                    move_ref(on && part > kTop);
                    if (!ok) break;
                    part = weigh_any();
                }
                if (!ok) break;
                sum += part;
                pk::tmem_store32(ts, p[0]);  // over the scores, which every pass is done with
                pk::tmem_store32(ts + 32, p[1]);
                pk::tmem_wait_store();
                pk::tmem_fence_before();
                __syncwarp();
                if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.p_ready[t]));
            }
            if (!kFixed) take_next();  // while the last product runs
            if (ok && n_tiles > 0) ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (ni - 1) & 1);
            if (!ok) break;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            if (on && a.lse)
                a.lse[q_row * a.q_heads + qh] = sum == 0.0f ? -INFINITY : (ref - fine + log2f(sum)) * 0.69314718055994531f;
            uint16_t *dst = a.out + q_row * a.o_ts + (int64_t)qh * a.o_hs;
            const bool bad = notes && (sm.any_bad[items & 1][0] | sm.any_bad[items & 1][1]) != 0;
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
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    float f0 = __uint_as_float(z[i]) * inv, f1 = __uint_as_float(z[i + 1]) * inv;
                    if (n_tiles == 0 || inv == 0.0f) f0 = f1 = 0.0f;
                    w[i / 2] = pk::Elem<DT>::from2(f0, f1);
                }
                if (bad) {
                    const int32_t *row = sm.bad_row[items & 1] + 16 * c;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        if (row[i] <= last) w[i / 2] |= 0x7fffu;
                        if (row[i + 1] <= last) w[i / 2] |= 0x7fff0000u;
                    }
                }
                pk::store32(dst + 16 * c, a.wide_out, w);
            }
            __syncwarp();
            ++items;
            if (lane == 0)
                asm volatile("st.release.cta.shared.u32 [%0], %1;" ::"r"(pk::smem_addr(&sm.epilogues[warp])), "r"(items) : "memory");
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

template <int D, uint32_t DT, bool kFixed>
cudaError_t launch_as(const Args &a, unsigned grid, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv,
                   cudaStream_t s) {
    constexpr size_t smem = Layout<D>::kBytes + sizeof(Small);
    static_assert(smem <= 227 * 1024, "shared memory of a block");
    static std::atomic<uint64_t> seen{0};
    const cudaError_t e = pk_allow_smem(k_attend_prompt<D, DT, kFixed>, smem, seen);
    return e != cudaSuccess ? e : pk_launch_smem(k_attend_prompt<D, DT, kFixed>, grid, kThreads, smem, s, a, mq, mk, mv);
}

template <int D, uint32_t DT>
cudaError_t launch(const Args &a, bool fixed, unsigned grid, const CUtensorMap &mq, const CUtensorMap &mk,
                   const CUtensorMap &mv, cudaStream_t s) {
    return fixed ? launch_as<D, DT, true>(a, grid, mq, mk, mv, s) : launch_as<D, DT, false>(a, grid, mq, mk, mv, s);
}

}  // namespace

// A tile: all heads of the group for as many tokens as fit 128 rows, or 128 heads of one token.
static uint32_t tile_heads_of(uint32_t group) { return group < (uint32_t)kRows ? group : kRows; }

// Every request rounds its tokens up to whole items: at most one more each.
uint64_t pk_attend_prompt_items(uint64_t n_q, uint32_t R, uint32_t q_heads, uint32_t kv_heads) {
    const uint32_t group = q_heads / kv_heads, heads = tile_heads_of(group);
    return (n_q / (2 * (kRows / heads)) + R) * ((group + heads - 1) / heads) * kv_heads;
}

cudaError_t pk_launch_attend_prompt(uint32_t dtype, const pk_heads &q, const pk_heads &k, const pk_heads &v,
                                    const pk_heads &out, float *lse, uint64_t n_q, uint64_t n_k, const int64_t *q_off,
                                    const int64_t *k_off, uint32_t R, uint32_t q_heads, uint32_t kv_heads,
                                    uint32_t head_dim, float scale, void *scratch, int32_t *status, cudaStream_t s) {
    Args a;
    a.out = static_cast<uint16_t *>(out.p);
    a.o_ts = out.tok_stride, a.o_hs = out.head_stride;
    a.wide_out = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && a.o_ts % 16 == 0 && a.o_hs % 16 == 0;
    a.lse = lse;
    a.q_off = q_off;
    a.k_off = k_off;
    a.tile_off = R > 32 ? static_cast<uint64_t *>(scratch) : nullptr;
    a.R = R;
    a.n_q = n_q;
    a.n_k = n_k;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.group = q_heads / kv_heads;
    a.tile_heads = tile_heads_of(a.group);
    a.tile_tokens = kRows / a.tile_heads;
    a.chunks = (a.group + a.tile_heads - 1) / a.tile_heads;
    a.scale2 = (float)((double)scale * 1.4426950408889634);
    a.status = status;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return e;
    CUtensorMap mq, mk{}, mv{};
    // without keys no key tile is ever loaded, and the maps are never read
    if ((e = map_of(&mq, q, n_q, q_heads, head_dim, dtype, a.tile_tokens, a.tile_heads)) != cudaSuccess ||
        (n_k && (e = map_of(&mk, k, n_k, kv_heads, head_dim, dtype, kKeys, 1)) != cudaSuccess) ||
        (n_k && (e = map_of(&mv, v, n_k, kv_heads, head_dim, dtype, kKeys, 1)) != cudaSuccess))
        return e;
    const uint32_t item_tokens = 2 * a.tile_tokens;
    if (a.tile_off)
        e = pk_launch(k_prompt_tiles, 1, kPlanThreads, s, q_off, k_off, R, n_q, n_k, item_tokens, a.chunks,
                      a.tile_off, status);
    if (e != cudaSuccess) return e;
    const uint64_t items = pk_attend_prompt_items(n_q, R, q_heads, kv_heads);  // fewer than 2^31, looked at before
    a.most_items = (uint32_t)items;
    const bool fixed = items <= (uint64_t)sms || n_k < kLongKeys * R;
    const unsigned grid = fixed && items > (uint64_t)sms ? (unsigned)sms : (unsigned)items;
    if (head_dim == 128)
        e = dtype == PK_BF16 ? launch<128, PK_BF16>(a, fixed, grid, mq, mk, mv, s) : launch<128, PK_FP16>(a, fixed, grid, mq, mk, mv, s);
    else
        e = dtype == PK_BF16 ? launch<64, PK_BF16>(a, fixed, grid, mq, mk, mv, s) : launch<64, PK_FP16>(a, fixed, grid, mq, mk, mv, s);
    return e != cudaSuccess ? e : cudaGetLastError();
}
