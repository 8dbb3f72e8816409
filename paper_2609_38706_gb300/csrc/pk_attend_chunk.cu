// pk_attend_chunk.cu -- attention of chunks of new tokens over the 4-bit pages of
// their requests, with or without a sliding window (pk_attend_chunk).
//
// out = v_scale sum_j p_j V_j / sum_j p_j over the keys j that a query sees, p_j =
// 2^(s_j - ref), s_j = scale k_scale log2(e) q . K_j; K and V are code * scale, which
// has six significant bits: exact in a half and in a bfloat16.  All products are of
// halves: queries in bfloat16 are scaled by a power of two a row first, which
// leaves them as they are (k_chunk_queries); where one row's values lie too far
// apart for that, the scale is so large that a row's power of two times it may leave
// 32 bits, or the page table is too narrow for them to be worth it (kHalfKeys), the
// call's products with K are of bfloat16s, to which K costs more to unpack (460 |
// 429 us for 4 x 512 tokens behind 16384).  Those sum q . (code * scale) in 32 bits,
// which queries of 2^109 and more can leave.
// ref moves as in pk_attend_prompt.cu: only when a tile's weights of a row sum to
// more than 2^15.
//
// Weights are rounded to halves for the product with V, whatever q's type: half a
// step is 2^-11 of a weight where bfloat16s are off by 2^-8 at the same rate; 32-bit
// weights would take V in 32 bits too and twice the product's time.  The largest one
// is 2^kBase and more (1 behind a far reference), so those that a half does not hold
// (below 2^-14, down to 0 from 2^-25 on) cost N keys at most N 2^-29 (2^-25) of their
// values.  A row's sum takes its weights unrounded, in 32 bits.
//
// Keys are counted without the gap that a window leaves: of a tile of queries the
// granules (16 tokens) of the first tokens and those from the first query's window
// on are one list, cut into tiles of 128 keys.  In its places a query sees last and
// below, down to low, and those before `sinks`.
//
// What bounds it is a tile's chain: scores, weights, product.  A key tile meets two
// tiles of 128 rows, so that unpacking it is paid once for 256 rows, and takes 3500
// cycles at head_dim 128, of which the products are 2048 (tensor pipe 56-62% busy,
// issue slots 52-58%, memory 5%); a warp's scores and weights of one tile are a chain
// of 1650 to 2000 cycles.  Full lengths, bf16, 32 heads over 8: 4 x 512 tokens behind
// 16384 430 us (1.30 PFLOP/s), 2048 behind 60000 1441 us (1.42); head_dim 64, 12 heads
// over 4: 12 x 700 behind 2048 117 us (0.53: the same chain for half of the products).
#include <cuda.h>
#include <cuda_runtime.h>
#include <float.h>

#include <algorithm>
#include <cmath>
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

// A unit that was cut, for k_chunk_join: its rows, and the blocks that had pieces of it.
struct alignas(32) Cut {
    int32_t first, last;     // blocks; first -1: none
    int32_t row0, tokens;    // row of q of its first token; tokens
    int32_t head0, heads;    // query heads
};

struct Args {
    const uint8_t *pool;
    uint64_t page_bytes, n_slots, page_stride, positions;  // positions: that a request can hold
    uint32_t page_grans;  // granules of one head in a page
    const uint16_t *q;
    int64_t q_ts, q_hs;
    uint16_t *half_q;   // [n_q][q_heads][D], queries in bfloat16 as halves; times row_down they are what they were
    float *row_down;    // [n_q][q_heads]
    uint8_t *too_wide;  // by block of k_chunk_queries: a row that halves do not hold
    uint32_t query_blocks;  // 0: the products with K take bfloat16s
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
    uint32_t blocks;  // of k_attend_chunk: the call's work is cut into so many equal shares at most
    int64_t *plan;    // [R + 2]: work of the requests before each one, then all units, by k_chunk_plan; NULL for up to 32 requests
    Cut *cuts;        // [blocks]: by block, the unit that its share's beginning cuts, if no share before it begins there too
    float4 *part_ml;  // [2 blocks][2][128]: (ref, fine, sum) of a piece's rows
    float *part_o;    // [2 blocks][2][128][D]
    int32_t *status;
};

__device__ __forceinline__ bool bad_offsets(int64_t qa, int64_t qb, uint64_t n_q) {
    return qa < 0 || qb < qa || (uint64_t)qb > n_q;
}

// The length of a request, 0 when it is out of range.
__device__ __forceinline__ int32_t good_length(const Args &a, int32_t len) {
    return len < 0 || (uint64_t)len > a.positions ? 0 : len;
}

// The work of a call, on a line: request after request, in one its KV heads (and parts of a group's heads), in one of
// those its units of 2 tile_tokens queries.  A unit weighs as much as the keys that it goes through and kUnitCost.  The
// line is cut into equal shares, one for each block: a block takes the units that its share holds, of the first and
// the last a piece of their keys.  So all blocks are done at about the same time, also where a call is a few rows over
// many keys (4 x 512 tokens behind 16384, 256 units: 604 -> 550 us against units cut in two).  Where that gains less
// than the pieces and their joining cost, a block takes the whole units that begin in its share.  That is judged by the
// mean unit, and is too good for a long request among many short ones, whose units are far above it: 40 tokens behind
// 60000 with 63 requests of 100 alone take 842 us, the two kinds in calls of their own 73 and 55.
// All three in keys.  A unit's start and end: 256 | 512 | 1024 are 65 | 65 | 86 us for 8 x 600 tokens behind 9000, window 1000
// (head_dim 64).  One more piece a block, and the joining: 768 | 1536 are 112 | 128 for 2 x 2000 behind 2000, 150 | 157 for
// 4 x 500 behind 4000, and 123 | 114 for 5 x 400 behind 2500.  Shares of 320 to 1280 keys at least are alike.
constexpr int64_t kUnitCost = 512;
constexpr int64_t kCutCost = 768;
constexpr int64_t kLeastShare = 640;

struct Req {
    int32_t q0, lq, len;
};
// Units of a request for one KV head and part of a group: their keys grow by `step` from `first` on, within 0 .. most.
struct Units {
    int64_t first, most;
    int32_t step, n;

    __device__ __forceinline__ Units(const Args &a, const Req &q) {
        step = 2 * (int32_t)a.tile_tokens;
        n = (int32_t)(((int64_t)q.lq + step - 1) / step);
        first = (int64_t)q.len - q.lq + step;
        most = q.len;
        if (a.window) most = min(most, (int64_t)a.sink_grans * 16 + a.window + step + 15);
    }
    __device__ __forceinline__ int64_t weight(int32_t u) const {
        return kUnitCost + min(max(first + (int64_t)step * u, (int64_t)0), most);
    }
    // Weight of the first u units.
    __device__ __forceinline__ int64_t before(int32_t u) const {
        const int64_t none = first > 0 ? 0 : -first / step + 1;                          // units without keys
        const int64_t rising = first >= most ? 0 : (most - first - 1) / step + 1;        // and those with fewer than most
        const int64_t lo = min(none, (int64_t)u), hi = max(lo, min(rising, (int64_t)u));
        return kUnitCost * u + first * (hi - lo) + step * ((lo + hi - 1) * (hi - lo) / 2) + most * (u - hi);
    }
};
// Work and units of a request.
__device__ __forceinline__ int64_t work_of(const Args &a, const Req &q, int64_t &all_units) {
    const Units units(a, q);
    all_units = (int64_t)units.n * a.chunks * a.kv_heads;
    return units.before(units.n) * a.chunks * a.kv_heads;
}

// The shares of `total`: block b has [start(b), start(b + 1)).
struct Shares {
    int64_t each;
    uint32_t more, n;  // the first `more` have one more
    bool whole;        // no unit is cut

    __device__ __forceinline__ Shares(const Args &a, int64_t total, int64_t units) {
        n = (uint32_t)min((int64_t)a.blocks, max(total / kLeastShare, (int64_t)1));
        each = total / n;
        more = (uint32_t)(total - each * n);
        const int64_t one = units ? total / units : 0;
        whole = max((units + n - 1) / n * one, each + one / 4) <= each + kCutCost;
    }
    __device__ __forceinline__ int64_t start(uint32_t b) const { return each * b + min(b, more); }
    __device__ __forceinline__ uint32_t block_of(int64_t x) const {
        const int64_t wide = (each + 1) * more;
        return x < wide ? (uint32_t)(x / (each + 1)) : more + (uint32_t)((x - wide) / each);
    }
};

// Where on the line a piece begins: unit u of part `part` of request r, `pos` of its weight behind its beginning.
struct Place {
    uint32_t r, part;
    int32_t u;
    int64_t pos;
};
// By a whole warp: x lies in request r, whose work begins at `before`.
__device__ __forceinline__ Place place_of(const Units &units, uint32_t r, int64_t before, int64_t x) {
    Place p;
    p.r = r;
    x -= before;
    const int64_t one = units.before(units.n);
    p.part = (uint32_t)(x / one);
    x -= p.part * one;
    int32_t lo = 0, hi = units.n;  // before(lo) <= x < before(hi)
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 31) / 32, u = lo + (int32_t)(threadIdx.x & 31) * step;
        const uint32_t in = __ballot_sync(0xffffffffu, u < hi && units.before(u) <= x);  // lane 0 is; a prefix of the lanes
        lo += (31 - __clz(in)) * step;
        hi = min(hi, lo + step);
    }
    p.u = lo;
    p.pos = x - units.before(lo);
    return p;
}

// The plan of more than 32 requests; of no work where an offset is out of order or range.
__global__ void __launch_bounds__(kPlanThreads) k_chunk_plan(const Args a) {
    __shared__ int64_t warp_sum[32];
    __shared__ unsigned long long all_units;
    __shared__ uint32_t bad;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    if (tid == 0) bad = 0, all_units = 0;
    const int64_t *q_off = a.q_off;
    const int32_t *kv_len = a.kv_len;
    int64_t *plan = a.plan;
    pk::pdl_wait(q_off, kv_len, plan);
    pk::pdl_launch_dependents();
    __syncthreads();
    int64_t base = 0;
    for (uint64_t r0 = 0; r0 < a.R; r0 += kPlanThreads) {
        const uint64_t r = r0 + tid;
        int64_t n = 0, units = 0;
        if (r < a.R) {
            const int64_t qa = __ldcg(q_off + r), qb = __ldcg(q_off + r + 1);
            const int32_t l = __ldcg(kv_len + r), len = good_length(a, l);
            if (l != len) pk::set_status(a.status, PK_ERR_ARG);
            if (bad_offsets(qa, qb, a.n_q))
                bad = 1;
            else
                n = work_of(a, Req{(int32_t)qa, (int32_t)(qb - qa), len}, units);
        }
#pragma unroll
        for (int d = 16; d; d /= 2) units += __shfl_xor_sync(0xffffffffu, units, d);
        if (lane == 0 && units) atomicAdd(&all_units, (unsigned long long)units);
        int64_t scan = n;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t o = __shfl_up_sync(0xffffffffu, scan, d);
            if (lane >= (uint32_t)d) scan += o;
        }
        if (lane == 31) warp_sum[wid] = scan;
        __syncthreads();
        int64_t before = base, total = 0;
        for (uint32_t w = 0; w < kPlanThreads / 32; ++w) {
            if (w < wid) before += warp_sum[w];
            total += warp_sum[w];
        }
        if (r < a.R) plan[1 + r] = before + scan;
        base += total;
        __syncthreads();
    }
    if (tid == 0) {
        plan[0] = 0;
        plan[a.R + 1] = (int64_t)all_units;
    }
    if (bad) {
        for (uint64_t r = tid; r <= a.R; r += kPlanThreads) plan[r] = 0;
        if (tid == 0) pk::set_status(a.status, PK_ERR_ARG);
    }
}

// One piece of a unit: 2 tiles of tile_tokens query tokens times tile_heads heads of one group, and some of their keys.
struct Item {
    Place at;
    Req q;
    int64_t line, left;   // where the block's share ends; what is left of it behind the piece
    int32_t skip;         // tokens in the gap, a multiple of 16: place x is position x, or x + skip behind the first granules
    int32_t first;        // first key tile of the piece
    int32_t n_tiles[2], n_all;
    uint32_t n_gran;      // granules of the unit's whole list
    bool cut, whole;      // not the whole unit; the block takes whole units

    __device__ __forceinline__ uint32_t head(const Args &a) const { return at.part / a.chunks; }
    __device__ __forceinline__ uint32_t chunk(const Args &a) const { return at.part % a.chunks; }
    __device__ __forceinline__ int32_t tok0(const Args &a) const { return at.u * 2 * (int32_t)a.tile_tokens; }
};

// Queries in bfloat16 as halves, times the power of two that brings a row's largest value to [2^14, 2^15): all values down
// to 2^-31 of it keep their 8 bits.  8 values a lane, of four rows at once, so that four loads are on their way.
constexpr int kQueryThreads = 256, kQueryRows = 4;
constexpr uint32_t kQueryBlocks = 1024;
template <int D>
__global__ void __launch_bounds__(kQueryThreads) k_chunk_queries(const Args a) {
    constexpr uint32_t kLanes = D / 8, kRowsAtOnce = kQueryThreads / kLanes;
    const uint16_t *q = a.q;
    const int64_t *q_off = a.q_off;
    pk::pdl_wait(q, q_off);
    pk::pdl_launch_dependents();
    const uint64_t rows = a.n_q * a.q_heads;
    const int64_t q_first = __ldcg(q_off), q_end = __ldcg(q_off + a.R);  // rows of no request may hold anything
    const uint32_t c = threadIdx.x % kLanes;
    bool wide = false;
    constexpr uint32_t kBlockRows = kRowsAtOnce * kQueryRows;
    for (uint64_t first = (uint64_t)blockIdx.x * kBlockRows; first < rows; first += (uint64_t)gridDim.x * kBlockRows) {
        const uint64_t row0 = first + threadIdx.x / kLanes;
        uint4 all[kQueryRows];
        bool on[kQueryRows];
#pragma unroll
        for (uint32_t k = 0; k < kQueryRows; ++k) {
            const uint64_t row = row0 + k * kRowsAtOnce, token = row / a.q_heads;
            on[k] = row < rows;
            all[k] = on[k] ? __ldcg(reinterpret_cast<const uint4 *>(q + (int64_t)token * a.q_ts +
                                                                   (int64_t)(row - token * a.q_heads) * a.q_hs + c * 8))
                           : make_uint4(0, 0, 0, 0);
            on[k] = on[k] && (int64_t)token >= q_first && (int64_t)token < q_end;
        }
#pragma unroll
        for (uint32_t k = 0; k < kQueryRows; ++k) {
            const uint64_t row = row0 + k * kRowsAtOnce;
            const uint32_t w[4] = {all[k].x, all[k].y, all[k].z, all[k].w};
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = pk::Elem<PK_BF16>::to2(w[i]);
                x[2 * i] = f.x, x[2 * i + 1] = f.y;
            }
            uint32_t bits = 0;  // of the largest magnitude, found on the bits, which finds a NaN too
#pragma unroll
            for (int i = 0; i < 8; ++i) bits = max(bits, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
            for (uint32_t d = 1; d < kLanes; d *= 2) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, d));
            const int e = bits == 0 || bits >= 0x7f800000u ? 14 : max((int)(bits >> 23) - 127, -110);  // 2^e <= the largest
            const float up = __uint_as_float((uint32_t)(14 - e + 127) << 23);
            uint32_t out[4];
            bool odd = bits >= 0x7f800000u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = x[2 * i] * up, hi = x[2 * i + 1] * up;
                const __half2 had = __floats2half2_rn(lo, hi);
                odd |= !(__low2float(had) == lo && __high2float(had) == hi);
                out[i] = *reinterpret_cast<const uint32_t *>(&had);
            }
            if (!on[k]) continue;
            wide |= odd;
            *reinterpret_cast<uint4 *>(a.half_q + row * D + c * 8) = make_uint4(out[0], out[1], out[2], out[3]);
            if (c == 0) a.row_down[row] = __uint_as_float((uint32_t)(e - 14 + 127) << 23);
        }
    }
    const int any = __syncthreads_or(wide);
    if (threadIdx.x == 0) a.too_wide[blockIdx.x] = (uint8_t)(any != 0);
    if (blockIdx.x == 0)  // all are read
        for (uint32_t i = gridDim.x + threadIdx.x; i < kQueryBlocks; i += kQueryThreads) a.too_wide[i] = 0;
}

// Shared memory of a CTA, from a 1024-byte boundary: Q (two tiles), the ring of K and V tiles in 16 bits, the ring of
// granules as they lie in the pages, then Small.  As much as fits: 2 | 3 stages at head_dim 128 are 578 | 435 us for 4 x 512
// tokens behind 16384 (at 64 4 | 8 are even, 285 | 292 for 12 x 1500 behind 2048, 122 | 121 for 12 x 700), 16 | 28 granules
// 219 | 202 us for 1 x 40 behind 120000, and 143 | 121 at head_dim 64 for 12 x 700.
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
constexpr uint32_t kItems = 4;       // items that the loading warp is ahead at most

// What the other warps have to know of an item, from the loading warp.
struct Piece {
    struct Tile {
        int32_t causal, hides[2];  // key tiles from the first on hide some key from some query; those between the others too
        int32_t off, base;         // position of the request's first query; what a position is more than its place in the piece
        int32_t sinks;             // place behind the first tokens
        int32_t tok0, row0, tokens, head0, heads;  // first token of the request, its row; how many; the same of query heads
        int32_t part;              // where the rows of a piece go; -1: the unit is not cut
    } tile[2];
    int32_t n_tiles[2], n_all;     // key tiles; n_all -1: no item, the end
    int32_t first, skip, len;
    uint32_t n_gran;
    int32_t halves;                // the call's queries are halves
};

struct Small {
    uint64_t full[8], empty[8];             // ring stages: tile ready; no longer read
    uint64_t gran_full[32], gran_empty[32]; // the same of granules
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], p_ready[2], o_done[2];
    uint64_t item_full[kItems], item_empty[kItems];
    uint64_t over;                          // every product that was issued is done (a matrix warp that gave up)
    uint32_t tmem, abort;
    uint8_t gran_lost[32];                  // what stands in a granule's place is another request's
    alignas(2) uint8_t flags[kNotes][2];    // by key tile and half of its keys: kMarked, kLost
    uint8_t marked[kNotes][128];            // by key, where kMarked: blocks of V that are NaN (0 stands in the tile)
    int64_t units;                          // up to 32 requests: all their units, the work of those up to each,
    int64_t work_end[32];                   // and what they are
    Req req[32];
    Piece piece[kItems];
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
    const Req q = {(int32_t)qa, (int32_t)(qb - qa), len};
    int64_t units, scan = work_of(a, q, units);
    if (bad) scan = 0;
#pragma unroll
    for (int d = 16; d; d /= 2) units += __shfl_xor_sync(0xffffffffu, units, d);
    if (lane == 0) sm.units = units;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t o = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    sm.work_end[lane] = scan;
    sm.req[lane] = q;
}

__device__ __forceinline__ Shares shares_of(const Args &a, const Small &sm, const int64_t *plan) {
    return plan ? Shares(a, __ldcg(plan + a.R), __ldcg(plan + a.R + 1)) : Shares(a, sm.work_end[31], sm.units);
}

// The request that holds place x of the line.
__device__ __forceinline__ int64_t find_request(const Args &a, const Small &sm, const int64_t *plan, const int64_t *q_off,
                                                const int32_t *kv_len, int64_t x, Item &it) {
    if (a.plan) {
        const uint32_t r = it.at.r = pk::warp_find_request(plan, a.R, x);
        it.q.q0 = (int32_t)__ldcg(q_off + r);
        it.q.lq = (int32_t)__ldcg(q_off + r + 1) - it.q.q0;
        it.q.len = good_length(a, __ldcg(kv_len + r));
        return __ldcg(plan + r);
    }
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t r = it.at.r = __popc(__ballot_sync(0xffffffffu, sm.work_end[lane] <= x)) & 31;
    it.q = sm.req[r];
    return r ? sm.work_end[r - 1] : 0;
}

// The keys of the piece that begins at it.at and has `room` of the block's share.
__device__ __forceinline__ void cut_item(const Args &a, const Units &units, int64_t room, Item &it) {
    const int64_t weight = units.weight(it.at.u), end = it.whole ? weight : min(weight, it.at.pos + room);
    it.left = room - (end - it.at.pos);
    it.cut = it.at.pos > 0 || end < weight;
    const int32_t off = it.q.len - it.q.lq, tok0 = it.tok0(a);  // off: position of the request's first query
    const int64_t low = (int64_t)off + tok0 - a.window + 1;
    const uint32_t low_gran = a.window && low > 0 ? (uint32_t)(low / 16) : 0;
    it.skip = low_gran > a.sink_grans ? (int32_t)(low_gran - a.sink_grans) * 16 : 0;
    int32_t n[2];
    it.n_gran = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int32_t t0 = tok0 + t * (int32_t)a.tile_tokens, t1 = min(t0 + (int32_t)a.tile_tokens, it.q.lq);
        const int32_t last = t1 > t0 ? off + t1 - 1 - it.skip : -1;
        n[t] = last >= 0 ? last / kKeys + 1 : 0;
        if (last >= 0) it.n_gran = (uint32_t)last / 16 + 1;
    }
    const int32_t all = max(n[0], n[1]);
    it.first = it.cut ? (int32_t)(all * it.at.pos / weight) : 0;
    const int32_t to = it.cut ? (int32_t)(all * end / weight) : all;
#pragma unroll
    for (int t = 0; t < 2; ++t) it.n_tiles[t] = max(min(n[t], to) - it.first, 0);
    it.n_all = max(it.n_tiles[0], it.n_tiles[1]);
}

// Lowest position that the query `tok` of a request sees behind the first tokens; off: position of the request's first.
__device__ __forceinline__ int32_t low_of(const Args &a, int32_t off, int32_t tok) {
    return a.window ? (int32_t)max((int64_t)off + tok - a.window + 1, (int64_t)0) : 0;
}

// Registers move to the softmax warps: 256 * 200 + 256 * 56 = 512 * 128, the launch's own.
constexpr int kRegsSoftmax = 200, kRegsOther = 56;
constexpr uint32_t kWarpLoad = 8, kWarpMma = 9, kWarpMake = 10;  // warps 0-7: softmax; from 10: makers

// Where a lane finds its codes and scales of K or V in a granule, and where it puts them as 16-bit values in a tile, in
// the 128-byte swizzle: 32 dimensions of a token, so that a warp takes 8 tokens (D = 128) or 16 at a step.  Eight lanes
// that store at once have two rows' (D = 128) or four rows' pieces: the upper half of the dimensions goes in another
// order, so that they lie in eight different 16-byte columns.
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

    // kRows tokens from row r of a granule on; `tile`: where row r goes.  Weights of 0 must not meet a NaN: of V (kClean)
    // the granule's rows from `valid` on, past the request's end, count as 0, and so do blocks marked NaN.
    template <bool kBf16, bool kClean>
    __device__ __forceinline__ void step(const uint8_t *from, const uint8_t *from_scales, uint8_t *tile, uint32_t r,
                                         int32_t valid) const {
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
                *reinterpret_cast<uint4 *>(tile + dst[i + n]) = make_uint4(h[0], h[1], h[2], h[3]);
            }
        }
    }
    __device__ __forceinline__ void zero(uint8_t *tile) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(tile + dst[i]) = make_uint4(0, 0, 0, 0);
    }
};

// One CTA an SM takes one item after another.  Warp roles: one copies Q tiles and
// granules, six make K and V tiles of granules, one issues the matrix products, and
// two warpgroups of four turn scores into weights, a thread a row, for one of the
// item's two tiles each: while one tile's scores are weighed the other's products
// run.  What is run seldom is loops, not unrolled: code that pushes the rest out of
// the instruction cache costs more than it (4 x 2048 tokens behind 32768, window
// 4096: 592 -> 499 us).  TMEM: scores of the tiles (128 columns each; the weights, two
// to a column, take the place of scores that have been read), then their outputs
// (D columns each).  Every counter of a barrier's use runs on over the items.
template <int D, uint32_t DT>
__global__ void __launch_bounds__(kThreads, 1) k_attend_chunk(const Args a, const __grid_constant__ CUtensorMap map_q,
                                                               const __grid_constant__ CUtensorMap map_half) {
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
        for (uint32_t i = 0; i < kItems; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.item_full[i]), 1);
            pk::mbar_init(pk::smem_addr(&sm.item_empty[i]), 8 + kMakers + 1);  // all that read it
        }
        pk::mbar_init(pk::smem_addr(&sm.over), 1);
        pk::mbar_fence_init();
        sm.abort = 0;
    }
    if (warp == kWarpMma) pk::tmem_alloc(pk::smem_addr(&sm.tmem), 512);
    const int64_t *plan = a.plan;
    const int64_t *q_off = a.q_off;
    const int32_t *kv_len = a.kv_len;
    const uint32_t *pages = a.pages;
    const uint8_t *pool = a.pool;
    const float *row_down = a.row_down;
    const uint8_t *too_wide = a.too_wide;
    pk::pdl_wait(plan, q_off, kv_len, pages, pool, row_down, too_wide);
    pk::pdl_launch_dependents();
    pk::tmem_fence_before();
    __syncthreads();
    pk::tmem_fence_after();
    const uint32_t tmem = pk::uniform(sm.tmem);

    volatile uint32_t *abort = &sm.abort;
    auto give_up = [&]() {
        *abort = 1;
        pk::set_status(a.status, PK_ERR_TIMEOUT);
    };

    // The loading warp's n-th item; back to it.
    auto wait_item = [&](uint32_t n) {
        return pk::mbar_wait_warp(pk::smem_addr(&sm.item_full[n % kItems]), n / kItems & 1);
    };
    auto return_item = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.item_empty[n % kItems]));
    };
    if (warp >= kWarpLoad) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kWarpLoad) {
            uint32_t count = 0, nq[2] = {0, 0};  // granules and Q tiles so far
            bool ok = true, sent = false;        // sent: a copy that `count` does not hold
            const uint32_t slot_shift = 31 - __clz(a.page_grans);
            const bool pow2 = (a.page_grans & (a.page_grans - 1)) == 0;
            if (!plan) {
                plan_here(a, sm, q_off, kv_len);
                __syncwarp();
            }
            bool halves = DT == PK_FP16 || a.query_blocks;
            if (DT == PK_BF16) {  // uniform
                uint32_t wide = 0;
                if (halves) {
#pragma unroll
                    for (uint32_t i = 0; i < kQueryBlocks / 512; ++i) {
                        const uint4 u = __ldcg(reinterpret_cast<const uint4 *>(too_wide) + 32 * i + lane);
                        wide |= u.x | u.y | u.z | u.w;
                    }
                }
                halves &= !__any_sync(0xffffffffu, wide != 0);
            }
            const CUtensorMap *map = DT == PK_BF16 && halves ? &map_half : &map_q;
            Item it;
            bool more;
            {
                const Shares shares = shares_of(a, sm, plan);
                int64_t x = shares.start(min(blockIdx.x, shares.n));
                it.line = shares.start(min(blockIdx.x + 1, shares.n));
                it.whole = shares.whole;
                more = x < it.line;
                while (more) {
                    const int64_t before = find_request(a, sm, plan, q_off, kv_len, x, it);
                    const Units units(a, it.q);
                    it.at = place_of(units, it.at.r, before, x);
                    if (!it.whole || it.at.pos == 0) {
                        cut_item(a, units, it.line - x, it);
                        break;
                    }
                    x += units.weight(it.at.u) - it.at.pos;  // the next unit
                    more = x < it.line;
                }
                if (a.blocks > 1) {  // what k_chunk_join has to know of the unit that this share's beginning cuts
                    Cut cut = {-1, 0, 0, 0, 0, 0};
                    if (more && it.at.pos > 0) {
                        const Units units(a, it.q);
                        const int64_t unit = x - it.at.pos;  // where it begins
                        const uint32_t before = shares.block_of(unit);
                        const int32_t tok0 = it.tok0(a);
                        const uint32_t head0 = it.chunk(a) * a.tile_heads;
                        if (before + 1 == blockIdx.x)
                            cut = Cut{(int32_t)before, (int32_t)shares.block_of(unit + units.weight(it.at.u) - 1), it.q.q0 + tok0,
                                      min(it.q.lq - tok0, units.step), (int32_t)(it.head(a) * a.group + head0),
                                      (int32_t)min(a.group - head0, a.tile_heads)};
                    }
                    if (lane == 0) a.cuts[blockIdx.x] = cut;
                }
            }
            auto take_next = [&]() {  // it begins with a unit
                more = it.left > 0;
                if (!more) return;
                Units units(a, it.q);
                it.at.pos = 0;
                if (++it.at.u == units.n) {
                    it.at.u = 0;
                    if (++it.at.part == a.kv_heads * a.chunks) {
                        find_request(a, sm, plan, q_off, kv_len, it.line - it.left, it);
                        it.at.part = 0;
                        units = Units(a, it.q);
                    }
                }
                cut_item(a, units, it.left, it);
            };
            auto tell = [&](Piece &to) {  // a lane a tile
                const int32_t tok0 = it.tok0(a) + (int32_t)(lane * a.tile_tokens), off = it.q.len - it.q.lq;
                const int32_t base = it.first * kKeys + it.skip;  // from positions to places behind the piece's first one
                const int32_t all_last = off + tok0 - base;       // all queries of the tile see what lies up to here
                const int32_t all_low = low_of(a, off, min(tok0 + (int32_t)a.tile_tokens, it.q.lq) - 1) - base;  // and from here
                const int32_t sinks = (int32_t)a.sinks - it.first * kKeys, gh0 = (int32_t)(it.chunk(a) * a.tile_heads);
                if (lane < 2) {
                    Piece::Tile &t = to.tile[lane];
                    t.causal = ((all_last - (kKeys - 1)) >> 7) + 1;
                    t.hides[0] = sinks >> 7;
                    t.hides[1] = a.window ? (all_low + kKeys - 1) >> 7 : 0;
                    t.off = off;
                    t.base = base;
                    t.sinks = sinks;
                    t.tok0 = tok0;
                    t.row0 = it.q.q0 + tok0;
                    t.tokens = min((int32_t)a.tile_tokens, it.q.lq - tok0);
                    t.head0 = (int32_t)(it.head(a) * a.group) + gh0;
                    t.heads = (int32_t)a.group - gh0;
                    // a block has one piece at most that begins inside a unit, and one that only ends there
                    t.part = it.cut ? (int32_t)(((2 * blockIdx.x + (it.at.pos == 0)) * 2 + lane) * kRows) : -1;
                    to.n_tiles[lane] = it.n_tiles[lane];
                }
                if (lane == 0) {
                    to.n_all = it.n_all;
                    to.first = it.first;
                    to.skip = it.skip;
                    to.len = it.q.len;
                    to.n_gran = it.n_gran;
                    to.halves = halves;
                }
            };
            pk::fence_proxy_async();  // pages written by an earlier kernel are read by the async proxy
            for (uint32_t items = 0; ok && !__any_sync(0xffffffffu, *abort != 0); ++items) {
                const uint32_t at = items % kItems;
                ok = items < kItems || pk::mbar_wait_warp(pk::smem_addr(&sm.item_empty[at]), (items / kItems + 1) & 1);
                if (!ok) break;
                if (more)
                    tell(sm.piece[at]);
                else if (lane == 0)
                    sm.piece[at].n_all = -1;
                __syncwarp();
                if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.item_full[at]));
                if (!more) break;
                const uint32_t v0 = 8 * (uint32_t)it.first, v1 = min(8 * (uint32_t)(it.first + it.n_all), it.n_gran);
                const uint32_t *row = pages + (uint64_t)it.at.r * a.page_stride;
                const uint32_t head = it.head(a);
                const int32_t skip = it.skip, n_all = it.n_all;
                const bool two[2] = {it.n_tiles[0] > 0, it.n_tiles[1] > 0};
                const int32_t q_head = (int32_t)(head * a.group + it.chunk(a) * a.tile_heads), q_row = it.q.q0 + it.tok0(a);
                uint64_t where = 0;  // lane l: address of the granule `base` + l of the list
                bool lost = false;   // slot 0's bytes stand in for a slot out of range
                auto find_granules = [&](uint32_t base) {
                    const uint32_t v = base + lane;
                    lost = false;
                    if (v < v1) {
                        const uint32_t gr = v >= a.sink_grans ? v + (uint32_t)skip / 16 : v;
                        const uint32_t page = pow2 ? gr >> slot_shift : gr / a.page_grans;
                        uint64_t slot = __ldcg(row + page);
                        if (slot >= a.n_slots) {
                            pk::set_status(a.status, PK_ERR_ARG);
                            slot = 0;
                            lost = true;
                        }
                        where = reinterpret_cast<uint64_t>(pool) + slot * a.page_bytes +
                                ((uint64_t)head * a.page_grans + (gr - page * a.page_grans)) * L::kGran;
                    }
                };
                for (uint32_t v = v0; ok && n_all > 0 && v < v1; v += 8) {
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
                            if (!ok || !two[t]) continue;
                            ok = nq[t] == 0 || pk::mbar_wait(pk::smem_addr(&sm.q_empty[t]), (nq[t] - 1) & 1);
                            if (!ok) break;
                            const uint32_t bar = pk::smem_addr(&sm.q_full[t]);
                            pk::mbar_expect(bar, q_bytes);
#pragma unroll
                            for (int b = 0; b < D / 64; ++b)
                                pk::tile_load3(smem + t * L::kTile + b * 16384, map, b * 64, q_head,
                                               q_row + t * (int)a.tile_tokens, bar);
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
        } else if (warp >= kWarpMake) {
            // Makers of K and V tiles: a tile's steps go round the six; the last two, which have fewer, look for what the
            // softmax warps have to know of it.
            using U = Unpack<D>;
            constexpr uint32_t kPerGran = 16 / U::kRows, kSteps = 8 * kPerGran;
            const uint32_t mine = warp - kWarpMake;
            const U lanes(lane);
            uint32_t n = 0, count = 0, tiles = 0;  // stages, granules, key tiles so far
            bool ok = true;
            auto wait_empty = [&](uint32_t n) {
                return n < L::kStages ||
                       pk::mbar_wait_warp(pk::smem_addr(&sm.empty[n % L::kStages]), (n / L::kStages + 1) & 1);
            };
            for (uint32_t items = 0; ok && !__any_sync(0xffffffffu, *abort != 0); ++items) {
                ok = wait_item(items);
                if (!ok) break;
                const volatile Piece &it = sm.piece[items % kItems];
                const int32_t n_all = it.n_all, skip = it.skip, len = it.len, halves = it.halves;
                const uint32_t first = (uint32_t)it.first, n_gran = it.n_gran;
                return_item(items);
                if (n_all < 0) break;
                for (int32_t j = 0; j < n_all; ++j) {
                    const uint32_t v0 = 8 * (first + j), have = min(n_gran - v0, 8u);
                    // Every warp waits for all of the tile's granules, a lane each, and gives all of them back: a place's
                    // next user may be another warp, and one that has not seen a use of it, or sees it too late, would
                    // take one state of the barrier for another.
                    const uint32_t c = count + lane;
                    ok = lane >= have || pk::mbar_wait(pk::smem_addr(&sm.gran_full[c % L::kGrans]), (c / L::kGrans) & 1);
                    ok = __all_sync(0xffffffffu, ok) && wait_empty(n);
                    if (!ok) break;
                    auto place = [&](uint32_t g) { return smem_c + L::kGranRing + (count + g) % L::kGrans * L::kGran; };
                    // tokens of a granule before the request's end
                    auto valid = [&](uint32_t g) { return len - (int32_t)(16 * (v0 + g)) - (v0 + g >= a.sink_grans ? skip : 0); };
                    uint8_t *tile = smem_c + L::kRing + n % L::kStages * L::kTile;
                    auto k_steps = [&](auto bf16) {
#pragma unroll 1
                        for (uint32_t s = mine; s < have * kPerGran; s += kMakers) {
                            const uint32_t g = s / kPerGran, r = s % kPerGran * U::kRows;
                            lanes.template step<decltype(bf16)::value, false>(place(g) + G::kK, place(g) + G::kKs,
                                                                              tile + s * U::kRows * 128, r, 16);
                        }
                    };
                    // a loop each, the seldom one out of the way (438 -> 431 us for 4 x 512 tokens behind 16384)
                    if (__builtin_expect(DT == PK_FP16 || halves, 1))
                        k_steps(std::false_type{});
                    else
                        k_steps(std::true_type{});
                    pk::fence_proxy_async_smem();
                    if (mine >= kMakers - 2) {  // blocks of V marked NaN, two tokens a lane
                        const uint32_t half = mine - (kMakers - 2);
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
                    }
                    __syncwarp();
                    if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[n % L::kStages]));
                    ++n;
                    ok = wait_empty(n);
                    if (!ok) break;
                    tile = smem_c + L::kRing + n % L::kStages * L::kTile;
                    uint32_t s = mine;
#pragma unroll 1
                    for (; s < have * kPerGran; s += kMakers) {
                        const uint32_t g = s / kPerGran, r = s % kPerGran * U::kRows;
                        lanes.template step<false, true>(place(g) + G::kV, place(g) + G::kVs, tile + s * U::kRows * 128, r,
                                                         valid(g));
                    }
#pragma unroll 1
                    for (; s < kSteps; s += kMakers)  // behind the last granule: weights of 0 must not meet what lies there
                        lanes.zero(tile + s * U::kRows * 128);
                    pk::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane < have) pk::mbar_arrive(pk::smem_addr(&sm.gran_empty[c % L::kGrans]));
                    if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[n % L::kStages]));
                    ++n;
                    count += have;
                    ++tiles;
                }
            }
            if (!ok && lane == 0) give_up();
            __syncwarp();
        } else if (warp == kWarpMma) {
            uint32_t qk_kind = 0;
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
                ok = wait_item(items);
                if (!ok) break;
                const volatile Piece &it = sm.piece[items % kItems];
                const int32_t n0 = (int32_t)pk::uniform(it.n_tiles[0]), n1 = (int32_t)pk::uniform(it.n_tiles[1]);
                const int32_t n_all = (int32_t)pk::uniform(it.n_all);
                qk_kind = pk::mma_idesc(DT == PK_BF16 && !pk::uniform(it.halves), 128, 128, false) |
                          (a.scale2 < 0.0f ? 1u << 13 : 0u);  // a negative scale negates Q
                return_item(items);
                if (n_all < 0) break;
                if (n_all == 0) continue;
                ok = wait_full(ring, use);
                if (!ok) break;
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
        uint32_t ni = 0, tiles = 0;  // key tiles weighed so far; key tiles of the CTA's items before the present one
        bool ok = true;
        for (uint32_t items = 0; ok && !__any_sync(0xffffffffu, *abort != 0); ++items) {
            ok = wait_item(items);
            if (!ok) break;
            const volatile Piece &it = sm.piece[items % kItems];
            const volatile Piece::Tile *mine = &it.tile[t];
            if (it.n_all < 0) break;
            const int32_t n_tiles = it.n_tiles[t];
            float scale2 = fabsf(a.scale2);
            const bool on = row_tok < mine->tokens && row_tok < (int32_t)a.tile_tokens && row_head < mine->heads;
            if (DT == PK_BF16 && on && it.halves)
                scale2 *= __ldcg(row_down + (int64_t)(mine->row0 + row_tok) * a.q_heads + mine->head0 + row_head);
            // a scale of 0 would make a masked -infinity NaN; the smallest normal one gives the same weights
            scale2 = fmaxf(scale2, FLT_MIN);
            const uint64_t scale22 = pk::pack2(scale2, scale2);
            // a weight is 2^(score - ref + fine), and fine is 0 but for a reference of kFar and more
            float ref = -FLT_MAX, fine = 0.0f, sum = 0.0f;
            uint32_t marked = 0;  // blocks of 16 dimensions in which the row saw a NaN of V
            bool lost = false;    // it saw a token whose slot is out of range
            bool far_off = false; // a row of the warp has a far reference
#pragma unroll 1
            for (int32_t j = 0; ok && j < n_tiles; ++j, ++ni) {
                // the row sees the tile's keys up to `see` that are not below `from`, or are below `first`
                const bool edge = j >= mine->causal || (j >= mine->hides[0] && j < mine->hides[1]);
                int32_t see = kKeys - 1, from = 0, first = 0;
                if (edge) {
                    const int32_t tok = mine->tok0 + row_tok, x0 = j * kKeys;
                    if (on) {
                        see = mine->off + tok - mine->base - x0;
                        from = low_of(a, mine->off, tok) - mine->base - x0;
                        first = mine->sinks - x0;
                    }
                }
                auto hidden = [&](int32_t i) { return i > see || (i < from && i >= first); };
                uint32_t x[3][32];
                ok = pk::mbar_wait_warp(pk::smem_addr(&sm.s_full[t]), ni & 1);
                if (!ok) break;
                pk::tmem_fence_after();
                pk::tmem_load32(ts, x[0]);
                // -infinity for the keys of a chunk of 32 that the row does not see; most chunks of an edge tile are seen
                // whole by all of a warp's rows.
                auto mask = [&](int c, uint32_t(&y)[32]) {
                    auto up_to = [&](int32_t n) { n -= 32 * c; return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };
                    const uint32_t seen = up_to(see + 1) & (~up_to(from) | up_to(first));
                    if (__all_sync(0xffffffffu, seen == ~0u)) return;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(seen & 1u << i)) y[i] = 0xff800000u;
                };
                // The largest score of the first n chunks.
                auto largest = [&](int n) {
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                    for (int c = 0; c < n; ++c) {
                        pk::tmem_load32(ts + 32 * c, x[0]);
                        pk::tmem_wait_load(x[0]);
                        if (edge) mask(c, x[0]);
#pragma unroll
                        for (int i = 0; i < 32; ++i) m4[i & 3] = fmaxf(m4[i & 3], __uint_as_float(x[0][i]));
                    }
                    pk::tmem_load32(ts, x[0]);  // for what comes next
                    return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                };
                // The weights by the reference so far, and their sum.
                uint32_t p[2][32];
                uint64_t ref2, sum2[4];
                auto weigh_chunk = [&](const uint32_t(&y)[32], uint32_t *to) {  // 32 keys
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float2 z = pk::unpack2(
                            pk::fma2(pk::pack2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), scale22, ref2));
                        z.x = pk::ex2(z.x);
                        z.y = pk::ex2(z.y);
                        sum2[i / 2 & 3] = pk::add2(sum2[i / 2 & 3], pk::pack2(z.x, z.y));
                        to[i / 2] = pk::Elem<PK_FP16>::from2(z.x, z.y);
                    }
                };
                auto weigh = [&]() {  // loads run ahead: 1 and 2 behind 0's use, 3 behind 1's (0's is on its way)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c != 2) pk::tmem_wait_load(x[c % 3]);
                        if (c == 0) {
                            pk::tmem_load32(ts + 32, x[1]);
                            pk::tmem_load32(ts + 64, x[2]);
                        } else if (c == 1) {
                            pk::tmem_wait_load(x[2]);
                            pk::tmem_load32(ts + 96, x[0]);
                        }
                        weigh_chunk(x[c % 3], p[c / 2] + c % 2 * 16);
                    }
                };
                // The same of an edge tile, in a loop of 64 keys: less code (against four chunks in a row, head_dim 64, bf16,
                // 12 x 1500 tokens behind 2048: 292 -> 260 us; for all tiles it is more for its moves: 4 x 512 behind 16384,
                // head_dim 128: 435 -> 446).
                auto weigh_edge = [&]() {
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        pk::tmem_wait_load(x[0]);
                        pk::tmem_load32(ts + 64 * h + 32, x[1]);
                        mask(2 * h, x[0]);
                        weigh_chunk(x[0], p[1]);
                        pk::tmem_wait_load(x[1]);
                        if (h == 0) pk::tmem_load32(ts + 64, x[0]);
                        mask(2 * h + 1, x[1]);
                        weigh_chunk(x[1], p[1] + 16);
                        if (h == 0) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) p[0][i] = p[1][i];
                        }
                    }
                };
                // The same where a row of the warp has a far reference, which few calls have: by 16 scores, with `fine`.
                auto weigh_far = [&]() {
                    float s = 0.0f;
                    uint32_t(&y)[16] = reinterpret_cast<uint32_t(&)[16]>(x[0]);
                    uint32_t w[64];  // by way of memory: a loop, as its code would take the place of what is run often
#pragma unroll 1
                    for (int c = 0; c < 8; ++c) {
                        pk::tmem_load16(ts + 16 * c, y);
                        pk::tmem_wait_load(y);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float f[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const bool off = edge && hidden(16 * c + i + h);
                                f[h] = off ? 0.0f : pk::ex2(fmaf(__uint_as_float(y[i + h]), scale2, -ref) + fine);
                                s += f[h];
                            }
                            w[8 * c + i / 2] = pk::Elem<PK_FP16>::from2(f[0], f[1]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 64; ++i) p[i / 32][i % 32] = w[i];
                    return s;
                };
                auto weigh_any = [&]() {
                    if (far_off) return weigh_far();
                    ref2 = pk::pack2(-ref, -ref);
                    sum2[0] = sum2[1] = sum2[2] = sum2[3] = 0;
                    edge ? weigh_edge() : weigh();
                    const float2 s0 = pk::unpack2(pk::add2(sum2[0], sum2[2])), s1 = pk::unpack2(pk::add2(sum2[1], sum2[3]));
                    return (s0.x + s1.x) + (s0.y + s1.y);
                };
                // Moves the reference of the rows that `over` names to the score `top`; their sum so far is rescaled.
                // Returns the factor.  That score's weight is then a power of two, which rounding leaves as it is: a row
                // with one key, or one that outweighs the others, gets its value of V and no more error.
                auto move_ref = [&](bool over, float top) {
                    const float m = top * scale2;
                    const bool moves = over && m > -INFINITY, far = moves && fabsf(m) >= kFar;
                    const float next = !moves ? ref : far ? m : m - kBase;
                    // far: what m's rounding lost comes off again, so the largest weight is 2^kBase or, where kBase
                    // is lost beside that, 1; not a number where m overflowed
                    const float next_fine = !moves ? fine : far ? kBase - fmaf(top, scale2, -m) : 0.0f;
                    const float f = pk::ex2((ref - next) + (next_fine - fine));
                    ref = next;
                    fine = next_fine;
                    far_off = __any_sync(0xffffffffu, fine != 0.0f);
                    sum *= f;
                    return f;
                };
                // from 32 keys alone: mostly no other is 2^11 times as heavy as the heaviest of them
                if (j == 0) move_ref(on, largest(1));
                // One pass over the scores takes the weights by the reference so far, with no look at the scores
                // first: a weight that has outgrown it shows in the sum, and only then the reference is moved and
                // the pass done again.  A row that saw no key yet (its window begins further on) has the lowest
                // reference, by which any weight is infinite.  Once does: behind a move no weight is above
                // 2^(kBase + 2).  Rows without a query, whose scores may be anything, have no say.
                float part_sum = weigh_any();
                if (__any_sync(0xffffffffu, on && part_sum > kTop)) {
                    const float f = move_ref(on && part_sum > kTop, largest(4));
                    if (j > 0) {  // the output so far too
                        ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (ni - 1) & 1);
                        if (!ok) break;
                        pk::tmem_fence_after();
#pragma unroll 1
                        for (int d = 0; d < D / 32; ++d) {
                            pk::tmem_load32(to + 32 * d, x[1]);
                            pk::tmem_wait_load(x[1]);
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[1][i] = __float_as_uint(__uint_as_float(x[1][i]) * f);
                            pk::tmem_store32(to + 32 * d, x[1]);
                        }
                        pk::tmem_load32(ts, x[0]);
                    }
                    part_sum = weigh_any();
                }
                sum += part_sum;
                pk::tmem_store32(ts, p[0]);  // over the scores, which every pass is done with
                pk::tmem_store32(ts + 32, p[1]);
                // The tile's notes, before it is given up: behind it the makers can go round while the other tile's products,
                // for which nobody waits for this warp, take their tiles.
                const uint32_t note = (tiles + j) % kNotes;
                const uint32_t flags = *reinterpret_cast<const volatile uint16_t *>(sm.flags[note]);
                pk::tmem_wait_store();
                pk::tmem_fence_before();
                if (flags) {
                    lost |= (flags & 0x0101u * kLost) != 0;
#pragma unroll 1
                    for (int32_t i = 0; i < kKeys; ++i)
                        if ((flags >> (i / 64 * 8) & kMarked) && !hidden(i)) marked |= sm.marked[note][i];
                }
                __syncwarp();
                if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.p_ready[t]));
            }
            tiles += (uint32_t)it.n_all;
            if (ok && n_tiles > 0) ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (ni - 1) & 1);
            if (!ok) break;
            if (lost) sum = __int_as_float(0x7fffffff);
            const bool cut = mine->part >= 0;
            const uint64_t part = cut ? (uint64_t)(mine->part + row) : 0;
            const int64_t q_row = (int64_t)mine->row0 + row_tok;
            const uint32_t qh = (uint32_t)(mine->head0 + row_head);
            const float inv = cut ? 1.0f : sum == 0.0f ? 0.0f : a.v_scale / sum;
            if (on && cut) a.part_ml[part] = make_float4(ref, fine, sum, 0.0f);
            if (on && !cut && a.lse)
                a.lse[q_row * a.q_heads + qh] = sum == 0.0f ? -INFINITY : (ref - fine + log2f(sum)) * 0.69314718055994531f;
            uint16_t *dst = a.out + q_row * a.o_ts + (int64_t)qh * a.o_hs;
            pk::tmem_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t z[32];
                if (n_tiles > 0) {  // else O was never written
                    __syncwarp();
                    pk::tmem_load32(to + 32 * c, z);
                    pk::tmem_wait_load(z);
                }
                if (!on) continue;
                const bool none = n_tiles == 0 || inv == 0.0f;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float f = none ? 0.0f : __uint_as_float(z[i]) * inv;
                    z[i] = __float_as_uint(marked >> (2 * c + i / 16) & 1 ? __int_as_float(0x7fffffff) : f);
                }
                uint32_t w[8];
                if (cut) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = z[8 * h + i];
                        pk::store32(reinterpret_cast<uint16_t *>(a.part_o + part * D + 32 * c + 8 * h), true, w);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < 16; i += 2)
                            w[i / 2] = pk::Elem<DT>::from2(__uint_as_float(z[16 * h + i]), __uint_as_float(z[16 * h + i + 1]));
                        pk::store32(dst + 32 * c + 16 * h, a.wide_out, w);
                    }
                }
            }
            return_item(items);
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

// Joins the pieces of the units that were cut, in the order of their keys: kJoinBlocks for a unit, a warp two rows.  Most
// units have two pieces, whose rows are on their way before their weights are known (1 x 40 tokens behind 120000, ten
// pieces a unit: 208 -> 201 us; 4 x 500 behind 4000: 153 -> 150).  It costs 17 to 20 us there, for 40 MB from the L2: rows
// of a warp 1 | 2 | 4 are 153 | 150 | 155 us, and more warps an SM by fewer registers nothing.
constexpr int kJoinThreads = 256, kJoinRows = 2, kJoinBlocks = 2 * kRows / (kJoinThreads / 32 * kJoinRows);
template <int D, uint32_t DT>
__global__ void __launch_bounds__(kJoinThreads) k_chunk_join(const Args a) {
    using V = std::conditional_t<D == 128, float4, float2>;  // of a row, a lane's part
    constexpr int kPer = D / 32;
    const Cut *cuts = a.cuts;
    const float4 *ml = a.part_ml;
    const float *po = a.part_o;
    pk::pdl_wait(cuts, ml, po);
    pk::pdl_launch_dependents();
    cuts += blockIdx.x / kJoinBlocks + 1;
    const int4 where = __ldcg(reinterpret_cast<const int4 *>(cuts));
    const int2 heads = __ldcg(reinterpret_cast<const int2 *>(cuts) + 2);
    if (where.x < 0) return;  // uniform
    const uint32_t lane = threadIdx.x & 31, b0 = (uint32_t)where.x, n = (uint32_t)where.y - b0 + 1;
    const uint32_t row0 = (blockIdx.x % kJoinBlocks * (kJoinThreads / 32) + threadIdx.x / 32) * kJoinRows;
    auto token_of = [&](int k) { return (row0 + k) / kRows * a.tile_tokens + (row0 + k) % kRows / a.tile_heads; };
    auto is_row = [&](int k) {
        const uint32_t in = (row0 + k) % kRows;
        return in / a.tile_heads < a.tile_tokens && token_of(k) < (uint32_t)where.w && in % a.tile_heads < (uint32_t)heads.y;
    };
    if (!is_row(0) && !is_row(1)) return;  // uniform per warp
    static_assert(kJoinRows == 2, "rows of a warp");
    auto part_of = [&](uint32_t i, int k) { return (uint64_t)(2 * (b0 + i) + (i == 0)) * 2 * kRows + row0 + k; };
    V u[2][kJoinRows];
    auto load = [&](uint32_t i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k)
                if (i + j < n) u[j][k] = __ldcg(reinterpret_cast<const V *>(po + part_of(i + j, k) * D) + lane);
    };
    // (ref, fine, sum) of piece i0 + lane.  The exponent of a piece's weights is ref - fine, which 32 bits may not hold:
    // differences are taken part by part.
    float4 y[kJoinRows];
    auto look = [&](uint32_t i0) {
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k)
            y[k] = i0 + lane < n ? __ldcg(ml + part_of(i0 + lane, k)) : make_float4(-FLT_MAX, 0.0f, 0.0f, 0.0f);
    };
    auto more = [](float2 x, float2 y) { return (x.x - y.x) - (x.y - y.y); };
    look(0);
    load(0);
    float2 top[kJoinRows];
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k) top[k] = make_float2(y[k].x, y[k].y);
    for (uint32_t i0 = 32; i0 < n; i0 += 32) {
        look(i0);
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k)
            if (more(make_float2(y[k].x, y[k].y), top[k]) > 0.0f) top[k] = make_float2(y[k].x, y[k].y);
    }
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k) {
#pragma unroll
        for (int d = 16; d; d /= 2) {
            const float2 z = make_float2(__shfl_xor_sync(0xffffffffu, top[k].x, d), __shfl_xor_sync(0xffffffffu, top[k].y, d));
            if (more(z, top[k]) > 0.0f) top[k] = z;
        }
        top[k] = make_float2(__shfl_sync(0xffffffffu, top[k].x, 0), __shfl_sync(0xffffffffu, top[k].y, 0));
    }
    float sum[kJoinRows] = {}, o[kJoinRows][kPer] = {};
    for (uint32_t i0 = 0; i0 < n; i0 += 32) {
        if (n > 32) look(i0);
        float f[kJoinRows];
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k)
            f[k] = y[k].z == 0.0f ? 0.0f : pk::ex2(more(make_float2(y[k].x, y[k].y), top[k]));
        for (uint32_t i = i0; i < min(n, i0 + 32); i += 2) {
            if (i) load(i);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (i + j >= n) break;
#pragma unroll
                for (int k = 0; k < kJoinRows; ++k) {
                    const float w = __shfl_sync(0xffffffffu, f[k], (i + j) & 31);
                    sum[k] += w * __shfl_sync(0xffffffffu, y[k].z, (i + j) & 31);
                    const float(&v)[kPer] = reinterpret_cast<const float(&)[kPer]>(u[j][k]);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) o[k][e] += w * v[e];
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k) {
        if (!is_row(k)) continue;
        const int64_t token = (int64_t)where.z + token_of(k);
        const uint32_t qh = (uint32_t)heads.x + (row0 + k) % kRows % a.tile_heads;
        const float inv = sum[k] == 0.0f ? 0.0f : a.v_scale / sum[k];
        uint32_t w[kPer / 2];
#pragma unroll
        for (int e = 0; e < kPer; e += 2) w[e / 2] = pk::Elem<DT>::from2(o[k][e] * inv, o[k][e + 1] * inv);
        uint32_t *dst = reinterpret_cast<uint32_t *>(a.out + token * a.o_ts + (int64_t)qh * a.o_hs + lane * kPer);
        if constexpr (kPer == 4)
            *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
        else
            *dst = w[0];
        if (lane == 0 && a.lse)
            a.lse[token * a.q_heads + qh] =
                sum[k] == 0.0f ? -INFINITY : (top[k].x - top[k].y + log2f(sum[k])) * 0.69314718055994531f;
    }
}

// What the host knows of a call are bounds; the kernels see the lengths.
struct Plan {
    uint64_t units, blocks;  // at most
    uint64_t plan_bytes, cut_bytes, ml_bytes, o_bytes, wide_bytes, down_bytes, half_bytes;  // wide_bytes 0: no halves
};

constexpr uint64_t kSms = 152;
// Keys that a call's units go through (half of them at head_dim 64) from which on halves of its queries pay for their
// making, as bfloat16s | halves: 400 tokens of 2 requests behind 4000 (0.5 M keys) 77 | 80 us, 1 x 40 behind 60000 (1.0 M)
// 118 | 112, 4 x 500 behind 4000 (1.2 M) 147 | 148, head_dim 64 12 x 700 behind 2048 (1.2 M) 130 | 132.
constexpr uint64_t kWorthHalves = 3ull << 18;
// And keys that a unit can have at least (twice as many at head_dim 64): what is made is a row's, what it saves a key's.
// 16 x 1024 tokens alone 215 | 262 us, 8 x 4096 behind 8192 with a window of 2048 985 | 1037, 4 x 2048 behind 32768 with
// one of 4096 487 | 478, 1 x 8192 alone 489 | 476; head_dim 64 12 x 1500 behind 2048 253 | 260, 6 x 3000 behind 4000
// 541 | 538.  The host knows the page table's width and the window, not the lengths: in a table for 4096 tokens and more
// 16 x 1024 alone make halves too and take 263 us.
constexpr uint64_t kHalfKeys = 4096;
Plan plan_of(const pk_kv_cache &kv, uint32_t dtype, uint32_t R, uint64_t n_q, uint32_t q_heads, uint64_t page_stride,
             uint32_t window, uint32_t sinks) {
    Plan p;
    p.units = pk_attend_prompt_items(n_q, R, q_heads, kv.kv_heads);
    uint64_t keys = page_stride * kv.page_tokens;
    if (window) keys = std::min<uint64_t>(keys, (uint64_t)sinks + 15 + window + 2 * kRows + 15);
    const uint64_t share = (uint64_t)kUnitCost + keys;  // of a unit
    p.blocks = p.units > kSms * kLeastShare ? kSms : std::min(kSms, std::max<uint64_t>(p.units * share / kLeastShare, 1));
    p.plan_bytes = R > 32 ? (((uint64_t)R + 2) * 8 + 31) & ~31ull : 0;
    p.cut_bytes = p.blocks * sizeof(Cut);
    p.ml_bytes = p.blocks > 1 ? 2 * p.blocks * 2 * kRows * 16 : 0;
    p.o_bytes = p.blocks > 1 ? 2 * p.blocks * 2 * kRows * kv.head_dim * 4 : 0;
    const bool halves = dtype == PK_BF16 && keys >= kHalfKeys * 128 / kv.head_dim &&
                        p.units >= kWorthHalves * 128 / kv.head_dim / keys;
    const uint64_t rows = halves ? n_q * q_heads : 0;
    p.wide_bytes = rows ? kQueryBlocks : 0;
    p.down_bytes = (rows * 4 + 31) & ~31ull;
    p.half_bytes = rows * kv.head_dim * 2;
    return p;
}

template <int D, uint32_t DT>
cudaError_t launch(const Args &a, const CUtensorMap &mq, const CUtensorMap &mh, cudaStream_t s) {
    constexpr size_t smem = Layout<D>::kBytes + sizeof(Small);
    static_assert(smem <= 227 * 1024, "shared memory of a block");
    static std::atomic<uint64_t> seen{0};
    cudaError_t e = pk_allow_smem(k_attend_chunk<D, DT>, smem, seen);
    if (e == cudaSuccess && a.query_blocks) e = pk_launch(k_chunk_queries<D>, a.query_blocks, kQueryThreads, s, a);
    if (e == cudaSuccess) e = pk_launch_smem(k_attend_chunk<D, DT>, a.blocks, kThreads, smem, s, a, mq, mh);
    if (e == cudaSuccess && a.blocks > 1) e = pk_launch(k_chunk_join<D, DT>, (a.blocks - 1) * (unsigned)kJoinBlocks, kJoinThreads, s, a);
    return e;
}

}  // namespace

uint64_t pk_attend_chunk_scratch_bytes_impl(const pk_kv_cache &kv, uint32_t dtype, uint32_t R, uint64_t n_q, uint32_t q_heads,
                                            uint64_t page_stride, uint32_t window, uint32_t sinks) {
    const Plan p = plan_of(kv, dtype, R, n_q, q_heads, page_stride, window, sinks);
    if (p.units > 0x7fffffffull) return UINT64_MAX;
    return p.plan_bytes + p.cut_bytes + p.ml_bytes + p.o_bytes + p.wide_bytes + p.down_bytes + p.half_bytes;
}

cudaError_t pk_launch_attend_chunk(const pk_kv_cache &kv, uint32_t dtype, const pk_heads &q, const pk_heads &out,
                                   float *lse, uint64_t n_q, const int64_t *q_off, uint32_t R, uint32_t q_heads,
                                   float scale, uint32_t window, uint32_t sinks, const int32_t *kv_len,
                                   const uint32_t *pages, uint64_t page_stride, void *scratch, int32_t *status,
                                   cudaStream_t s) {
    const Plan p = plan_of(kv, dtype, R, n_q, q_heads, page_stride, window, sinks);
    Args a;
    a.q = static_cast<const uint16_t *>(q.p);
    a.q_ts = q.tok_stride;
    a.q_hs = q.head_stride;
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
    a.blocks = (uint32_t)p.blocks;
    uint8_t *at = static_cast<uint8_t *>(scratch);
    a.plan = R > 32 ? reinterpret_cast<int64_t *>(at) : nullptr;
    a.cuts = reinterpret_cast<Cut *>(at + p.plan_bytes);
    a.part_ml = reinterpret_cast<float4 *>(at + p.plan_bytes + p.cut_bytes);
    a.part_o = reinterpret_cast<float *>(at + p.plan_bytes + p.cut_bytes + p.ml_bytes);
    at += p.plan_bytes + p.cut_bytes + p.ml_bytes + p.o_bytes;
    a.too_wide = at;
    a.row_down = reinterpret_cast<float *>(at + p.wide_bytes);
    a.half_q = reinterpret_cast<uint16_t *>(at + p.wide_bytes + p.down_bytes);
    const uint64_t query_rows = kQueryThreads / (kv.head_dim / 8) * kQueryRows;  // of a block at once
    // A row's factor of scores is scale2 * 2^(e - 14), e up to 127: where that can leave 32 bits, which would make NaN of a
    // score of 0, the call takes bfloat16 products, which need no factor.
    const bool halves = p.wide_bytes && std::fabs(a.scale2) < 0x1p15f;
    a.query_blocks = halves ? (uint32_t)std::min<uint64_t>((n_q * q_heads + query_rows - 1) / query_rows, kQueryBlocks) : 0;
    a.status = status;
    CUtensorMap mq, mh{};
    cudaError_t e = map_of(&mq, q, n_q, q_heads, kv.head_dim, dtype, a.tile_tokens, a.tile_heads);
    if (e == cudaSuccess && a.query_blocks)
        e = map_of(&mh, pk_heads{a.half_q, (int64_t)q_heads * kv.head_dim, kv.head_dim}, n_q, q_heads, kv.head_dim, PK_FP16,
                   a.tile_tokens, a.tile_heads);
    if (e == cudaSuccess && a.plan) e = pk_launch(k_chunk_plan, 1, kPlanThreads, s, a);
    if (e != cudaSuccess) return e;
    if (kv.head_dim == 128)
        e = dtype == PK_BF16 ? launch<128, PK_BF16>(a, mq, mh, s) : launch<128, PK_FP16>(a, mq, mh, s);
    else
        e = dtype == PK_BF16 ? launch<64, PK_BF16>(a, mq, mh, s) : launch<64, PK_FP16>(a, mq, mh, s);
    return e != cudaSuccess ? e : cudaGetLastError();
}
