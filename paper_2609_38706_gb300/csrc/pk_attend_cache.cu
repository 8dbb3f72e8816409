// pk_attend_cache.cu -- attention of one or a few tokens a request over the
// 4-bit pages of its slots (pk_attend_cache).
//
// With s_j = scale * k_scale * (q . K_j), p_j = 2^(s_j log2 e - ref) and one
// pass over the tokens, o = v_scale * sum p_j V_j / sum p_j: the format's
// tensor scales leave the loop, and what is left of a value, code * scale, has
// six significant bits, so it is exact in a half; so are the values of q, scaled
// by a power of two (small ones beside a large one in two halves), and every
// product of the QK step is exact in 32 bits.  `ref` is a running score near the maximum; it moves
// only when a p would pass 2^15 (a warp vote), so rescaling is rare, and to the
// maximum itself, so that the heaviest p is a power of two, which its rounding to
// a half leaves as it is: a row with one key gets that key's value exactly.
//
// The work is reading the pages once: 1.125 D bytes a token and KV head.  A
// granule (16 tokens of one head) is one contiguous bulk copy; every warp has
// its own ring of copies in flight and needs no other warp until the end.
// Tokens are the rows of the products (S^T = K Q^T, O^T = V^T P^T), queries
// their 8 columns, so a group of up to 8 query heads fills the matrix
// instruction and dequantised values feed it straight from registers:
// mma.sync suits these 8-column products, whose operands never lie in shared
// memory as 16-bit values (tcgen05 would need them there).
//
// 16 requests of up to 131072 tokens (8 KV heads, groups of 8, D = 128): 328 us
// for both launches, 25 of it the join, 5.4 TB/s of pages; the attention takes 76%
// of the memory's cycles and 65% of the issue slots (dequantising is 58% of the
// ALU's).  128 requests of up to 2048: 62.5 us, 5 of it the page weights: 1024 CTAs
// of unequal lengths for 608 places.  Short caches: two launches, 8 us.  With a
// window the granules that no query sees are left out of the count, so the work is
// that of a short cache: 128 requests of 8192 tokens, window 1024, 49 us, 9 of it the
// page weights; 2 or 3 splits of such windows are 59 or 65 us, 2 or 3 warps a CTA 53 to
// 55 (with one split 52, but 135 for 77 at 64 x 8192, window 4096).
#include <cuda_runtime.h>
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"
#include "pk_tma.cuh"

namespace {

// Four warps a CTA and four CTAs an SM: against eight and two, the start and the
// end of one CTA are covered by three others (16 x 131072 cached tokens: 343 ->
// 324 us; 128 x 2048: 69 -> 65 us).
constexpr int kWarps = 4;
constexpr uint32_t kSlots = 152 * 16 / kWarps;  // CTAs that the GPU holds
constexpr int kThreads = 32 * kWarps;
constexpr uint32_t kRanked = 256, kRankedGrans = 64;  // requests that are ranked by length: most of them, least size
constexpr int kFinishWarps = 8, kFinishThreads = 32 * kFinishWarps;
constexpr float kTop = 15.0f;   // p stays below 2^kTop (half: 2^16)
// Scores (times log2 e) from here on are further apart than a half's exponents, and so is a product from its rounding:
// a reference that far is met with rounded products, by which the heaviest score is kBase or nothing above it.
constexpr float kFar = 16777216.0f;
constexpr float kBase = 8.0f;   // the largest p when ref moves: 2^kBase, so 22 bits of range lie below it

struct Args {
    const uint8_t *pool;
    uint64_t page_bytes, n_slots;
    uint32_t page_tokens, page_grans, kv_heads, group, n_q, rows, row_tiles, R;
    uint32_t splits, split_grans;  // granules of one split
    bool by_length;                // the longest requests' blocks come first
    float scale2, v_scale;         // scale2 = scale * k_scale * log2 e
    uint32_t window, sinks, sink_grans;  // window 0: none; granules that hold the first `sinks` tokens
    uint32_t weigh_blocks, sink_blocks;  // of k_cache_finish: that weigh a request's pages; of them for the first tokens' pages
    const uint16_t *q;
    int64_t q_ts, q_hs;
    uint16_t *out;
    int64_t o_ts, o_hs;
    float *lse;
    const int32_t *kv_len;
    const uint32_t *pages;
    uint64_t page_stride;
    float *part_o;    // [R][kv_heads][row_tiles][splits][tile rows][D], splits > 1
    float2 *part_ml;  // the same without D: (ref, sum)
    float2 *gran_ml;  // [R][kv_heads][row_tiles][granules][gran_rows]: (sum, ref) of a granule
    uint32_t gran_stride, gran_rows;
    float *page_weight;
    int32_t *status;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// D(16x8) += A(16x16) B(16x8), halves into 32 bits.
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Stands for the sum of a row that a slot out of range has a part in: its request's outputs are NaN, and its pages'
// weights stay.  Sums are not negative.
constexpr float kLost = -1.0f;
// What a row's weighted values are multiplied with, and ln of its sum by the reference m, of a sum l.
__device__ __forceinline__ float inverse(const Args &a, float l, bool gone) {
    return gone ? __int_as_float(0x7fffffff) : l == 0.0f ? 0.0f : a.v_scale / l;
}
__device__ __forceinline__ float log_sum(float m, float l, bool gone) {
    return gone ? __int_as_float(0x7fffffff) : l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// The length of request r, 0 when it is out of range.
__device__ __forceinline__ int32_t length_of(const int32_t *kv_len, uint64_t r, uint64_t most) {
    const int32_t len = __ldcg(kv_len + r);
    return len < 0 || (uint64_t)len > most ? 0 : len;
}

// With a window a request's granules that some query sees are counted without the gap between those of the first tokens
// and those of the window: granule v of them is granule v, or v + skip from sink_grans on.
__device__ __forceinline__ uint32_t gap_of(const Args &a, int32_t len) {
    const int64_t low = (int64_t)len - a.n_q - a.window + 1;  // first position that the first query's window holds
    const uint32_t first = low > 0 ? (uint32_t)(low / 16) : 0;
    return first > a.sink_grans ? first - a.sink_grans : 0;
}

// How a variant is cut: columns (8 query rows each), granules that a warp takes
// at once, stages of its ring, CTAs an SM.  Two granules share the waiting, the
// look for a new reference and the loop around them (338 instructions a granule
// one by one); with 16 rows of 128 dimensions the accumulators leave room for one.
template <int D, int NT>
struct Shape {
    static constexpr int kGrans = D == 128 && NT == 2 ? 1 : 2;
    static constexpr int kStages = kGrans == 2 ? 3 : 4;
    static constexpr uint32_t kStage = kGrans * pk::Granule<D>::kBytes;
    static constexpr uint32_t kRing = kStages * kStage;  // a warp's; holds its [8 NT][D] outputs at the end
    static_assert(kRing >= 8 * NT * D * 4, "outputs fit the ring");
};

// The n-th request by length, longest first, in 64 steps of the longest; within a step by number.  By every warp for
// itself: a search over the steps that counts by votes.
__device__ __forceinline__ uint32_t nth_longest(const int32_t *kv_len, uint32_t R, uint32_t n) {
    constexpr int kPer = kRanked / 32;
    const uint32_t lane = threadIdx.x & 31;
    int32_t x[kPer], most = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        x[k] = 32 * k + lane < R ? max(__ldcg(kv_len + 32 * k + lane), 0) : -1;
        most = max(most, x[k]);
    }
    const int shift = max(26 - __clz(__reduce_max_sync(0xffffffffu, most)), 0);
#pragma unroll
    for (int k = 0; k < kPer; ++k) x[k] >>= shift;  // 0..63; -1 stays
    int32_t step = 0;  // the largest that more than n requests reach
    uint32_t above = 0;
#pragma unroll
    for (int bit = 32; bit; bit /= 2) {
        uint32_t reach = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (32 * k < R) reach += __popc(__ballot_sync(0xffffffffu, x[k] >= step + bit));
        if (reach > n)
            step += bit;
        else
            above = reach;  // fewer as `step + bit` falls: in the end those above `step`
    }
    uint32_t m = n - above, r = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const bool in = x[k] == step;
        const uint32_t all = __ballot_sync(0xffffffffu, in), before = __popc(all & ((1u << lane) - 1));
        const uint32_t hit = __ballot_sync(0xffffffffu, in && before == m);
        if (hit) r = 32 * k + __ffs(hit) - 1;
        m -= __popc(all);  // past the request's own: wraps, and nothing is hit
    }
    return r;
}

// One CTA: one request, KV head, tile of 8 NT query rows and split of the
// tokens.  Warp w takes the split's steps w, w + kWarps, ... of kGrans granules.
// Lane = 4 g + c.
template <int D, int NT, uint32_t DT, bool kWeigh, bool kWindow>
__global__ void __launch_bounds__(kThreads, 16 / kWarps) k_attend_cache(const Args a) {
    using G = pk::Granule<D>;
    using S = Shape<D, NT>;
    constexpr int TG = S::kGrans;
    constexpr int kSteps = D / 16;  // k16 steps of QK, m16 tiles of PV
    constexpr int kRows = 8 * NT;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kWarps][S::kStages];
    __shared__ float s_ref[kWarps][kRows], s_sum[kWarps][kRows];

    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    uint32_t id = blockIdx.x;
    const uint32_t split = id % a.splits;
    id /= a.splits;
    const uint32_t tile = id % a.row_tiles;
    id /= a.row_tiles;
    const uint32_t head = id % a.kv_heads;
    uint32_t r = id / a.kv_heads;

    uint8_t *ring = smem + warp * S::kRing;
    const uint32_t ring_s = pk::smem_addr(ring), bar_s = pk::smem_addr(&bars[warp][0]);
    if (lane == 0) {
        for (int i = 0; i < S::kStages; ++i) pk::mbar_init(bar_s + 8 * i, 1);
        pk::mbar_fence_init();
    }
    __syncwarp();

    const uint8_t *pool = a.pool;
    const uint16_t *qp = a.q;
    const int32_t *kv_len = a.kv_len;
    const uint32_t *pages = a.pages;
    pk::pdl_wait(pool, qp, kv_len, pages);
    pk::fence_proxy_async();  // pages written by an earlier kernel are read by the async proxy
    if (a.by_length) r = nth_longest(kv_len, a.R, r);

    const uint64_t most = a.page_stride * a.page_tokens;
    const int32_t len = length_of(kv_len, r, most);
    if (len != __ldcg(kv_len + r) && tid == 0) pk::set_status(a.status, PK_ERR_ARG);
    const uint32_t skip = kWindow ? gap_of(a, len) : 0;
    auto gran_of = [&](uint32_t v) { return kWindow && v >= a.sink_grans ? v + skip : v; };
    const uint32_t n_gran = ((uint32_t)len + 15) / 16 - skip;
    const uint32_t g0 = split * a.split_grans, g1 = min(g0 + a.split_grans, n_gran);
    if (a.splits > 1 && g0 >= n_gran) return;  // no partial result: the combination counts the splits itself
    const uint32_t steps = g0 < g1 ? (g1 - g0 + TG - 1) / TG : 0;
    const uint32_t mine = warp < steps ? (steps - warp + kWarps - 1) / kWarps : 0;

    pages += (uint64_t)r * a.page_stride;
    const uint32_t slot_shift = 31 - __clz(a.page_grans);
    const bool pow2 = (a.page_grans & (a.page_grans - 1)) == 0;
    // lane l holds where the warp's granule ahead * TG + l lies.  A slot out of range is reported; slot 0's bytes stand
    // in for what it should hold, and `lost` keeps all that is made of them from the outputs.
    uint32_t ahead = 0;
    bool lost = false;
    uint64_t where = 0;
    auto find_granules = [&](uint32_t k) {
        ahead = k;
        const uint32_t at = g0 + (warp + (k + lane / TG) * kWarps) * TG + lane % TG;
        if (at < g1) {
            const uint32_t gr = gran_of(at);
            const uint32_t page = pow2 ? gr >> slot_shift : gr / a.page_grans;
            uint64_t slot = __ldcg(pages + page);
            if (slot >= a.n_slots) {
                pk::set_status(a.status, PK_ERR_ARG);
                slot = 0;
                lost = true;
            }
            where = reinterpret_cast<uint64_t>(pool) + slot * a.page_bytes +
                    ((uint64_t)head * a.page_grans + (gr - page * a.page_grans)) * G::kBytes;
        }
    };
    auto issue = [&](uint32_t k) {
        if (k >= mine) return;  // uniform
        if (k >= ahead + 32 / TG) find_granules(k);
        const uint64_t src = __shfl_sync(0xffffffffu, where, (k - ahead) * TG + lane % TG);
        const uint32_t st = k % S::kStages;
        const uint32_t n = min(g1 - (g0 + (warp + k * kWarps) * TG), (uint32_t)TG);
        if (lane == 0) pk::mbar_expect(bar_s + 8 * st, n * G::kBytes);
        __syncwarp();
        if (lane < n)  // a lane a granule
            pk::bulk_load(ring_s + st * S::kStage + lane * G::kBytes, reinterpret_cast<const void *>(src), G::kBytes,
                          bar_s + 8 * st);
    };
    find_granules(0);
#pragma unroll
    for (int k = 0; k < S::kStages; ++k) issue(k);

    // Q: column n = g of tile nt, dimensions c D/4 + 4 s + {0..3} at step s; scaled by a power of two that
    // brings the row's largest value to [2^7, 2^8).  A half then holds all 8 or 11 bits of what is above 2^-14 or
    // so; where a row has nonzero values below (`wide`), their rest goes through a second product (see step()).
    uint32_t qf[NT][kSteps][2];
    bool wide = false;
    uint32_t up_bits[NT];  // that power of two
    float mul[NT][2];   // for columns 2c, 2c + 1
    int32_t last[NT][2], low[NT][2];  // a column sees the positions low .. last, and those below a.sinks up to last
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const uint32_t row = tile * kRows + nt * 8 + g;
        const bool on = row < a.rows;
        const uint32_t i = on ? row / a.group : 0;
        const uint16_t *src = qp + ((int64_t)r * a.n_q + i) * a.q_ts +
                              (int64_t)(head * a.group + (on ? row - i * a.group : 0)) * a.q_hs + c * (D / 4);
        float x[D / 4], top = 0.0f;
#pragma unroll
        for (int s = 0; s < kSteps; s += 2) {
            const uint4 u = on ? __ldcg(reinterpret_cast<const uint4 *>(src + 4 * s)) : make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = pk::Elem<DT>::to2(w[j]);
                x[4 * s + 2 * j] = f.x;
                x[4 * s + 2 * j + 1] = f.y;
                top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        int e = (int)(__float_as_uint(top) >> 23) - 127;  // 2^e <= top
        e = top == 0.0f || e == 128 ? 7 : max(e, -110);
        const float up = __uint_as_float((uint32_t)(7 - e + 127) << 23);
        const float down = __uint_as_float((uint32_t)(e - 7 + 127) << 23);
        up_bits[nt] = __float_as_uint(up);
        uint32_t least = 0xffffffffu;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            qf[nt][s][0] = half2_of(x[4 * s] * up, x[4 * s + 1] * up);
            qf[nt][s][1] = half2_of(x[4 * s + 2] * up, x[4 * s + 3] * up);
            least = __vminu2(least, __vminu2(qf[nt][s][0] & 0x7c007c00u, qf[nt][s][1] & 0x7c007c00u));
        }
        // only a half without an exponent can have lost something
        if ((least & 0xffffu) == 0 || least >> 16 == 0) {
#pragma unroll
            for (int i = 0; i < D / 4; ++i) wide |= __half2float(__float2half_rn(x[i] * up)) != x[i] * up;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // past 32 bits it would make NaN of a score of 0; scores that are made smaller, all beyond 2^50, keep their order
            mul[nt][j] = fminf(fmaxf(a.scale2 * __shfl_sync(0xffffffffu, down, 4 * (2 * c + j)), -FLT_MAX), FLT_MAX);
            const uint32_t cr = tile * kRows + nt * 8 + 2 * c + j;
            last[nt][j] = len - (int32_t)a.n_q + (int32_t)(cr < a.rows ? cr / a.group : a.n_q - 1);
            low[nt][j] = kWindow ? (int32_t)max((int64_t)last[nt][j] - a.window + 1, (int64_t)0) : 0;
        }
    }

    wide = __any_sync(0xffffffffu, wide);

    float o[NT][kSteps][4], ref[NT][2], sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.0f;
        ref[nt][0] = ref[nt][1] = -FLT_MAX;
        sum[nt][0] = sum[nt][1] = 0.0f;
    }
    // positions all_low .. all_see are seen by every query
    const int32_t all_see = len - (int32_t)a.n_q;
    const int32_t all_low = kWindow ? (int32_t)max((int64_t)len - a.window, (int64_t)0) : 0;
    // where this lane's granule sums of the first step go: lanes of g = 0..3 write, column 2c + (g & 1) of granule
    // g >> 1 (of tile nt: + 8 nt)
    float2 *gran_at = nullptr;
    if (kWeigh)
        gran_at = a.gran_ml + ((((uint64_t)(r * a.kv_heads + head) * a.row_tiles + tile) * a.gran_stride + g0 +
                                warp * TG + (g >> 1)) * a.gran_rows + 2 * c + (g & 1));
    bool gave_up = false, far = false;  // far: a reference of the warp's is

    // One step: TG granules in stage `st`.  kEdge: some query does not see some token of them.  kWide: what the halves
    // of Q lost of a small value beside a large one, times 2^38 a half again, has its own product with K (exact down
    // to 2^-62 of the row's largest value); such rows are rare, so it is read from Q again at each step.
    auto step = [&](uint32_t k, uint32_t st, auto edge, auto with_rest) {
        constexpr bool kEdge = decltype(edge)::value, kWide = decltype(with_rest)::value;
        const uint8_t *gr = ring + st * S::kStage;
        const uint32_t v0 = g0 + (warp + k * kWarps) * TG;
        int32_t pos0[TG];  // first positions of the granules
#pragma unroll
        for (int h = 0; h < TG; ++h) pos0[h] = (int32_t)(gran_of(v0 + h) * 16);

        // S^T = K Q^T: rows g and g + 8 of a granule's 16 are tokens
        float s[TG][NT][4];
#pragma unroll
        for (int h = 0; h < TG; ++h) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[h][nt][0] = s[h][nt][1] = s[h][nt][2] = s[h][nt][3] = 0.0f;
            uint32_t w[2][D / 32];   // this lane's code words of tokens g and g + 8
            uint32_t sc[2][D / 64];  // their scales, twice in a half2
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint8_t *row = gr + h * G::kBytes + G::kK + (g + 8 * t) * G::kRow + c * (D / 8);
                const uint8_t *ss = gr + h * G::kBytes + G::kKs + (g + 8 * t) * G::kScales + c * (D / 64);
                uint32_t z;
                if (D == 128) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(row);
                    w[t][0] = u.x, w[t][1] = u.y, w[t][D == 128 ? 2 : 0] = u.z, w[t][D == 128 ? 3 : 1] = u.w;
                    z = pk::e4m3_to_half2(*reinterpret_cast<const uint16_t *>(ss));
                    sc[t][D == 128 ? 1 : 0] = __byte_perm(z, z, 0x3232);
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(row);
                    w[t][0] = u.x, w[t][1] = u.y;
                    z = pk::e4m3_to_half2(*ss);
                }
                sc[t][0] = __byte_perm(z, z, 0x1010);
            }
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t h0[4], h1[4];
                pk::e2m1x8_to_half2(w[0][j], h0);
                pk::e2m1x8_to_half2(w[1][j], h1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h0[i] = hmul2(h0[i], sc[0][j / 2]);
                    h1[i] = hmul2(h1[i], sc[1][j / 2]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma(s[h][nt], h0[0], h1[0], h0[1], h1[1], qf[nt][2 * j][0], qf[nt][2 * j][1]);
                    mma(s[h][nt], h0[2], h1[2], h0[3], h1[3], qf[nt][2 * j + 1][0], qf[nt][2 * j + 1][1]);
                }
            }
            if (kWide) {
#pragma unroll 1
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t row = tile * kRows + nt * 8 + g, i = row / a.group;
                    const uint16_t *src = qp + ((int64_t)r * a.n_q + i) * a.q_ts +
                                          (int64_t)(head * a.group + (row - i * a.group)) * a.q_hs + c * (D / 4);
                    const float up = __uint_as_float(NT == 2 && nt ? up_bits[NT - 1] : up_bits[0]);
                    float rest[4] = {};
#pragma unroll 1
                    for (int j = 0; j < D / 32; ++j) {
                        const uint4 u = row < a.rows ? __ldcg(reinterpret_cast<const uint4 *>(src + 8 * j))
                                                     : make_uint4(0, 0, 0, 0);
                        const uint32_t y[4] = {u.x, u.y, u.z, u.w};
                        uint32_t b[4], kf[2][4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 f = pk::Elem<DT>::to2(y[i]);
                            const float lo = f.x * up, hi = f.y * up;
                            const __half2 had = __floats2half2_rn(lo, hi);
                            b[i] = half2_of((lo - __low2float(had)) * 0x1p38f, (hi - __high2float(had)) * 0x1p38f);
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const uint8_t *tok = gr + h * G::kBytes + G::kK + (g + 8 * t) * G::kRow + c * (D / 8) + 4 * j;
                            const uint8_t *ss = gr + h * G::kBytes + G::kKs + (g + 8 * t) * G::kScales + c * (D / 64) + j / 2;
                            const uint32_t z = pk::e4m3_to_half2(*ss);
                            pk::e2m1x8_to_half2(*reinterpret_cast<const uint32_t *>(tok), kf[t]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) kf[t][i] = hmul2(kf[t][i], __byte_perm(z, z, 0x1010));
                        }
                        mma(rest, kf[0][0], kf[1][0], kf[0][1], kf[1][1], b[0], b[1]);
                        mma(rest, kf[0][2], kf[1][2], kf[0][3], kf[1][3], b[2], b[3]);
                    }
#pragma unroll
                    for (int n2 = 0; n2 < NT; ++n2)
                        if (n2 == nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[h][n2][e] = fmaf(rest[e], 0x1p-38f, s[h][n2][e]);
                }
            }
        }

        // p = 2^x, x = s * mul - ref: [0] (token g, column 2c) [1] (g, 2c + 1) [2] (g + 8, 2c) [3] (g + 8, 2c + 1)
        float x[TG][NT][4];
        auto exponents_by = [&](auto rounded) {
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < TG; ++h)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float &y = x[h][nt][e];
                        if (decltype(rounded)::value)
                            y = __fmul_rn(s[h][nt][e], mul[nt][e & 1]) - ref[nt][e & 1];
                        else
                            y = fmaf(s[h][nt][e], mul[nt][e & 1], -ref[nt][e & 1]);
                        const int32_t pos = pos0[h] + (int32_t)(g + 8 * (e >> 1));
                        if (kEdge && pos > last[nt][e & 1]) y = -INFINITY;
                        if (kEdge && kWindow && pos < low[nt][e & 1] && pos >= (int32_t)a.sinks) y = -INFINITY;
                        top = fmaxf(top, y);
                    }
            return top > kTop;
        };
        auto exponents = [&]() { return far ? exponents_by(std::true_type{}) : exponents_by(std::false_type{}); };
        if (__any_sync(0xffffffffu, exponents())) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // the column's largest score, from the scores that it sees
                    float m = -INFINITY;
#pragma unroll
                    for (int h = 0; h < TG; ++h)
#pragma unroll
                        for (int e = j; e < 4; e += 2)
                            m = fmaxf(m, x[h][nt][e] == -INFINITY ? -INFINITY : __fmul_rn(s[h][nt][e], mul[nt][j]));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                    if (m - ref[nt][j] > kTop) {
                        const float to = m - kBase;
                        const float f = ex2(ref[nt][j] - to);
                        ref[nt][j] = to;
                        sum[nt][j] *= f;
#pragma unroll
                        for (int i = 0; i < kSteps; ++i) o[nt][i][j] *= f, o[nt][i][j + 2] *= f;
                    }
                    far |= fabsf(ref[nt][j]) >= kFar && ref[nt][j] != -FLT_MAX;
                }
            far = __any_sync(0xffffffffu, far);
            exponents();
        }
        uint32_t pf[TG][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float t[TG][2];
#pragma unroll
            for (int h = 0; h < TG; ++h) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = ex2(x[h][nt][e]);
                t[h][0] = p[0] + p[2];
                t[h][1] = p[1] + p[3];
                sum[nt][0] += t[h][0];
                sum[nt][1] += t[h][1];
                // rounded to halves for the product with V; the sums keep 32 bits
                pf[h][nt][0] = transpose8x8(half2_of(p[0], p[1]));
                pf[h][nt][1] = transpose8x8(half2_of(p[2], p[3]));
            }
            if (kWeigh) {
                // over a granule's 16 tokens: lanes keep column 2c + (g & 1) of granule (g >> 1) & 1
                const bool odd = g & 1, second = g & 2;
                float u[TG];
#pragma unroll
                for (int h = 0; h < TG; ++h)
                    u[h] = (odd ? t[h][1] : t[h][0]) + __shfl_xor_sync(0xffffffffu, odd ? t[h][0] : t[h][1], 4);
                float v = TG == 2 ? (second ? u[TG - 1] : u[0]) + __shfl_xor_sync(0xffffffffu, second ? u[0] : u[TG - 1], 8)
                                  : u[0] + __shfl_xor_sync(0xffffffffu, u[0], 8);
                v += __shfl_xor_sync(0xffffffffu, v, 16);
                const uint32_t col = nt * 8 + 2 * c + (g & 1);
                if (g < 2 * TG && tile * kRows + col < a.rows && (!kEdge || (TG == 2 && (g & 2) ? pos0[TG - 1] : pos0[0]) < len))
                    gran_at[(uint64_t)k * (kWarps * TG) * a.gran_rows + nt * 8] =
                        make_float2(v, odd ? ref[nt][1] : ref[nt][0]);
            }
        }

        // O^T += V^T P^T: this lane's tokens 2c, 2c + 1, 2c + 8, 2c + 9, dimensions g D/8 ..
#pragma unroll
        for (int h = 0; h < TG; ++h) {
            uint32_t v[4][D / 64], vs[2], b[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t tok = 2 * c + (t & 1) + 8 * (t >> 1);
                const uint8_t *row = gr + h * G::kBytes + G::kV + tok * G::kRow + g * (D / 16);
                if (D == 128) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(row);
                    v[t][0] = u.x, v[t][D == 128 ? 1 : 0] = u.y;
                } else {
                    v[t][0] = *reinterpret_cast<const uint32_t *>(row);
                }
                b[t] = gr[h * G::kBytes + G::kVs + tok * G::kScales + (D == 128 ? g : g / 2)];
            }
            if (kEdge) {
                // A token that some query does not see has p = 0 there, which must not meet a NaN; a token that
                // none sees is stale bytes.  Blocks marked NaN count as 0, and the queries that do see them get
                // their NaN by hand.
                uint32_t bad = 0;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t tok = 2 * c + (t & 1) + 8 * (t >> 1);
                    if (pos0[h] + (int32_t)tok >= len) {
                        b[t] = 0;
                    } else if ((b[t] & 0x7f) == 0x7f) {
                        b[t] = 0;
                        bad |= 1u << tok;
                    }
                }
                if (__any_sync(0xffffffffu, bad != 0)) {
                    bad |= __shfl_xor_sync(0xffffffffu, bad, 1);
                    bad |= __shfl_xor_sync(0xffffffffu, bad, 2);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const auto up_to = [](int32_t n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1; };
                            uint32_t m = up_to(last[nt][j] - pos0[h] + 1);  // tokens here that it sees
                            if (kWindow) m &= ~up_to(low[nt][j] - pos0[h]) | up_to((int32_t)a.sinks - pos0[h]);
                            if (bad & m) {
#pragma unroll
                                for (int i = 0; i < kSteps; ++i)
                                    o[nt][i][j] = o[nt][i][j + 2] = __int_as_float(0x7fffffff);
                            }
                        }
                }
            }
            vs[0] = pk::e4m3_to_half2(b[0] | b[1] << 8);
            vs[1] = pk::e4m3_to_half2(b[2] | b[3] << 8);
            if (h == TG - 1) {
                __syncwarp();  // every lane has read the stage
                issue(k + S::kStages);
            }
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                // byte i of a word: dimensions 2i (low half) and 2i + 1; pair up the tokens of one dimension
                uint32_t lo[2][4], hi[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t y = v[2 * t][j], z = v[2 * t + 1][j];
                    pk::e2m1x8_to_half2((y & 0x0f0f0f0fu) | ((z << 4) & 0xf0f0f0f0u), lo[t]);
                    pk::e2m1x8_to_half2(((y >> 4) & 0x0f0f0f0fu) | (z & 0xf0f0f0f0u), hi[t]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = hmul2(lo[0][i], vs[0]), a1 = hmul2(hi[0][i], vs[0]);
                    const uint32_t a2 = hmul2(lo[1][i], vs[1]), a3 = hmul2(hi[1][i], vs[1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(o[nt][4 * j + i], a0, a1, a2, a3, pf[h][nt][0], pf[h][nt][1]);
                }
            }
        }
    };

    auto walk = [&](auto with_rest) {
        uint32_t st = 0, turn = 0;
#pragma unroll 1
        for (uint32_t k = 0; k < mine; ++k) {
            if (!pk::mbar_wait_warp(bar_s + 8 * st, turn & 1)) {
                gave_up = true;
                for (uint32_t i = k + 1; i < min(k + S::kStages, mine); ++i)  // no copy of its own stays in flight
                    pk::mbar_wait(bar_s + 8 * (i % S::kStages), (i / S::kStages) & 1);
                break;
            }
            const uint32_t v0 = g0 + (warp + k * kWarps) * TG;
            const int32_t begin = (int32_t)(gran_of(v0) * 16), end = (int32_t)(gran_of(v0 + TG - 1) * 16 + 16);
            const bool hides = kWindow && begin < all_low && end > (int32_t)a.sinks;
            if (decltype(with_rest)::value || end - 1 > all_see || hides)
                step(k, st, std::true_type{}, with_rest);
            else
                step(k, st, std::false_type{}, with_rest);
            if (++st == S::kStages) st = 0, ++turn;
        }
    };
    if (wide)
        walk(std::true_type{});
    else
        walk(std::false_type{});
    if (gave_up && lane == 0) pk::set_status(a.status, PK_ERR_TIMEOUT);
    pk::pdl_launch_dependents();

    lost = __any_sync(0xffffffffu, lost) || gave_up;

    // join the warps: O of each goes to its own ring, [row][D]
    float *ow = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x = sum[nt][j];
#pragma unroll
            for (int d = 4; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
            const uint32_t q = nt * 8 + 2 * c + j;
            if (g == 0) s_ref[warp][q] = ref[nt][j], s_sum[warp][q] = lost ? kLost : x;
#pragma unroll
            for (int i = 0; i < kSteps; ++i)  // tile i, rows g and g + 8: dimensions g D/8 + 2i, + 1
                *reinterpret_cast<float2 *>(ow + q * D + g * (D / 8) + 2 * i) =
                    make_float2(o[nt][i][j], o[nt][i][j + 2]);
        }
    __syncthreads();
    const uint64_t part = (((uint64_t)(r * a.kv_heads + head) * a.row_tiles + tile) * a.splits + split) * kRows;
#pragma unroll 1
    for (uint32_t x = tid * 2; x < kRows * D; x += 2 * kThreads) {
        const uint32_t q = x / D, d = x % D, row = tile * kRows + q;
        if (row >= a.rows) break;  // rows only grow from here
        float m = -FLT_MAX, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
        bool gone = false;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_ref[w][q]), gone |= s_sum[w][q] == kLost;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = ex2(s_ref[w][q] - m);
            const float2 y = *reinterpret_cast<const float2 *>(
                reinterpret_cast<const float *>(smem + w * S::kRing) + q * D + d);
            l += f * s_sum[w][q];
            o0 += f * y.x;
            o1 += f * y.y;
        }
        if (d == 0 && a.part_ml) a.part_ml[part + q] = make_float2(m, gone ? kLost : l);
        if (a.splits > 1) {
            *reinterpret_cast<float2 *>(a.part_o + (part + q) * D + d) = make_float2(o0, o1);
        } else {
            const uint32_t i = row / a.group, qh = head * a.group + row - i * a.group;
            const float inv = inverse(a, l, gone);
            const int64_t t = (int64_t)r * a.n_q + i;
            *reinterpret_cast<uint32_t *>(a.out + t * a.o_ts + (int64_t)qh * a.o_hs + d) =
                pk::Elem<DT>::from2(o0 * inv, o1 * inv);
            if (d == 0 && a.lse) a.lse[t * (a.kv_heads * a.group) + qh] = log_sum(m, l, gone);
        }
    }
}

// Splits of one request that hold tokens that a query sees.
template <bool kWindow>
__device__ __forceinline__ uint32_t live_splits(const Args &a, int32_t len) {
    const uint32_t n_gran = ((uint32_t)len + 15) / 16 - (kWindow ? gap_of(a, len) : 0);
    return (n_gran + a.split_grans - 1) / a.split_grans;
}

constexpr uint32_t kStatRows = 512;

// Pages that a warp of k_cache_finish weighs: short ones by several, four granules at once (pages of 16 tokens, 128 x
// 2048 tokens, by one | four: 63.5 | 60.4 us).
__host__ __device__ constexpr uint32_t pages_a_warp(uint32_t page_grans) { return page_grans < 4 ? 4 / page_grans : 1; }

// The rest of a call, by block: the first ones join the splits of the query
// rows (a warp a row), the others add to the pages' weights
//     page_weight[r][j] += sum over heads, rows and granules of the page of
//                          (granule's sum of p) * 2^(its ref - ref) / sum,
// a warp a page, lanes over (head, row), in an order that depends on the sizes
// alone.  Both need a row's final reference and sum over the splits; the
// weighing blocks find them again, which costs less than waiting for a launch.
template <int D, uint32_t DT, bool kWindow>
__global__ void __launch_bounds__(kFinishThreads) k_cache_finish(const Args a, uint32_t tile_rows, uint32_t join_blocks) {
    __shared__ float2 stat[kStatRows];  // (ref, 1 / sum) of (head, row)
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t *kv_len = a.kv_len;
    const float *part_o = a.part_o;
    const float2 *part_ml = a.part_ml, *gran_ml = a.gran_ml;
    float *weight = a.page_weight;
    pk::pdl_wait(kv_len, part_o, part_ml, gran_ml, weight);
    pk::pdl_launch_dependents();
    const uint64_t most = a.page_stride * a.page_tokens;
    if (blockIdx.x < join_blocks) {
        const uint64_t id = (uint64_t)blockIdx.x * kFinishWarps + warp;
        if (id >= (uint64_t)a.R * a.kv_heads * a.rows) return;
        const uint64_t rh = id / a.rows;
        const uint32_t row = (uint32_t)(id % a.rows);
        const uint32_t r = (uint32_t)(rh / a.kv_heads), head = (uint32_t)(rh % a.kv_heads);
        const uint32_t n = live_splits<kWindow>(a, length_of(kv_len, r, most));
        const uint64_t first = (rh * a.row_tiles + row / tile_rows) * a.splits * tile_rows + row % tile_rows;
        float m = -FLT_MAX;
        for (uint32_t s = lane; s < n; s += 32) m = fmaxf(m, __ldcg(part_ml + first + (uint64_t)s * tile_rows).x);
#pragma unroll
        for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        constexpr int kPer = D / 32;
        float l = 0.0f, o[kPer] = {};
        bool gone = false;
#pragma unroll 4
        for (uint32_t s = 0; s < n; ++s) {
            const uint64_t at = first + (uint64_t)s * tile_rows;
            const float2 ml = __ldcg(part_ml + at);
            const float f = ex2(ml.x - m);
            gone |= ml.y == kLost;
            l += f * ml.y;
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                const float2 y = __ldcg(reinterpret_cast<const float2 *>(part_o + at * D + lane * kPer + i));
                o[i] += f * y.x;
                o[i + 1] += f * y.y;
            }
        }
        const uint32_t i = row / a.group, qh = head * a.group + row - i * a.group;
        const float inv = inverse(a, l, gone);
        const int64_t t = (int64_t)r * a.n_q + i;
#pragma unroll
        for (int x = 0; x < kPer; x += 2)
            *reinterpret_cast<uint32_t *>(a.out + t * a.o_ts + (int64_t)qh * a.o_hs + lane * kPer + x) =
                pk::Elem<DT>::from2(o[x] * inv, o[x + 1] * inv);
        if (lane == 0 && a.lse) a.lse[t * (a.kv_heads * a.group) + qh] = log_sum(m, l, gone);
        return;
    }
    const uint32_t per = pages_a_warp(a.page_grans), block_pages = kFinishWarps * per;
    const uint32_t blocks = a.weigh_blocks;
    const uint32_t id = blockIdx.x - join_blocks, r = id / blocks;
    const int32_t len = length_of(kv_len, r, most);
    const uint32_t n = live_splits<kWindow>(a, len), n_gran = ((uint32_t)len + 15) / 16;
    const uint32_t skip = kWindow ? gap_of(a, len) : 0;  // the granules [sink_grans, sink_grans + skip) nobody sees
    // with a window: blocks of pages for the first tokens, then those from the window's first page on. A block for every
    // page of the table, most with nothing to do: 52.1 against 48.9 us at 128 x 8192 tokens behind a window of 1024.
    uint32_t block = id % blocks;
    if (kWindow && block >= a.sink_blocks)
        block += max((a.sink_grans + skip) / a.page_grans / block_pages, a.sink_blocks) - a.sink_blocks;
    if ((uint64_t)block * block_pages >= a.page_stride) return;  // uniform
    const uint32_t page0 = block * block_pages;
    const uint64_t block_end = ((uint64_t)page0 + block_pages) * a.page_grans;
    // uniform: no token in these pages, or none that is seen
    if ((uint64_t)page0 * a.page_grans >= n_gran) return;
    if (kWindow && (uint64_t)page0 * a.page_grans >= a.sink_grans && block_end <= (uint64_t)a.sink_grans + skip) return;
    const uint32_t total = a.kv_heads * a.rows;
    const uint32_t page = page0 + warp * per, gr0 = page * a.page_grans, gr1 = min(gr0 + per * a.page_grans, n_gran);
    float acc[4] = {};  // of the granules gr0 + i mod 4
    for (uint32_t base = 0; base < total; base += kStatRows) {
        __syncthreads();
        for (uint32_t x = tid; x < kStatRows && base + x < total; x += kFinishThreads) {
            const uint32_t head = (base + x) / a.rows, row = (base + x) % a.rows;
            const uint64_t first = (((uint64_t)r * a.kv_heads + head) * a.row_tiles + row / tile_rows) * a.splits *
                                       tile_rows + row % tile_rows;
            float m = -FLT_MAX, l = 0.0f;
            bool gone = false;
#pragma unroll 8
            for (uint32_t s = 0; s < n; ++s) {
                const float2 ml = __ldcg(part_ml + first + (uint64_t)s * tile_rows);
                const float to = fmaxf(m, ml.x);
                l = l * ex2(m - to) + ml.y * ex2(ml.x - to);
                m = to;
                gone |= ml.y == kLost;
            }
            stat[x] = make_float2(m, l == 0.0f || gone ? 0.0f : 1.0f / l);
        }
        __syncthreads();
        for (uint32_t x = lane; x < kStatRows && base + x < total; x += 32) {
            const uint32_t head = (base + x) / a.rows, row = (base + x) % a.rows;
            const float2 st = stat[x];
            if (st.y == 0.0f) continue;  // no key, or a slot out of range: nothing is added, whatever the sums hold
            const float2 *src = gran_ml + (((uint64_t)r * a.kv_heads + head) * a.row_tiles + row / tile_rows) *
                                              a.gran_stride * a.gran_rows + row % tile_rows;
#pragma unroll 2
            for (uint32_t gr = gr0; gr < gr1; gr += 4) {
                float2 y[4];
                bool in[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t at = !kWindow || gr + i < a.sink_grans ? gr + i : gr + i - skip;  // among those seen
                    in[i] = gr + i < gr1 && (!kWindow || gr + i < a.sink_grans || gr + i >= a.sink_grans + skip);
                    y[i] = in[i] ? __ldcg(src + (uint64_t)at * a.gran_rows) : make_float2(0.0f, -FLT_MAX);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (in[i]) acc[i] += y[i].x * ex2(y[i].y - st.x) * st.y;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 16; d; d /= 2) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], d);
    // lane p adds to page p of the warp's
    if (lane < per && gr0 + lane * a.page_grans < gr1) {
        float sum = per == 1 ? (acc[0] + acc[1]) + (acc[2] + acc[3]) : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (per > 1 && i / a.page_grans == lane) sum += acc[i];
        weight[(uint64_t)r * a.page_stride + page + lane] += sum;
    }
}

struct Plan {
    uint32_t rows, tile_rows, row_tiles, splits, split_grans, max_grans;
    uint64_t part_rows, o_bytes, ml_bytes, gran_bytes;
    uint64_t blocks, join, weigh;  // of k_attend_cache; of k_cache_finish
    uint32_t weigh_blocks, sink_blocks;
};

uint64_t up16(uint64_t x) { return (x + 15) & ~15ull; }

// How the call is cut.  Tiles of 8 query rows, or 16 where there are more: a
// second column of tiles uses the dequantised values again.  Splits: enough
// CTAs for kWaves rounds, so that requests of different lengths even out, but of
// kMinGrans granules at least: below that a split's start and the join cost more
// than it gives (128 x 2048 tokens, by least granules of a split: 32 74 us, 64
// 67 us, 128 65 us).  Where that leaves places free, shorter ones down to
// kLeastGrans fill them: the call then lasts as long as one split.
constexpr uint64_t kWaves = 6, kMinGrans = 128, kLeastGrans = 32;
Plan plan_of(const pk_kv_cache &kv, uint32_t R, uint32_t n_q, uint32_t q_heads, uint64_t page_stride, bool weigh,
             uint32_t window, uint32_t sinks) {
    Plan p;
    p.rows = q_heads / kv.kv_heads * n_q;
    p.tile_rows = p.rows <= 8 ? 8 : 16;
    p.row_tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
    p.max_grans = (uint32_t)(page_stride * kv.page_tokens / 16);
    // with a window: the first tokens' granules, and those that window + n_q - 1 positions can touch
    if (window)
        p.max_grans = (uint32_t)std::min<uint64_t>(p.max_grans, ((uint64_t)sinks + 15) / 16 + ((uint64_t)window + n_q + 14) / 16 + 1);
    const uint64_t units = (uint64_t)R * kv.kv_heads * p.row_tiles;
    auto up = [](uint64_t x, uint64_t by) { return by ? (x + by - 1) / by : 1; };
    uint64_t n = std::min(up(kSlots * kWaves, units), up(p.max_grans, kMinGrans));
    if (units * n < kSlots) n = std::max(n, std::min(up(kSlots, units), up(p.max_grans, kLeastGrans)));
    if (n < 1) n = 1;
    p.split_grans = (uint32_t)((p.max_grans + n - 1) / n);
    p.split_grans = (p.split_grans + 2 * kWarps - 1) / (2 * kWarps) * (2 * kWarps);  // whole steps of all warps
    if (p.split_grans == 0) p.split_grans = 2 * kWarps;
    p.splits = p.max_grans ? (p.max_grans + p.split_grans - 1) / p.split_grans : 1;
    p.part_rows = units * p.splits * p.tile_rows;
    p.o_bytes = p.splits > 1 ? up16(p.part_rows * kv.head_dim * 4) : 0;
    p.ml_bytes = p.splits > 1 || weigh ? up16(p.part_rows * 8) : 0;
    const uint64_t gran_rows = p.rows < p.tile_rows ? p.rows : p.tile_rows;
    p.gran_bytes = weigh ? up16(units * p.max_grans * gran_rows * 8) : 0;
    p.blocks = units * p.splits;
    p.join = p.splits > 1 ? ((uint64_t)R * kv.kv_heads * p.rows + kFinishWarps - 1) / kFinishWarps : 0;
    const uint64_t block_pages = kFinishWarps * pages_a_warp(kv.page_tokens / 16);
    uint64_t weigh_blocks = up(page_stride, block_pages);
    p.sink_blocks = 0;
    if (window) {
        p.sink_blocks = (uint32_t)std::min<uint64_t>(up(up(sinks, kv.page_tokens), block_pages), weigh_blocks);
        const uint64_t pages = ((uint64_t)window + n_q) / kv.page_tokens + 2;  // that a request's windows touch, at most
        weigh_blocks = std::min<uint64_t>(weigh_blocks, p.sink_blocks + pages / block_pages + 2);
    }
    p.weigh_blocks = (uint32_t)weigh_blocks;
    p.weigh = weigh ? weigh_blocks * R : 0;
    return p;
}

template <int D, int NT, uint32_t DT>
cudaError_t launch(const Args &a, const Plan &p, cudaStream_t s) {
    const int variant = (a.page_weight != nullptr) + 2 * (a.window != 0);
    void (*const kerns[4])(Args) = {k_attend_cache<D, NT, DT, false, false>, k_attend_cache<D, NT, DT, true, false>,
                                    k_attend_cache<D, NT, DT, false, true>, k_attend_cache<D, NT, DT, true, true>};
    void (*const kern)(Args) = kerns[variant];
    constexpr size_t smem = (size_t)kWarps * Shape<D, NT>::kRing;
    static std::atomic<uint64_t> seen[4] = {};
    cudaError_t e = pk_allow_smem(kern, smem, seen[variant]);
    if (e != cudaSuccess) return e;
    e = pk_launch_smem(kern, (unsigned)p.blocks, kThreads, smem, s, a);
    if (e == cudaSuccess && p.join + p.weigh)
        e = pk_launch(a.window ? k_cache_finish<D, DT, true> : k_cache_finish<D, DT, false>, (unsigned)(p.join + p.weigh),
                      kFinishThreads, s, a, p.tile_rows, (uint32_t)p.join);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

uint64_t pk_attend_cache_scratch_bytes_impl(const pk_kv_cache &kv, uint32_t R, uint32_t n_q, uint32_t q_heads,
                                            uint64_t page_stride, bool weigh, uint32_t window, uint32_t sinks) {
    const Plan p = plan_of(kv, R, n_q, q_heads, page_stride, weigh, window, sinks);
    if (p.blocks > 0x7fffffffull || p.join + p.weigh > 0x7fffffffull) return UINT64_MAX;
    return p.o_bytes + p.ml_bytes + p.gran_bytes;
}

cudaError_t pk_launch_attend_cache(const pk_kv_cache &kv, uint32_t dtype, const pk_heads &q, const pk_heads &out,
                                   float *lse, uint32_t R, uint32_t n_q, uint32_t q_heads, float scale,
                                   const int32_t *kv_len, const uint32_t *pages, uint64_t page_stride,
                                   float *page_weight, uint32_t window, uint32_t sinks, void *scratch, int32_t *status,
                                   cudaStream_t s) {
    const Plan p = plan_of(kv, R, n_q, q_heads, page_stride, page_weight, window, sinks);
    Args a;
    a.pool = static_cast<const uint8_t *>(kv.pool_dev);
    a.page_bytes = pk_kv_page_bytes(kv.page_tokens, kv.kv_heads, kv.head_dim);
    a.n_slots = kv.n_slots;
    a.page_tokens = kv.page_tokens;
    a.page_grans = kv.page_tokens / 16;
    a.kv_heads = kv.kv_heads;
    a.group = q_heads / kv.kv_heads;
    a.n_q = n_q;
    a.rows = p.rows;
    a.row_tiles = p.row_tiles;
    a.R = R;
    a.splits = p.splits;
    a.split_grans = p.split_grans;
    // One CTA a request and head, and more of them than the GPU holds: the longest first, so that the last to start are
    // the shortest (128 x 2048 tokens: 65.6 -> 63.5 us; 100 x 1500, D = 64: 36.9 -> 35.2).  The search costs short
    // ones more than it gives (250 x 300: 31.7 -> 38.4 us).  Behind a window most requests weigh the same, and it costs
    // more than it gives (window 1024: 128 x 8192 tokens 50.9 -> 53.6, 250 x up to 1200, D = 64, 21.7 -> 23.1), but for
    // lengths about the window (128 x up to 1500: 46.9 -> 43.6; window 4096, 128 x up to 4096: even).
    a.by_length = !window && p.splits == 1 && R > 1 && R <= kRanked && p.max_grans >= kRankedGrans &&
                  (uint64_t)R * kv.kv_heads * p.row_tiles > kSlots;
    a.scale2 = (float)((double)scale * kv.k_scale * 1.4426950408889634);
    a.v_scale = kv.v_scale;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.sink_grans = (a.sinks + 15) / 16;
    a.weigh_blocks = p.weigh_blocks;
    a.sink_blocks = p.sink_blocks;
    a.q = static_cast<const uint16_t *>(q.p);
    a.q_ts = q.tok_stride;
    a.q_hs = q.head_stride;
    a.out = static_cast<uint16_t *>(out.p);
    a.o_ts = out.tok_stride;
    a.o_hs = out.head_stride;
    a.lse = lse;
    a.kv_len = kv_len;
    a.pages = pages;
    a.page_stride = page_stride;
    uint8_t *at = static_cast<uint8_t *>(scratch);
    a.part_o = p.o_bytes ? reinterpret_cast<float *>(at) : nullptr;
    a.part_ml = p.ml_bytes ? reinterpret_cast<float2 *>(at + p.o_bytes) : nullptr;
    a.gran_ml = p.gran_bytes ? reinterpret_cast<float2 *>(at + p.o_bytes + p.ml_bytes) : nullptr;
    a.gran_stride = p.max_grans;
    a.gran_rows = p.rows < p.tile_rows ? p.rows : p.tile_rows;
    a.page_weight = page_weight;
    a.status = status;
    const bool wide = p.tile_rows == 16;
    if (kv.head_dim == 128) {
        if (dtype == PK_BF16) return wide ? launch<128, 2, PK_BF16>(a, p, s) : launch<128, 1, PK_BF16>(a, p, s);
        return wide ? launch<128, 2, PK_FP16>(a, p, s) : launch<128, 1, PK_FP16>(a, p, s);
    }
    if (dtype == PK_BF16) return wide ? launch<64, 2, PK_BF16>(a, p, s) : launch<64, 1, PK_BF16>(a, p, s);
    return wide ? launch<64, 2, PK_FP16>(a, p, s) : launch<64, 1, PK_FP16>(a, p, s);
}
