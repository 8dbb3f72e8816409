// pk_kv.cu -- the 4-bit page store: quantise new K/V into their pages
// (pk_kv_write) and read pages back as 16-bit rows (pk_kv_read).
//
// A value is code * scale * k_scale (v_scale): per block of 16 dimensions the
// scale is e4m3(max|x| / 6 / k_scale) and a code e2m1(x / (scale * k_scale)).
// A lane has a whole block, so nothing is exchanged between lanes, and each byte
// moves once: 4 D bytes a token and head of rows, 1.125 D of pages.  64 prompts
// of 1024 to 2048 tokens (8 heads, D = 128, 511 MB either way): write 109 us, 4.7
// TB/s, held by the issue of the conversions (62% of the slots); read 89 us, 5.7
// TB/s.  Small calls are a chain of latencies: request, page, row, 4 us for one
// token a request.
#include <cuda_runtime.h>

#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"

namespace {

constexpr int kMoveThreads = 256;

struct Move {
    uint8_t *pool;
    uint64_t page_bytes, n_slots;
    uint32_t page_tokens, granules;  // granules of one head in a page
    uint32_t heads, heads_per_warp;
    bool wide;   // every block of x starts on 32 bytes
    float g[2];  // k_scale, v_scale
    uint16_t *x[2];
    int64_t ts[2], hs[2];
    uint64_t n_tokens;
    const int64_t *tok_off;
    const int32_t *start;
    uint32_t R;
    const uint32_t *pages;
    uint64_t page_stride, positions;  // positions: that a request can hold
    int32_t *status;
};

// x / den, correctly rounded, from inv = 1 / den correctly rounded: the quotient
// x * inv corrected once by its exact remainder (P. Markstein, "Computation of
// elementary functions on the IBM RISC System/6000 processor", 1990, theorem on
// quotients), for operands far from the ends of the range.  The sum of the two
// loses the sign of a zero.
__device__ __forceinline__ float divide(float x, float den, float inv) {
    const float y = __fmul_rn(x, inv);
    return copysignf(__fmaf_rn(__fmaf_rn(-y, den, x), inv, y), x);
}

// One block of 16 dimensions: 8 words of 16-bit values -> 8 code bytes and a
// scale byte.  The largest magnitude is found on the bits (same order), which
// also finds an infinity or NaN.  den = s * g and the true division x / den
// are the format's definition (pk.h): a tie between two codes is then decided
// by the values, not by a reciprocal's rounding.  A quotient below 2^-3 is code
// 0 however it is rounded, so divide() holds while den and the largest quotient,
// a / den, are far from the ends of the range.  Elsewhere (no calibrated scale is
// there) the plain division is called: past the top, divide() would take an
// infinity from an infinity.
template <uint32_t DT>
__device__ __forceinline__ void quantise16(const uint4 (&v)[2], float g, uint2 *codes, uint32_t *scale) {
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
    const bool finite = m < pk::Elem<DT>::kInfBits;
    const float a = pk::Elem<DT>::to1((uint16_t)m);
    const uint32_t s = finite ? pk::e4m3_byte(fminf(__fdiv_rn(a * (1.0f / 6.0f), g), 448.0f)) : 0x7fu;
    const float den = __fmul_rn(pk::e4m3_to_float(s), g);
    uint32_t out[2] = {0, 0};
    if (finite && den > 0x1p-60f && den < 0x1p60f && a < den * 0x1p60f) {
        const float inv = __frcp_rn(den);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = pk::Elem<DT>::to2(w[i]);
            out[i / 4] |= pk::e2m1_pair(divide(x.x, den, inv), divide(x.y, den, inv)) << (8 * (i % 4));
        }
    } else {
        const bool live = finite && den > 0.0f;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            uint32_t u = w[0];
#pragma unroll
            for (int k = 1; k < 8; ++k) u = i == k ? w[k] : u;
            const float2 x = pk::Elem<DT>::to2(u);
            const float lo = live ? __fdiv_rn(x.x, den) : copysignf(0.0f, x.x);
            const float hi = live ? __fdiv_rn(x.y, den) : copysignf(0.0f, x.y);
            const uint32_t c = pk::e2m1_pair(lo, hi) << (8 * (i % 4));
            if (i < 4) out[0] |= c; else out[1] |= c;
        }
    }
    *codes = make_uint2(out[0], out[1]);
    *scale = s;
}

// D/16 lanes hold one token (16 dimensions each), so a warp takes 512/D tokens
// at a time and walks over heads_per_warp heads: the search for the tokens'
// requests is paid once.  Codes of a token are D/2 consecutive bytes and
// consecutive tokens of a granule follow each other, so whole 32-byte sectors
// are written where four tokens (two for D = 64's codes) lie together.
template <int D, uint32_t DT, bool kWrite>
__global__ void __launch_bounds__(kMoveThreads) k_kv_move(const Move a) {
    constexpr uint32_t kLanes = D / 16, kTokens = 32 / kLanes;
    using G = pk::Granule<D>;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t n_groups = (a.n_tokens + kTokens - 1) / kTokens;
    const uint32_t head_parts = (a.heads + a.heads_per_warp - 1) / a.heads_per_warp;
    const uint64_t group = (uint64_t)(blockIdx.x / head_parts) * (kMoveThreads / 32) + threadIdx.x / 32;
    const uint32_t h0 = blockIdx.x % head_parts * a.heads_per_warp;
    const int64_t *tok_off = a.tok_off;
    const int32_t *start = a.start;
    const uint32_t *pages = a.pages;
    uint8_t *pool = a.pool;
    uint16_t *xk = a.x[0], *xv = a.x[1];
    pk::pdl_wait(tok_off, start, pages, pool, xk, xv);

    // every request's offsets are looked at once, whatever the tokens do
    for (uint64_t r = (uint64_t)blockIdx.x * kMoveThreads + threadIdx.x; r < a.R;
         r += (uint64_t)gridDim.x * kMoveThreads) {
        const int64_t o0 = __ldcg(tok_off + r), o1 = __ldcg(tok_off + r + 1), s = __ldcg(start + r);
        if (o0 < 0 || o1 < o0 || (uint64_t)o1 > a.n_tokens || s < 0 ||
            (uint64_t)(s + (o1 - o0)) > a.positions)
            pk::set_status(a.status, PK_ERR_ARG);
    }
    if (group >= n_groups) return;  // uniform per warp

    const int64_t t0 = (int64_t)(group * kTokens);
    const int64_t t = t0 + lane / kLanes;
    const uint32_t r = pk::lane_request_window(tok_off, a.R, t0, __ldcg(tok_off + a.R), t);
    const int64_t first = __ldcg(tok_off + r), next = __ldcg(tok_off + r + 1);
    const bool mine = first >= 0 && t >= first && t < next && (uint64_t)next <= a.n_tokens;
    const int64_t pos = mine ? (int64_t)__ldcg(start + r) + (t - first) : -1;
    bool on = mine && pos >= t - first && (uint64_t)pos < a.positions;
    uint32_t slot = 0;
    const uint32_t page = on ? (uint32_t)pos / a.page_tokens : 0;
    if (on) {
        slot = __ldcg(pages + (uint64_t)r * a.page_stride + page);
        if (slot >= a.n_slots) {
            pk::set_status(a.status, PK_ERR_ARG);
            on = false;
        }
    }
    pk::pdl_launch_dependents();
    if (!on) return;  // no warp-wide step follows

    const uint32_t in_page = (uint32_t)pos - page * a.page_tokens;
    const uint32_t tok = in_page % pk::kGranTokens, block = lane % kLanes;
    uint8_t *base = pool + (uint64_t)slot * a.page_bytes + (uint64_t)(in_page / pk::kGranTokens) * G::kBytes;
    const uint32_t h1 = min(h0 + a.heads_per_warp, a.heads);
    // two heads at a time, all their loads ahead of the first store (the compiler cannot tell that they do not overlap)
    for (uint32_t h = h0; h < h1; h += 2) {
        const uint32_t pair = min(h1 - h, 2u);
        uint8_t *gran[2];
        uint4 x[2][2][2];
        uint2 c[2][2];
        uint32_t sc[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            gran[i] = base + (uint64_t)(h + i) * a.granules * G::kBytes;
            if (i >= pair) break;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (kWrite) {
                    pk::load32((j ? xv : xk) + t * a.ts[j] + (int64_t)(h + i) * a.hs[j] + block * 16, a.wide, x[i][j]);
                } else {
                    c[i][j] = __ldcg(reinterpret_cast<const uint2 *>(gran[i] + (j ? G::kV : G::kK) + tok * G::kRow + block * 8));
                    sc[i][j] = __ldcg(gran[i] + (j ? G::kVs : G::kKs) + tok * G::kScales + block);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i >= pair) break;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (kWrite) {
                    quantise16<DT>(x[i][j], a.g[j], &c[i][j], &sc[i][j]);
                    *reinterpret_cast<uint2 *>(gran[i] + (j ? G::kV : G::kK) + tok * G::kRow + block * 8) = c[i][j];
                    *(gran[i] + (j ? G::kVs : G::kKs) + tok * G::kScales + block) = (uint8_t)sc[i][j];
                } else {
                    const float den = __fmul_rn(pk::e4m3_to_float(sc[i][j]), a.g[j]);
                    uint32_t half[8], w[8];
                    pk::e2m1x8_to_half2(c[i][j].x, *reinterpret_cast<uint32_t(*)[4]>(half));
                    pk::e2m1x8_to_half2(c[i][j].y, *reinterpret_cast<uint32_t(*)[4]>(half + 4));
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&half[k]));
                        w[k] = pk::Elem<DT>::from2(__fmul_rn(f.x, den), __fmul_rn(f.y, den));
                    }
                    pk::store32((j ? xv : xk) + t * a.ts[j] + (int64_t)(h + i) * a.hs[j] + block * 16, a.wide, w);
                }
            }
        }
    }
}

}  // namespace

cudaError_t pk_launch_kv_move(bool write, const pk_kv_cache &kv, uint32_t dtype, const pk_heads &k, const pk_heads &v,
                              uint64_t n_tokens, const int64_t *tok_off, const int32_t *start, uint32_t R,
                              const uint32_t *pages, uint64_t page_stride, int32_t *status, cudaStream_t s) {
    Move a;
    a.pool = static_cast<uint8_t *>(kv.pool_dev);
    a.page_bytes = pk_kv_page_bytes(kv.page_tokens, kv.kv_heads, kv.head_dim);
    a.n_slots = kv.n_slots;
    a.page_tokens = kv.page_tokens;
    a.granules = kv.page_tokens / pk::kGranTokens;
    a.heads = kv.kv_heads;
    a.g[0] = kv.k_scale;
    a.g[1] = kv.v_scale;
    const pk_heads *x[2] = {&k, &v};
    a.wide = true;
    for (int j = 0; j < 2; ++j) {
        a.x[j] = static_cast<uint16_t *>(x[j]->p);
        a.ts[j] = x[j]->tok_stride;
        a.hs[j] = x[j]->head_stride;
        a.wide &= (reinterpret_cast<uintptr_t>(a.x[j]) & 31) == 0 && a.ts[j] % 16 == 0 && a.hs[j] % 16 == 0;
    }
    a.n_tokens = n_tokens;
    a.tok_off = tok_off;
    a.start = start;
    a.R = R;
    a.pages = pages;
    a.page_stride = page_stride;
    a.positions = page_stride * kv.page_tokens < 1ull << 31 ? page_stride * kv.page_tokens : 1ull << 31;
    a.status = status;
    const uint32_t tokens = 512 / kv.head_dim;
    const uint64_t groups = (n_tokens + tokens - 1) / tokens;
    // one head a warp while that leaves SMs without work, else up to 8
    a.heads_per_warp = 1;
    while (a.heads_per_warp < 8 && a.heads_per_warp < a.heads && groups * a.heads / a.heads_per_warp > 152 * 64)
        a.heads_per_warp *= 2;
    const uint32_t parts = (a.heads + a.heads_per_warp - 1) / a.heads_per_warp;
    const uint64_t blocks = (groups + kMoveThreads / 32 - 1) / (kMoveThreads / 32) * parts;
    if (blocks > 0x7fffffffull) return cudaErrorInvalidValue;
    void (*const kernels[2][2][2])(Move) = {
        {{k_kv_move<64, PK_BF16, false>, k_kv_move<64, PK_BF16, true>},
         {k_kv_move<64, PK_FP16, false>, k_kv_move<64, PK_FP16, true>}},
        {{k_kv_move<128, PK_BF16, false>, k_kv_move<128, PK_BF16, true>},
         {k_kv_move<128, PK_FP16, false>, k_kv_move<128, PK_FP16, true>}}};
    const cudaError_t e = pk_launch(kernels[kv.head_dim == 128][dtype][write], (unsigned)blocks, kMoveThreads, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}
