// pk_rotate.cu -- norms of queries and keys, a head at a time, and the rotation
// by their positions, in one pass (pk_rotate).
//
//     y = x / sqrt(mean(x^2) + eps) * w              (where weights are given)
//     (a, b) -> amp (a cos t - b sin t, a sin t + b cos t),   t = pos * f_i
//
// An angle is held in turns: f_i is a 64-bit fraction of a turn, so pos * f_i mod
// 2^64 is the product's part behind the whole turns, exact for any position, where
// a 32-bit product would be off by 0.004 rad at position 100000.  Its upper half,
// rounded to 24 bits (2^-26 of a turn at most), goes to sincospi.  All else is
// 32-bit arithmetic, rounded once, at the end.
//
// A lane holds the 16 values of 8 pairs of one head, so that nothing but the norm's
// sum crosses lanes, and the angles, which are a token's, serve all its heads.  The
// work is moving each value once either way, 4 bytes a value: 8 requests of up to 8192
// tokens of 40 heads, 128 values each (959 MB), take 161 us, 88% of a copy's rate, at
// 79% of the issue slots; the next row of a warp is on its way while one is worked on.
#include <cuda_runtime.h>
#include <float.h>

#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"

namespace {

constexpr int kThreads = 256;

struct Rotate {
    const uint16_t *x[2];  // queries, keys
    uint16_t *y[2];
    int64_t x_ts[2], x_hs[2], y_ts[2], y_hs[2];
    uint32_t heads[2];
    const uint16_t *w[2];
    float eps;
    const uint64_t *turns;
    uint32_t rotary_dim;
    float amplitude;
    uint64_t n_tokens;
    const int64_t *tok_off;
    const int32_t *start;
    uint32_t R;
    uint32_t parts, part_steps;  // warps that share a token; steps of each
    int32_t *status;
};

// Lane c of a head's D/16 holds two pieces of 8 values.  Halves: the pairs are (i, i + rot/2), so piece c and the
// one rot/2 behind it, and behind the rotated values two neighbours.  Interleaved, (2i, 2i + 1): two neighbours.
template <bool kHalves>
__device__ __forceinline__ void pieces_of(uint32_t c, uint32_t rotary_dim, uint32_t (&at)[2]) {
    const uint32_t pairs = rotary_dim / 16;  // lanes whose values are rotated
    if (kHalves && c < pairs) {
        at[0] = 8 * c;
        at[1] = 8 * (c + pairs);
    } else {
        at[0] = 16 * c;
        at[1] = 16 * c + 8;
    }
}

// D/16 lanes a head, 512/D heads a warp at a time; a warp takes part_steps such
// steps of one token's heads, queries first.
template <int D, uint32_t DT, bool kHalves>
__global__ void __launch_bounds__(kThreads, 4) k_rotate(const Rotate a) {
    constexpr uint32_t kLanes = D / 16, kHeads = 32 / kLanes;
    using E = pk::Elem<DT>;
    const uint32_t lane = threadIdx.x & 31, c = lane % kLanes;
    const uint64_t warp = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const uint64_t t = warp / a.parts;
    const uint32_t first_step = (uint32_t)(warp % a.parts) * a.part_steps;
    const int64_t *tok_off = a.tok_off;
    const int32_t *start = a.start;
    const uint64_t *turns = a.turns;
    const uint16_t *xq = a.x[0], *xk = a.x[1], *wq = a.w[0], *wk = a.w[1];
    pk::pdl_wait(tok_off, start, turns, xq, xk, wq, wk);
    pk::pdl_launch_dependents();

    uint32_t at[2];
    pieces_of<kHalves>(c, a.rotary_dim, at);
    // A step's rows, on their way while the one before is worked on, the first while its request is looked for.
    const uint32_t all = a.heads[0] + a.heads[1], end = min((first_step + a.part_steps) * kHeads, all);
    uint4 next[2] = {};
    auto load = [&](uint32_t h) {
        if (h >= end || t >= a.n_tokens) return;
        const bool key = h >= a.heads[0];
        const uint32_t in = key ? h - a.heads[0] : h;
        const uint16_t *src = (key ? xk : xq) + (int64_t)t * a.x_ts[key] + (int64_t)in * a.x_hs[key];
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = __ldcg(reinterpret_cast<const uint4 *>(src + at[i]));
    };
    uint32_t h = first_step * kHeads + lane / kLanes;
    load(h);

    // every request's offsets are looked at once, whatever the tokens do
    for (uint64_t r = (uint64_t)blockIdx.x * kThreads + threadIdx.x; r < a.R; r += (uint64_t)gridDim.x * kThreads) {
        const int64_t o0 = __ldcg(tok_off + r), o1 = __ldcg(tok_off + r + 1), s = __ldcg(start + r);
        if (o0 < 0 || o1 < o0 || (uint64_t)o1 > a.n_tokens || s < 0 || s + (o1 - o0) > (int64_t)1 << 31)
            pk::set_status(a.status, PK_ERR_ARG);
    }
    if (t >= a.n_tokens) return;  // uniform per warp

    // Through L1, as the table and the weights below: a few lines that every warp reads are a queue at the L2 (8 x 6144
    // tokens of 40 heads: 262 -> 171 us).
    const uint32_t r = pk::warp_find_request<true>(tok_off, a.R, (int64_t)t);
    const int64_t o0 = tok_off[r], o1 = tok_off[r + 1], s = start[r];
    const int64_t pos = s + ((int64_t)t - o0);
    // a token of no request, or of bad offsets, is left as it is
    if (o0 < 0 || (int64_t)t < o0 || (int64_t)t >= o1 || (uint64_t)o1 > a.n_tokens || s < 0 || pos >= (int64_t)1 << 31)
        return;

    const bool rotated = c < a.rotary_dim / 16;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const ulonglong2 f = rotated ? *reinterpret_cast<const ulonglong2 *>(turns + 8 * c + i) : make_ulonglong2(0, 0);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint64_t turn = (k ? f.y : f.x) * (uint64_t)pos;
            sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn[i + k], &cs[i + k]);
            sn[i + k] *= a.amplitude;
            cs[i + k] *= a.amplitude;
        }
    }
    uint4 w[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint16_t *p = j ? wk : wq;
#pragma unroll
        for (int i = 0; i < 2; ++i) w[j][i] = p ? *reinterpret_cast<const uint4 *>(p + at[i]) : make_uint4(0, 0, 0, 0);
    }

    for (uint32_t h0 = first_step * kHeads; h0 < end; h0 += kHeads, h += kHeads) {
        const bool on = h < end, key = h >= a.heads[0];
        const uint4 v[2] = {next[0], next[1]};
        load(h + kHeads);
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = E::to2(u[k]);
                x[i][2 * k] = f.x;
                x[i][2 * k + 1] = f.y;
            }
        }
        auto square_sum = [&]() {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) ss = fmaf(x[i][k], x[i][k], ss);
#pragma unroll
            for (int d = 1; d < (int)kLanes; d *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
            return ss;
        };
        const bool norm = (key ? wk : wq) != nullptr;
        if (wq || wk) {  // uniform: the sum is taken by all lanes
            float ss = square_sum();
            float inv = rsqrtf(ss * (1.0f / D) + a.eps);
            // squares past the top of 32 bits (|x| above 1e18): eps is nothing beside them
            if (__any_sync(0xffffffffu, ss > FLT_MAX)) {
                const bool big = ss > FLT_MAX;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[i][k] *= big && norm ? 0x1p-68f : 1.0f;
                ss = square_sum();
                if (big) inv = rsqrtf(ss * (1.0f / D));
            }
            if (norm) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 m = key ? w[1][i] : w[0][i];
                    const uint32_t u[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 f = E::to2(u[k]);
                        x[i][2 * k] = x[i][2 * k] * inv * f.x;
                        x[i][2 * k + 1] = x[i][2 * k + 1] * inv * f.y;
                    }
                }
            }
        }
        if (rotated) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float &p = kHalves ? x[0][i] : x[i / 4][2 * i % 8], &q = kHalves ? x[1][i] : x[i / 4][2 * i % 8 + 1];
                const float u = p, z = q;
                p = fmaf(u, cs[i], -(z * sn[i]));
                q = fmaf(u, sn[i], z * cs[i]);
            }
        }
        if (!on) continue;
        const uint32_t in = key ? h - a.heads[0] : h;
        uint16_t *dst = (key ? a.y[1] : a.y[0]) + (int64_t)t * a.y_ts[key] + (int64_t)in * a.y_hs[key];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<uint4 *>(dst + at[i]) = make_uint4(E::from2(x[i][0], x[i][1]), E::from2(x[i][2], x[i][3]),
                                                                  E::from2(x[i][4], x[i][5]), E::from2(x[i][6], x[i][7]));
    }
}

}  // namespace

cudaError_t pk_launch_rotate(uint32_t dtype, const pk_heads &q, const pk_heads &k, const pk_heads &q_out,
                             const pk_heads &k_out, uint64_t n_tokens, uint32_t q_heads, uint32_t kv_heads,
                             uint32_t head_dim, const pk_rotary &rotary, const void *q_weight, const void *k_weight,
                             float eps, const int64_t *tok_off, const int32_t *start, uint32_t R, int32_t *status,
                             cudaStream_t s) {
    Rotate a;
    const pk_heads *in[2] = {&q, &k}, *out[2] = {&q_out, &k_out};
    for (int j = 0; j < 2; ++j) {
        a.x[j] = static_cast<const uint16_t *>(in[j]->p);
        a.y[j] = static_cast<uint16_t *>(out[j]->p);
        a.x_ts[j] = in[j]->tok_stride, a.x_hs[j] = in[j]->head_stride;
        a.y_ts[j] = out[j]->tok_stride, a.y_hs[j] = out[j]->head_stride;
    }
    a.heads[0] = q_heads;
    a.heads[1] = kv_heads;
    a.w[0] = static_cast<const uint16_t *>(q_weight);
    a.w[1] = static_cast<const uint16_t *>(k_weight);
    a.eps = eps;
    a.turns = rotary.turns_dev;
    a.rotary_dim = rotary.rotary_dim;
    a.amplitude = rotary.amplitude;
    a.n_tokens = n_tokens;
    a.tok_off = tok_off;
    a.start = start;
    a.R = R;
    a.status = status;
    // A token's heads to one warp, which then has its angles once; to more, each with fewer steps one behind the other,
    // while that leaves SMs without work (64 tokens of 40 heads: 9.1 -> 3.2 us).
    const uint32_t steps = (q_heads + kv_heads + 512 / head_dim - 1) / (512 / head_dim);
    a.part_steps = 1;
    while (a.part_steps < steps && n_tokens * steps / a.part_steps > 152 * 48) a.part_steps *= 2;
    if (a.part_steps > steps) a.part_steps = steps;
    a.parts = (steps + a.part_steps - 1) / a.part_steps;
    const uint64_t blocks = (n_tokens * a.parts + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffull) return cudaErrorInvalidValue;
    void (*const kernels[2][2][2])(Rotate) = {
        {{k_rotate<64, PK_BF16, true>, k_rotate<64, PK_BF16, false>}, {k_rotate<64, PK_FP16, true>, k_rotate<64, PK_FP16, false>}},
        {{k_rotate<128, PK_BF16, true>, k_rotate<128, PK_BF16, false>}, {k_rotate<128, PK_FP16, true>, k_rotate<128, PK_FP16, false>}}};
    const cudaError_t e = pk_launch(kernels[head_dim == 128][dtype][rotary.interleaved != 0], (unsigned)blocks, kThreads, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}
