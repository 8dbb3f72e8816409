// pk_attend_prompt.cu -- causal attention over packed prompts with grouped
// heads (pk_attend_prompt).
#include <cuda_runtime.h>
#include <float.h>

#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"
#include "pk_tma.cuh"

namespace {

constexpr int kTileRows = 64;   // (query token, head of the group) rows of a CTA
constexpr int kKeys = 64;
constexpr int kThreads = 128;
constexpr int kPlanThreads = 1024;

struct Args {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;
    float *lse;
    const int64_t *q_off, *k_off;
    uint64_t *tile_off;  // [R + 1]: tiles of the requests before r
    uint32_t R, q_heads, kv_heads, group;
    float scale2;  // scale * log2 e
    int32_t *status;
};

// tile_off: how many row tiles the requests before each one have; all zero
// where an offset is out of order or range.
__global__ void __launch_bounds__(kPlanThreads)
k_prompt_tiles(const int64_t *q_off, const int64_t *k_off, uint32_t R, uint64_t n_q, uint64_t n_k, uint32_t group,
               uint32_t tile_rows, uint64_t *tile_off, int32_t *status) {
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
            if (a < 0 || b < a || (uint64_t)b > n_q || e < 0 || f < e || (uint64_t)f > n_k)
                bad = 1;
            else
                n = ((uint64_t)(b - a) * group + tile_rows - 1) / tile_rows;
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

template <uint32_t DT>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (DT == PK_BF16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t movm(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// A CTA takes 64 rows of one request and KV head, row = query token * group +
// head of the group, and walks over the keys in tiles of 64 with the running
// maximum and sum of a softmax; a warp has 16 rows.
template <int D, uint32_t DT>
__global__ void __launch_bounds__(kThreads) k_attend_prompt(const Args a) {
    constexpr int kPad = D + 8;
    __shared__ __align__(16) uint16_t ks[kKeys][kPad], vs[kKeys][kPad];
    __shared__ int32_t bad_row[D];  // first visible-to-some key whose V is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint64_t *tile_off = a.tile_off;
    const int64_t *q_off = a.q_off, *k_off = a.k_off;
    const uint16_t *qp = a.q, *kp = a.k, *vp = a.v;
    pk::pdl_wait(tile_off, q_off, k_off, qp, kp, vp);
    pk::pdl_launch_dependents();
    const uint32_t head = blockIdx.x % a.kv_heads;
    const uint64_t tile = blockIdx.x / a.kv_heads;
    if (tile >= __ldcg(tile_off + a.R)) return;
    const uint32_t r = pk::warp_find_request(reinterpret_cast<const int64_t *>(tile_off), a.R, (int64_t)tile);
    const int64_t q0 = __ldcg(q_off + r), k0 = __ldcg(k_off + r);
    const int32_t lq = (int32_t)(__ldcg(q_off + r + 1) - q0), lk = (int32_t)(__ldcg(k_off + r + 1) - k0);
    // the last rows first: they have the most keys
    const int64_t row0 = (int64_t)(__ldcg(tile_off + r + 1) - 1 - tile) * kTileRows;
    const int64_t n_rows = (int64_t)lq * a.group;

    int32_t last[2];   // last key of rows g and g + 8
    int64_t tok[2];
    uint32_t qh[2];
    bool on[2];
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t row = row0 + warp * 16 + g + 8 * j;
        on[j] = row < n_rows;
        const int64_t i = on[j] ? row / a.group : 0;
        tok[j] = q0 + i;
        qh[j] = head * a.group + (on[j] ? (uint32_t)(row - i * a.group) : 0);
        last[j] = on[j] ? (int32_t)i + lk - lq : -1;
        const uint16_t *src = qp + tok[j] * a.q_ts + (int64_t)qh[j] * a.q_hs;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int x = 0; x < 2; ++x)
                qf[s][j + 2 * x] =
                    on[j] ? __ldcg(reinterpret_cast<const uint32_t *>(src + 16 * s + 8 * x + 2 * c)) : 0;
    }
    const int64_t top_row = min(row0 + kTileRows, n_rows) - 1;
    const int32_t first_last = (int32_t)(row0 / a.group) + lk - lq;      // smallest `last` of the tile
    const int32_t n_keys = (int32_t)(top_row / a.group) + lk - lq + 1;   // keys that some row sees
    for (int d = tid; d < D; d += kThreads) bad_row[d] = 0x7fffffff;

    float o[D / 8][4], m[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    for (int32_t j0 = 0; j0 < n_keys; j0 += kKeys) {
        const bool edge = j0 + kKeys - 1 > first_last;
        __syncthreads();
        for (int x = tid; x < kKeys * D / 8; x += kThreads) {
            const int row = x / (D / 8), col = x % (D / 8) * 8;
            uint4 u = make_uint4(0, 0, 0, 0), w = u;
            if (j0 + row < n_keys) {
                u = __ldcg(reinterpret_cast<const uint4 *>(kp + (k0 + j0 + row) * a.k_ts + (int64_t)head * a.k_hs + col));
                w = __ldcg(reinterpret_cast<const uint4 *>(vp + (k0 + j0 + row) * a.v_ts + (int64_t)head * a.v_hs + col));
            }
            if (edge) {  // p = 0 must not meet an infinity or NaN
                uint16_t *h = reinterpret_cast<uint16_t *>(&w);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((h[i] & 0x7fffu) >= pk::Elem<DT>::kInfBits) {
                        atomicMin(&bad_row[col + i], j0 + row);
                        h[i] = 0;
                    }
            }
            *reinterpret_cast<uint4 *>(&ks[row][col]) = u;
            *reinterpret_cast<uint4 *>(&vs[row][col]) = w;
        }
        __syncthreads();
        float s[kKeys / 8][4];
#pragma unroll
        for (int n = 0; n < kKeys / 8; ++n) {
            s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
            for (int x = 0; x < D / 16; ++x)
                mma<DT>(s[n], qf[x], *reinterpret_cast<const uint32_t *>(&ks[n * 8 + g][16 * x + 2 * c]),
                        *reinterpret_cast<const uint32_t *>(&ks[n * 8 + g][16 * x + 8 + 2 * c]));
        }
        float mx[2] = {m[0], m[1]};
#pragma unroll
        for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] *= a.scale2;
                if (edge && j0 + n * 8 + (int)(2 * c) + (e & 1) > last[e >> 1]) s[n][e] = -INFINITY;
                mx[e >> 1] = fmaxf(mx[e >> 1], s[n][e]);
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 1));
            mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 2));
            const float f = exp2f(m[j] - mx[j]);
            m[j] = mx[j];
            l[j] *= f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) o[i][2 * j] *= f, o[i][2 * j + 1] *= f;
        }
#pragma unroll
        for (int n = 0; n < kKeys / 8; n += 2) {
            uint32_t pf[4];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p0 = exp2f(s[n + x][2 * j] - m[j]), p1 = exp2f(s[n + x][2 * j + 1] - m[j]);
                    l[j] += p0 + p1;
                    pf[j + 2 * x] = pk::Elem<DT>::from2(p0, p1);
                }
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const uint32_t b0 = movm(*reinterpret_cast<const uint32_t *>(&vs[n * 8 + g][8 * i + 2 * c]));
                const uint32_t b1 = movm(*reinterpret_cast<const uint32_t *>(&vs[n * 8 + 8 + g][8 * i + 2 * c]));
                mma<DT>(o[i], pf, b0, b1);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
        if (!on[j]) continue;
        const float inv = l[j] == 0.0f ? 0.0f : 1.0f / l[j];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const int d = 8 * i + 2 * c;
            float x = o[i][2 * j] * inv, y = o[i][2 * j + 1] * inv;
            if (bad_row[d] <= last[j]) x = __int_as_float(0x7fffffff);
            if (bad_row[d + 1] <= last[j]) y = __int_as_float(0x7fffffff);
            *reinterpret_cast<uint32_t *>(a.out + tok[j] * a.o_ts + (int64_t)qh[j] * a.o_hs + d) =
                pk::Elem<DT>::from2(x, y);
        }
        if (c == 0 && a.lse)
            a.lse[tok[j] * a.q_heads + qh[j]] =
                l[j] == 0.0f ? -INFINITY : (m[j] + log2f(l[j])) * 0.69314718055994531f;
    }
}

}  // namespace

cudaError_t pk_launch_attend_prompt(uint32_t dtype, const pk_heads &q, const pk_heads &k, const pk_heads &v,
                                    const pk_heads &out, float *lse, uint64_t n_q, uint64_t n_k, const int64_t *q_off,
                                    const int64_t *k_off, uint32_t R, uint32_t q_heads, uint32_t kv_heads,
                                    uint32_t head_dim, float scale, void *scratch, int32_t *status, cudaStream_t s) {
    Args a;
    a.q = static_cast<const uint16_t *>(q.p);
    a.k = static_cast<const uint16_t *>(k.p);
    a.v = static_cast<const uint16_t *>(v.p);
    a.out = static_cast<uint16_t *>(out.p);
    a.q_ts = q.tok_stride, a.q_hs = q.head_stride;
    a.k_ts = k.tok_stride, a.k_hs = k.head_stride;
    a.v_ts = v.tok_stride, a.v_hs = v.head_stride;
    a.o_ts = out.tok_stride, a.o_hs = out.head_stride;
    a.lse = lse;
    a.q_off = q_off;
    a.k_off = k_off;
    a.tile_off = static_cast<uint64_t *>(scratch);
    a.R = R;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.group = q_heads / kv_heads;
    a.scale2 = (float)((double)scale * 1.4426950408889634);
    a.status = status;
    cudaError_t e = pk_launch(k_prompt_tiles, 1, kPlanThreads, s, q_off, k_off, R, n_q, n_k, a.group,
                              (uint32_t)kTileRows, a.tile_off, status);
    if (e != cudaSuccess) return e;
    // every request rounds its rows up to whole tiles: at most one more tile each
    const uint64_t tiles = (n_q * a.group + kTileRows - 1) / kTileRows + R;
    if (tiles * kv_heads > 0x7fffffffull) return cudaErrorInvalidValue;
    const unsigned grid = (unsigned)(tiles * kv_heads);
    if (head_dim == 128)
        e = dtype == PK_BF16 ? pk_launch(k_attend_prompt<128, PK_BF16>, grid, kThreads, s, a)
                             : pk_launch(k_attend_prompt<128, PK_FP16>, grid, kThreads, s, a);
    else
        e = dtype == PK_BF16 ? pk_launch(k_attend_prompt<64, PK_BF16>, grid, kThreads, s, a)
                             : pk_launch(k_attend_prompt<64, PK_FP16>, grid, kThreads, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}
