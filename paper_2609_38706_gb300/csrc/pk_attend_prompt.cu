// pk_attend_prompt.cu -- causal attention over packed prompts with grouped
// heads (pk_attend_prompt).
#include <cuda.h>
#include <cuda_runtime.h>
#include <float.h>

#include <type_traits>

#include "pk_device.cuh"
#include "pk_internal.h"
#include "pk_kv.cuh"
#include "pk_tcgen05.cuh"
#include "pk_tma.cuh"

namespace {

constexpr int kTileRows = 256;  // (query token, head of the group) rows of a CTA: two tiles of 128
constexpr int kKeys = 128;      // keys of a tile
constexpr int kThreads = 384;
constexpr float kTop = 15.0f;   // p stays below 2^kTop (half: 2^16)
constexpr float kBase = 8.0f;   // the largest p when the reference moves: 2^kBase
constexpr int kPlanThreads = 1024;

struct Args {
    const uint16_t *q;
    uint16_t *out;
    int64_t q_ts, q_hs, o_ts, o_hs;
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

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Shared memory of a CTA, from a 1024-byte boundary: Q (two tiles), the ring
// of K and V tiles, then the small things.
template <int D>
struct Layout {
    static constexpr uint32_t kTile = 128 * D * 2;  // 128 rows; blocks of [128][64] values, 16 KB each
    static constexpr uint32_t kStages = D == 128 ? 4 : 8;
    static constexpr uint32_t kRing = 2 * kTile;
    static constexpr uint32_t kBytes = kRing + kStages * kTile;
};

struct Small {
    uint64_t full[8], empty[8];    // ring stages: tile ready (loaded, and an edge tile's V made finite); no longer read
    uint64_t s_full[2], p_ready[2], o_done[2];
    uint64_t q_ready, edge_v[4];   // Q in shared memory; an edge tile's V loaded, by edge tile
    uint32_t tmem, abort;
    int32_t bad_row[128];          // first key of an edge tile whose V is not finite, by dimension
};

using Yes = std::true_type;
using No = std::false_type;

constexpr uint32_t kWarpLoad = 8, kWarpMma = 9, kWarpClean = 10;  // warps 0-7: softmax

template <int D, uint32_t DT>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_prompt(const Args a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using L = Layout<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Small sm;
    const uint32_t smem = (pk::smem_addr(smem_raw) + 1023) & ~1023u;
    uint8_t *smem_p = smem_raw + (smem - pk::smem_addr(smem_raw));
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (uint32_t i = 0; i < L::kStages; ++i) {
            pk::mbar_init(pk::smem_addr(&sm.full[i]), 2);  // the loader twice, or the two cleaning warps
            pk::mbar_init(pk::smem_addr(&sm.empty[i]), 1);
        }
        for (int t = 0; t < 2; ++t) {
            pk::mbar_init(pk::smem_addr(&sm.s_full[t]), 1);
            pk::mbar_init(pk::smem_addr(&sm.p_ready[t]), 4);
            pk::mbar_init(pk::smem_addr(&sm.o_done[t]), 1);
        }
        pk::mbar_init(pk::smem_addr(&sm.q_ready), 8);
        for (int i = 0; i < 4; ++i) pk::mbar_init(pk::smem_addr(&sm.edge_v[i]), 1);
        pk::mbar_fence_init();
        sm.abort = 0;
    }
    if (tid < 128) sm.bad_row[tid] = 0x7fffffff;
    const uint64_t *tile_off = a.tile_off;
    const int64_t *q_off = a.q_off, *k_off = a.k_off;
    const uint16_t *qp = a.q;
    pk::pdl_wait(tile_off, q_off, k_off, qp);
    pk::pdl_launch_dependents();
    const uint32_t head = blockIdx.x % a.kv_heads;
    const uint64_t tile = blockIdx.x / a.kv_heads;
    if (tile >= __ldcg(tile_off + a.R)) return;  // uniform; nothing allocated yet
    if (warp == kWarpMma) pk::tmem_alloc(pk::smem_addr(&sm.tmem), 512);
    const uint32_t r = pk::warp_find_request(reinterpret_cast<const int64_t *>(tile_off), a.R, (int64_t)tile);
    const int64_t q0 = __ldcg(q_off + r), k0 = __ldcg(k_off + r);
    const int32_t lq = (int32_t)(__ldcg(q_off + r + 1) - q0), lk = (int32_t)(__ldcg(k_off + r + 1) - k0);
    // the last rows first: they have the most keys
    const int64_t row0 = (int64_t)(__ldcg(tile_off + r + 1) - 1 - tile) * kTileRows;
    const int64_t n_rows = (int64_t)lq * a.group;
    // per tile of 128 rows: how many key tiles its rows see, and the first key that some row does not
    int32_t n_tiles[2], first_last[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t r0 = row0 + 128 * t, r1 = min(r0 + 128, n_rows);  // [r0, r1)
        const int32_t keys = r1 > r0 ? (int32_t)((r1 - 1) / a.group) + lk - lq + 1 : 0;
        n_tiles[t] = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
        first_last[t] = (int32_t)(r0 / a.group) + lk - lq;
    }
    const int32_t n_all = max(n_tiles[0], n_tiles[1]);
    // From this key tile on, some row does not see some key: p = 0 there, which must not meet an infinity or NaN
    // of V.  At most three tiles: 256 rows hold at most 256 queries.
    const int32_t first_edge = first_last[0] + 1 >= kKeys ? (first_last[0] + 1) / kKeys : 0;
    pk::tmem_fence_before();
    __syncthreads();
    pk::tmem_fence_after();
    const uint32_t tmem = sm.tmem;
    const uint32_t tmem_s[2] = {tmem, tmem + 128}, tmem_o[2] = {tmem + 256, tmem + 256 + D};
    auto give_up = [&]() {
        if (lane == 0) {
            *reinterpret_cast<volatile uint32_t *>(&sm.abort) = 1;
            pk::set_status(a.status, PK_ERR_TIMEOUT);
        }
    };

    float inv = 0.0f;
    int32_t last = -1;
    if (warp == kWarpLoad) {
        if (lane == 0) {
            pk::fence_proxy_async();
            uint32_t n = 0;
            for (int32_t j = 0; j < n_all; ++j) {
                bool ok = true;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++n) {
                    const uint32_t st = n % L::kStages;
                    const bool dirty = kv && j >= first_edge;
                    const uint32_t bar = pk::smem_addr(dirty ? &sm.edge_v[(j - first_edge) & 3] : &sm.full[st]);
                    ok = ok && (n < L::kStages || pk::mbar_wait(pk::smem_addr(&sm.empty[st]), (n / L::kStages + 1) & 1));
                    if (!ok) break;
                    // only now: the barrier's earlier phase is over, as the stage was read
                    if (!dirty) pk::mbar_arrive(bar);
                    pk::mbar_expect(bar, L::kTile);
#pragma unroll
                    for (int b = 0; b < D / 64; ++b)
                        pk::tile_load3(smem + L::kRing + st * L::kTile + b * 16384, kv ? &map_v : &map_k, b * 64,
                                       (int)head, (int)(k0 + (int64_t)j * kKeys), bar);
                }
                if (!ok) {
                    give_up();
                    break;
                }
            }
            // no copy of its own stays in flight
            for (uint32_t i = n > L::kStages ? n - L::kStages : 0; i < n; ++i)
                pk::mbar_wait(pk::smem_addr(&sm.full[i % L::kStages]), (i / L::kStages) & 1);
        }
        __syncwarp();
    } else if (warp == kWarpMma) {
        if (lane == 0) {
            constexpr uint32_t kQk = pk::mma_idesc(DT == PK_BF16, 128, 128, false);
            constexpr uint32_t kPv = pk::mma_idesc(DT == PK_BF16, 128, D, true);
            bool ok = n_all == 0 || pk::mbar_wait(pk::smem_addr(&sm.q_ready), 0);
            auto stage_of = [&](uint32_t n) { return smem + L::kRing + (n % L::kStages) * L::kTile; };
            auto wait_full = [&](uint32_t n) {
                return pk::mbar_wait(pk::smem_addr(&sm.full[n % L::kStages]), (n / L::kStages) & 1);
            };
            auto qk = [&](int t, uint32_t n) {
                const uint32_t q = smem + t * L::kTile, k = stage_of(n);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    pk::mma_ss(tmem_s[t], pk::mma_desc(q + (s / 4) * 16384 + (s % 4) * 32, 16, 1024),
                               pk::mma_desc(k + (s / 4) * 16384 + (s % 4) * 32, 16, 1024), kQk, s > 0);
                pk::mma_commit(pk::smem_addr(&sm.s_full[t]));
            };
            if (ok && n_all) {
                ok = wait_full(0);
                pk::tmem_fence_after();
                if (ok) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        if (n_tiles[t] > 0) qk(t, 0);
                    pk::mma_commit(pk::smem_addr(&sm.empty[0]));
                }
            }
            for (int32_t j = 0; ok && j < n_all; ++j) {
                const uint32_t nv = 2 * j + 1, nk = 2 * j + 2;
                ok = wait_full(nv);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || j >= n_tiles[t]) continue;
                    ok = pk::mbar_wait(pk::smem_addr(&sm.p_ready[t]), j & 1);
                    if (!ok) break;
                    pk::tmem_fence_after();
                    const uint32_t v = stage_of(nv);
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        pk::mma_ts(tmem_o[t], tmem_s[t] + 8 * s, pk::mma_desc(v + s * 2048, 16384, 1024), kPv,
                                   j > 0 || s > 0);
                    pk::mma_commit(pk::smem_addr(&sm.o_done[t]));
                    if (j + 1 < n_tiles[t]) {
                        ok = wait_full(nk);
                        if (!ok) break;
                        qk(t, nk);
                    }
                }
                if (ok) {
                    pk::mma_commit(pk::smem_addr(&sm.empty[nv % L::kStages]));
                    if (j + 1 < n_all) pk::mma_commit(pk::smem_addr(&sm.empty[nk % L::kStages]));
                }
            }
            if (!ok) give_up();
        }
        __syncwarp();
    } else if (warp >= kWarpClean) {
        // V of the tiles at the causal edge and at the request's end: rows past its last key become 0, and so do
        // infinities and NaN, which are noted for the queries that do attend them
        bool ok = true;
        for (int32_t j = first_edge; ok && j < n_all; ++j) {
            const uint32_t st = (2 * j + 1) % L::kStages;
            ok = pk::mbar_wait_warp(pk::smem_addr(&sm.edge_v[(j - first_edge) & 3]), 0);  // used once
            if (!ok) break;
            uint8_t *v = smem_p + L::kRing + st * L::kTile;
            for (uint32_t x = tid - 32 * kWarpClean; x < L::kTile / 16; x += 64) {
                const uint32_t row = x / 8 % 128, chunk = (x ^ row) & 7;
                uint4 *at = reinterpret_cast<uint4 *>(v + x * 16);
                uint4 u = *at;
                const int32_t key = j * kKeys + (int32_t)row;
                constexpr uint32_t kInf = pk::Elem<DT>::kInfBits;
                if (key >= lk) {
                    if (u.x | u.y | u.z | u.w) *at = make_uint4(0, 0, 0, 0);
                    continue;
                }
                uint32_t w[4] = {u.x, u.y, u.z, u.w};
                bool found = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t d = x / 1024 * 64 + chunk * 8 + 2 * i;
                    if ((w[i] & 0x7fffu) >= kInf) {
                        atomicMin(&sm.bad_row[d], key);
                        w[i] &= 0xffff0000u;
                        found = true;
                    }
                    if ((w[i] >> 16 & 0x7fffu) >= kInf) {
                        atomicMin(&sm.bad_row[d + 1], key);
                        w[i] &= 0xffffu;
                        found = true;
                    }
                }
                if (found) *at = make_uint4(w[0], w[1], w[2], w[3]);
            }
            pk::fence_proxy_async();
            __syncwarp();
            if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.full[st]));
        }
        if (!ok) give_up();
    } else {
        const uint32_t t = warp >> 2;
        const int64_t row = row0 + tid;  // warps 0-3: tile 0, 4-7: tile 1; thread = row = TMEM lane
        const uint32_t lane_base = (warp & 3) * 32 << 16;
        const uint32_t flip = a.scale2 < 0.0f ? 0x80008000u : 0u;  // a negative scale goes into Q
        const float scale2 = fabsf(a.scale2);
        // Q: 8 lanes bring 128 bytes of a row; rows past the end are 0
        if (n_tiles[t] > 0) {
#pragma unroll 4
            for (int i = 0; i < 32 * (D / 64) / 4; ++i) {
                const uint32_t b = i / 8, rr = (warp & 3) * 32 + i % 8 * 4 + lane / 8, chunk = lane & 7;
                const int64_t qr = row0 + 128 * t + rr;
                uint4 u = make_uint4(0, 0, 0, 0);
                if (qr < n_rows) {
                    const int64_t i2 = qr / a.group;
                    u = __ldcg(reinterpret_cast<const uint4 *>(qp + (q0 + i2) * a.q_ts +
                                                               (int64_t)(head * a.group + (uint32_t)(qr - i2 * a.group)) * a.q_hs +
                                                               b * 64 + chunk * 8));
                    u.x ^= flip, u.y ^= flip, u.z ^= flip, u.w ^= flip;
                }
                *reinterpret_cast<uint4 *>(smem_p + t * L::kTile + b * 16384 + rr * 128 + ((chunk ^ (rr & 7)) << 4)) = u;
            }
            pk::fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.q_ready));

        const bool on = row < n_rows;
        const int64_t qi = on ? row / a.group : 0;
        last = on ? (int32_t)qi + lk - lq : -1;
        float ref = -FLT_MAX, sum = 0.0f;
        bool ok = true;
        const uint32_t ts = tmem_s[t] + lane_base, to = tmem_o[t] + lane_base;
#pragma unroll 1
        for (int32_t j = 0; j < n_tiles[t]; ++j) {
            ok = pk::mbar_wait_warp(pk::smem_addr(&sm.s_full[t]), j & 1);
            if (!ok) break;
            pk::tmem_fence_after();
            const bool edge = j * kKeys + kKeys - 1 > first_last[t];
            const int32_t see = last - j * kKeys;  // columns up to here
            float m = -INFINITY;
            uint32_t x[32];
            auto find_max = [&](auto masked) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    pk::tmem_load32(ts + 32 * c, x);
                    pk::tmem_wait_load(x);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!decltype(masked)::value || 32 * c + i <= see) m = fmaxf(m, __uint_as_float(x[i]));
                }
            };
            edge ? find_max(Yes{}) : find_max(No{});
            m *= scale2;
            const bool over = m > ref + kTop;
            if (__any_sync(0xffffffffu, over)) {
                const float next = over ? ceilf(m) - kBase : ref;
                const float f = ex2(ref - next);
                ref = next;
                sum *= f;
                if (j > 0) {
                    ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (j - 1) & 1);
                    if (!ok) break;
                    pk::tmem_fence_after();
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        pk::tmem_load32(to + 32 * c, x);
                        pk::tmem_wait_load(x);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
                        pk::tmem_store32(to + 32 * c, x);
                    }
                }
            }
            float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            auto weigh = [&](auto masked) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t p[16];
                    pk::tmem_load32(ts + 32 * c, x);
                    pk::tmem_wait_load(x);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float p0 = ex2(fmaf(__uint_as_float(x[i]), scale2, -ref));
                        float p1 = ex2(fmaf(__uint_as_float(x[i + 1]), scale2, -ref));
                        if (decltype(masked)::value) {
                            if (32 * c + i > see) p0 = 0.0f;
                            if (32 * c + i + 1 > see) p1 = 0.0f;
                        }
                        part[i / 2 & 3] += p0 + p1;
                        p[i / 2] = pk::Elem<DT>::from2(p0, p1);
                    }
                    pk::tmem_store16(ts + 16 * c, p);  // over scores that both passes have read
                }
            };
            edge ? weigh(Yes{}) : weigh(No{});
            sum += (part[0] + part[1]) + (part[2] + part[3]);
            pk::tmem_wait_store();
            pk::tmem_fence_before();
            __syncwarp();
            if (lane == 0) pk::mbar_arrive(pk::smem_addr(&sm.p_ready[t]));
        }
        if (ok && n_tiles[t] > 0) ok = pk::mbar_wait_warp(pk::smem_addr(&sm.o_done[t]), (n_tiles[t] - 1) & 1);
        if (!ok) give_up();
        inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (on && a.lse)
            a.lse[(q0 + qi) * a.q_heads + head * a.group + (uint32_t)(row - qi * a.group)] =
                sum == 0.0f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
    }
    __syncthreads();  // bad_row is final
    pk::tmem_fence_after();
    if (warp < 8 && sm.abort == 0) {
        const uint32_t t = warp >> 2;
        const int64_t row = row0 + tid;
        const bool on = row < n_rows;
        const int64_t qi = on ? row / a.group : 0;
        uint16_t *dst = a.out + (q0 + qi) * a.o_ts + (int64_t)(head * a.group + (uint32_t)(on ? row - qi * a.group : 0)) * a.o_hs;
        const bool any = n_tiles[t] > 0;  // else O was never written
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t x[32];
            __syncwarp();
            if (any) {
                pk::tmem_load32(tmem_o[t] + ((warp & 3) * 32 << 16) + 32 * c, x);
                pk::tmem_wait_load(x);
            }
            if (on) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    float y[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        y[e] = any && inv != 0.0f ? __uint_as_float(x[i + e]) * inv : 0.0f;
                        if (sm.bad_row[32 * c + i + e] <= last) y[e] = __int_as_float(0x7fffffff);
                    }
                    w[i / 2] = pk::Elem<DT>::from2(y[0], y[1]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    reinterpret_cast<uint4 *>(dst + 32 * c)[i] =
                        make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
            }
        }
    }
    pk::tmem_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        pk::tmem_fence_after();
        pk::tmem_free(tmem, 512);
    }
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

EncodeTiled encoder() {
    static const EncodeTiled fn = []() -> EncodeTiled {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// [tokens][heads][D] as a 3-D map whose box is 128 tokens of one head and 64 dimensions, in the 128-byte swizzle;
// tokens past the end read as 0.
cudaError_t map_of(CUtensorMap *map, const pk_heads &h, uint64_t n, uint32_t heads, uint32_t D, uint32_t dtype) {
    const EncodeTiled enc = encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {D, heads, n};
    // a dimension of one entry has no stride
    const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)h.head_stride * 2 : D * 2u, n > 1 ? (cuuint64_t)h.tok_stride * 2 : D * 2u};
    const cuuint32_t box[3] = {64, 1, kKeys}, unit[3] = {1, 1, 1};
    const CUresult e = enc(map, dtype == PK_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                           h.p, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return e == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, uint32_t DT>
cudaError_t launch(const Args &a, unsigned grid, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t s) {
    constexpr size_t smem = Layout<D>::kBytes + 1024;
    const cudaError_t e = cudaFuncSetAttribute(k_attend_prompt<D, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return e != cudaSuccess ? e : pk_launch_smem(k_attend_prompt<D, DT>, grid, kThreads, smem, s, a, mk, mv);
}

}  // namespace

cudaError_t pk_launch_attend_prompt(uint32_t dtype, const pk_heads &q, const pk_heads &k, const pk_heads &v,
                                    const pk_heads &out, float *lse, uint64_t n_q, uint64_t n_k, const int64_t *q_off,
                                    const int64_t *k_off, uint32_t R, uint32_t q_heads, uint32_t kv_heads,
                                    uint32_t head_dim, float scale, void *scratch, int32_t *status, cudaStream_t s) {
    Args a;
    a.q = static_cast<const uint16_t *>(q.p);
    a.out = static_cast<uint16_t *>(out.p);
    a.q_ts = q.tok_stride, a.q_hs = q.head_stride;
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
    CUtensorMap mk, mv;
    if (n_k == 0) {  // no key tile is ever loaded: any valid map will do
        mk = mv = CUtensorMap{};
    } else if ((e = map_of(&mk, k, n_k, kv_heads, head_dim, dtype)) != cudaSuccess ||
               (e = map_of(&mv, v, n_k, kv_heads, head_dim, dtype)) != cudaSuccess) {
        return e;
    }
    if (head_dim == 128)
        e = dtype == PK_BF16 ? launch<128, PK_BF16>(a, grid, mk, mv, s) : launch<128, PK_FP16>(a, grid, mk, mv, s);
    else
        e = dtype == PK_BF16 ? launch<64, PK_BF16>(a, grid, mk, mv, s) : launch<64, PK_FP16>(a, grid, mk, mv, s);
    return e != cudaSuccess ? e : cudaGetLastError();
}
