// pk_evict_pages.cu -- cut each request's page list to a budget by accumulated
// attention weight (pk_evict_pages).
#include <cuda_runtime.h>

#include "pk_device.cuh"
#include "pk_internal.h"

namespace {

// Weights as unsigned keys in the same order: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t b = __float_as_uint(w == 0.0f ? 0.0f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;  // -inf -> 0x007fffff: above NaN
}

constexpr int kBins = 2048;

// One CTA per request.  The lightest page that stays is found by a radix
// select over the 32-bit keys of the pages between the sinks and the recent
// ones (11 + 11 + 10 bits: three histogram passes, the later ones from
// cache), so no order of the pages is ever formed; then one pass writes kept
// and dropped pages in index order.  With T the key of that lightest page, a
// page stays when its key is above T, or equal to it while `ties` last: both
// ranks come from one scan of the two flags, packed.
template <int kThreads>
__global__ void __launch_bounds__(kThreads)
k_evict_pages(const uint32_t *pages, const float *weight, const int32_t *kv_len, uint64_t stride,
              uint32_t page_tokens, uint32_t budget, uint32_t sinks, uint32_t recent, uint32_t *pages_out,
              float *weight_out, int32_t *kv_len_out, uint32_t *evicted, int32_t *status) {
    constexpr int kWarps = kThreads / 32;
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t warp_sum[2][kWarps];
    __shared__ uint32_t pick[2];  // chosen bin, keys still to take inside it
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint64_t r = blockIdx.x;
    pk::pdl_wait(pages, weight, kv_len, pages_out, weight_out, kv_len_out, evicted, status);
    pk::pdl_launch_dependents();
    pages += r * stride;
    weight += r * stride;
    pages_out += r * budget;
    weight_out += r * budget;
    if (evicted) evicted += r * stride;

    int64_t len = __ldcg(kv_len + r);
    if (len < 0 || (uint64_t)len > stride * page_tokens) {
        if (tid == 0) pk::set_status(status, PK_ERR_ARG);
        len = 0;
    }
    const uint32_t n = (uint32_t)((len + page_tokens - 1) / page_tokens);
    const bool cut = n > budget;
    const uint32_t m0 = cut ? sinks : n, m1 = cut ? n - recent : n;  // the pages that compete
    uint32_t want = cut ? budget - sinks - recent : 0;               // how many of them stay
    uint32_t T = 0xffffffffu;  // no key reaches it: no finite, infinite or NaN weight has this key
    if (want) {
        uint32_t prefix = 0, mask = 0;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int b = tid; b < kBins; b += kThreads) hist[b] = 0;
            __syncthreads();
            for (uint32_t j0 = m0; j0 < m1; j0 += kThreads) {
                const uint32_t j = j0 + tid;
                uint32_t bin = 0xffffffffu;
                if (j < m1) {
                    const uint32_t key = weight_key(__ldcg(weight + j));
                    if ((key & mask) == prefix) bin = (key >> shift) & ((1u << bits) - 1);
                }
                // equal weights are common (pages that never got any): one add for a warp that agrees
                const uint32_t bin0 = __shfl_sync(0xffffffffu, bin, 0);
                if (__all_sync(0xffffffffu, bin == bin0)) {
                    if (lane == 0 && bin != 0xffffffffu) atomicAdd(&hist[bin], 32u);
                } else if (bin != 0xffffffffu) {
                    atomicAdd(&hist[bin], 1u);
                }
            }
            __syncthreads();
            // from the top: the bin in which the want-th key lies
            constexpr int kPer = kBins / kThreads;
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) mine += hist[kBins - 1 - (tid * kPer + i)];
            uint32_t scan = mine;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, scan, d);
                if (lane >= (uint32_t)d) scan += o;
            }
            if (lane == 31) warp_sum[0][wid] = scan;
            __syncthreads();
            uint32_t before = scan - mine;
            for (uint32_t w = 0; w < wid; ++w) before += warp_sum[0][w];
            if (before < want && before + mine >= want) {  // one thread
#pragma unroll 1
                for (int i = 0; i < kPer; ++i) {
                    const uint32_t b = kBins - 1 - (tid * kPer + i), c = hist[b];
                    if (before + c >= want) {
                        pick[0] = b;
                        pick[1] = want - before;
                        break;
                    }
                    before += c;
                }
            }
            __syncthreads();
            prefix |= pick[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            want = pick[1];
        }
        T = prefix;
    }
    const uint32_t ties = want;  // keys equal to T that stay

    uint32_t gt_base = 0, eq_base = 0, turn = 0;
    for (uint32_t j0 = 0; j0 < n; j0 += kThreads, turn ^= 1) {
        const uint32_t j = j0 + tid;
        uint32_t slot = 0;
        float w = 0.0f;
        bool gt = false, eq = false;
        if (j < n) {
            slot = __ldcg(pages + j);
            w = __ldcg(weight + j);
            const uint32_t key = weight_key(w);
            gt = j < m0 || j >= m1 || key > T;
            eq = !gt && key == T;
        }
        const uint32_t bg = __ballot_sync(0xffffffffu, gt), be = __ballot_sync(0xffffffffu, eq);
        if (lane == 0) warp_sum[turn][wid] = (uint32_t)__popc(bg) | (uint32_t)__popc(be) << 16;
        __syncthreads();  // two buffers: the next chunk's sums go to the other one
        uint32_t before = 0, total = 0;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
            const uint32_t s = warp_sum[turn][k];
            if ((uint32_t)k < wid) before += s;
            total += s;
        }
        const uint32_t below = (1u << lane) - 1;
        const uint32_t g = gt_base + (before & 0xffffu) + __popc(bg & below);
        const uint32_t e = eq_base + (before >> 16) + __popc(be & below);
        const uint32_t at = g + min(e, ties);  // kept pages before j
        if (j < n) {
            if (gt || (eq && e < ties)) {
                pages_out[at] = slot;
                weight_out[at] = w;
            } else if (evicted) {
                evicted[j - at] = slot;
            }
        }
        gt_base += total & 0xffffu;
        eq_base += total >> 16;
    }
    const uint32_t kept = min(n, budget);
    for (uint32_t j = kept + tid; j < budget; j += kThreads) {
        pages_out[j] = PK_NO_SLOT;
        weight_out[j] = 0.0f;
    }
    if (evicted)
        for (uint64_t j = n - kept + tid; j < stride; j += kThreads) evicted[j] = PK_NO_SLOT;
    if (tid == 0) kv_len_out[r] = (int32_t)(len - (int64_t)(n - kept) * page_tokens);
}

}  // namespace

cudaError_t pk_launch_evict_pages(const uint32_t *pages, const float *weight, const int32_t *kv_len, uint32_t R,
                                  uint64_t page_stride, uint32_t page_tokens, uint32_t budget, uint32_t sinks,
                                  uint32_t recent, uint32_t *pages_out, float *weight_out, int32_t *kv_len_out,
                                  uint32_t *evicted, int32_t *status, cudaStream_t s) {
    if (R > 0x7fffffffu) return cudaErrorInvalidValue;
    const cudaError_t e =
        page_stride <= 1024
            ? pk_launch(k_evict_pages<256>, R, 256, s, pages, weight, kv_len, page_stride, page_tokens, budget, sinks,
                        recent, pages_out, weight_out, kv_len_out, evicted, status)
            : pk_launch(k_evict_pages<1024>, R, 1024, s, pages, weight, kv_len, page_stride, page_tokens, budget,
                        sinks, recent, pages_out, weight_out, kv_len_out, evicted, status);
    return e != cudaSuccess ? e : cudaGetLastError();
}
