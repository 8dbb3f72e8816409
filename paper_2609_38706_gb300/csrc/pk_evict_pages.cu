// pk_evict_pages.cu -- cut each request's page list to a budget by accumulated
// attention weight (pk_evict_pages).
#include <cuda_runtime.h>

#include <type_traits>

#include "pk_device.cuh"
#include "pk_internal.h"

namespace {

// Weights as unsigned keys in the same order: NaN lowest, -0 equal to 0; no key is 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 1;
    const uint32_t b = __float_as_uint(w == 0.0f ? 0.0f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;  // -inf -> 0x007fffff: above NaN
}

constexpr uint32_t kFew = 512;  // keys that one warp goes on with

// One CTA per request whose row fits its registers, kPer consecutive pages a
// thread.  A page stays when its key is among the `budget` largest, sinks and
// recent pages having the largest key of all; of equal keys the lower index
// stays.  The search narrows [lo, hi) around the budget-th largest key: a guess
// in proportion to the keys on either side, how many keys reach it, and once
// exactly `budget` do, these are the pages.  Guesses in proportion take a third
// of the steps that the key's 32 bits would, and a step is kPer compares a
// thread and one barrier.  Kept and dropped pages are put in order in shared
// memory and leave in whole lines.  Bound by the issue of those steps: 512 rows of
// up to 8192 pages to 1024, 34 us with 53% of the issue slots taken and 512 CTAs
// for 304 places; its bytes alone would be 7 us.
template <int kThreads, int kPer>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
k_evict_resident(const uint32_t *pages, const float *weight, const int32_t *kv_len, uint32_t stride,
                 uint32_t page_tokens, uint32_t budget, uint32_t sinks, uint32_t recent, uint32_t *pages_out,
                 float *weight_out, int32_t *kv_len_out, uint32_t *evicted, int32_t *status) {
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint32_t order[];  // [stride]: dropped pages, in order
    __shared__ uint32_t warp_sum[2][32], result[3], found;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint64_t r = blockIdx.x;
    if (tid == 0) found = 0;
    pk::pdl_wait(pages, weight, kv_len, pages_out, weight_out, kv_len_out, evicted, status);
    pk::pdl_launch_dependents();
    pages += r * stride;
    weight += r * stride;
    pages_out += r * budget;
    weight_out += r * budget;
    if (evicted) evicted += r * stride;

    const uint32_t j0 = tid * kPer;
    // kPer consecutive values of a row, as whole vectors where its start allows it
    auto fetch = [&](const uint32_t *row, uint32_t(&x)[kPer]) {
        if (j0 + kPer <= stride && (reinterpret_cast<uintptr_t>(row) & 15) == 0) {
#pragma unroll
            for (int i = 0; i < kPer; i += 4) {
                const uint4 u = __ldcg(reinterpret_cast<const uint4 *>(row + j0 + i));
                x[i] = u.x, x[i + 1] = u.y, x[i + 2] = u.z, x[i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) x[i] = j0 + i < stride ? __ldcg(row + j0 + i) : 0u;
        }
    };
    uint32_t key[kPer];
    fetch(reinterpret_cast<const uint32_t *>(weight), key);
    int64_t len = __ldcg(kv_len + r);
    if (len < 0 || (uint64_t)len > (uint64_t)stride * page_tokens) {
        if (tid == 0) pk::set_status(status, PK_ERR_ARG);
        len = 0;
    }
    const uint32_t n = (uint32_t)((len + page_tokens - 1) / page_tokens);
    const uint32_t kept = min(n, budget);
    uint32_t least = 0xffffffffu, most = 0;  // of the competing keys
    if (j0 >= sinks && j0 + kPer + recent <= n) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            key[i] = weight_key(__uint_as_float(key[i]));
            least = min(least, key[i]), most = max(most, key[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t j = j0 + i;
            const bool safe = j < sinks || j + recent >= n;
            key[i] = j >= n ? 0u : safe ? 0xffffffffu : weight_key(__uint_as_float(key[i]));
            if (j < n && !safe) least = min(least, key[i]), most = max(most, key[i]);
        }
    }
    // a sum over the block; two buffers, so one barrier a call
    uint32_t turn = 0;
    auto block_sum = [&](uint32_t x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (lane == 0) warp_sum[turn][wid] = x;
        __syncthreads();
        x = __reduce_add_sync(0xffffffffu, lane < kWarps ? warp_sum[turn][lane] : 0u);
        turn ^= 1;
        return x;
    };
    uint32_t T = 0, ties = 0;  // keys above T stay, and of those equal to it the first `ties`
    const bool cut = n > budget;
    if (cut) {
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) warp_sum[0][wid] = least, warp_sum[1][wid] = most;
        __syncthreads();
        // lo: at least `budget` keys reach it (n_lo), hi: fewer do (n_hi)
        uint32_t lo = __reduce_min_sync(0xffffffffu, lane < kWarps ? warp_sum[0][lane] : 0xffffffffu);
        uint32_t hi = __reduce_max_sync(0xffffffffu, lane < kWarps ? warp_sum[1][lane] : 0u) + 1;
        uint32_t n_lo = n, n_hi = sinks + recent;
        __syncthreads();
        bool exact = n_hi == budget;
        if (exact) lo = hi;
        // One guess, by the share of keys on either side and every third time by halves; count(cand) says how many
        // keys reach it.
        auto narrow = [&](uint32_t step, auto count) {
            const float share = step % 3 == 2 ? 0.5f : __fdividef((float)(n_lo - budget), (float)(n_lo - n_hi));
            const uint32_t cand = min(max(lo + (uint32_t)((float)(hi - lo) * share), lo + 1), hi - 1);
            const uint32_t c = count(cand);
            if (c >= budget)
                lo = cand, n_lo = c, exact = c == budget;
            else
                hi = cand, n_hi = c;
        };
        uint32_t step = 0;
#pragma unroll 1
        for (; !exact && hi - lo > 1 && n_lo - n_hi > kFew; ++step)
            narrow(step, [&](uint32_t cand) {
                uint32_t c = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i) c += key[i] >= cand;
                return block_sum(c);
            });
        if (!exact && hi - lo > 1) {
            // few keys are left in [lo, hi): gathered in shared memory, in any order, for one warp to go on with
            uint32_t c = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) c += key[i] >= lo && key[i] < hi;
            uint32_t scan = c;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, scan, d);
                if (lane >= (uint32_t)d) scan += o;
            }
            uint32_t at = 0;
            if (lane == 31 && scan) at = atomicAdd(&found, scan);
            at = __shfl_sync(0xffffffffu, at, 31) + scan - c;
            if (c) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (key[i] >= lo && key[i] < hi) order[at++] = key[i];
            }
            __syncthreads();
            if (wid == 0) {
                uint32_t x[kFew / 32];
                const uint32_t beyond = n_hi, few = found;
#pragma unroll
                for (int i = 0; i < kFew / 32; ++i) x[i] = lane + 32 * i < few ? order[lane + 32 * i] : 0u;
#pragma unroll 1
                for (; !exact && hi - lo > 1; ++step)
                    narrow(step, [&](uint32_t cand) {
                        uint32_t k = 0;
#pragma unroll
                        for (int i = 0; i < kFew / 32; ++i) k += x[i] >= cand;
                        return beyond + __reduce_add_sync(0xffffffffu, k);
                    });
                if (lane == 0) result[0] = lo, result[1] = n_hi, result[2] = exact;
            }
            __syncthreads();
            lo = result[0], n_hi = result[1], exact = result[2] != 0;
        }
        T = exact ? lo - 1 : lo;
        ties = exact ? 0 : budget - n_hi;
    }
    // places in order: ranks of the two flags from one scan, packed
    uint32_t gt = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const bool in = j0 + i < n;
        gt |= (uint32_t)(in && (!cut || key[i] > T)) << i;
        eq |= (uint32_t)(in && cut && key[i] == T && ties) << i;
    }
    const uint32_t mine = __popc(gt) | __popc(eq) << 16;
    uint32_t scan = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    if (lane == 31) warp_sum[turn][wid] = scan;
    __syncthreads();
    uint32_t before = lane < wid ? warp_sum[turn][lane] : 0u;  // wid < 32
    before = __reduce_add_sync(0xffffffffu, before) + scan - mine;
    const uint32_t g0 = before & 0xffffu, e0 = before >> 16;
    // Pages and weights are read (again) now: only the keys had to live through the search.  Kept ones go out as they
    // are, an eighth of a thread's or so; dropped ones are put in order in shared memory and leave in whole vectors.
    auto place = [&](const uint32_t *row, uint32_t *out, bool dropped, auto some_ties) {
        uint32_t x[kPer];
        fetch(row, x);
        uint32_t g = g0, e = e0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool tie = decltype(some_ties)::value && (eq >> i & 1);
            const uint32_t first = decltype(some_ties)::value ? g + min(e, ties) : g;  // kept pages before this one
            if ((gt >> i & 1) || (tie && e < ties))
                out[first] = x[i];
            else if (dropped && j0 + i < n)
                order[j0 + i - first] = x[i];
            g += gt >> i & 1;
            e += tie;
        }
    };
    uint32_t *const weight_bits = reinterpret_cast<uint32_t *>(weight_out);
    if (ties) {
        place(pages, pages_out, evicted != nullptr, std::true_type{});
        place(reinterpret_cast<const uint32_t *>(weight), weight_bits, false, std::true_type{});
    } else {
        place(pages, pages_out, evicted != nullptr, std::false_type{});
        place(reinterpret_cast<const uint32_t *>(weight), weight_bits, false, std::false_type{});
    }
    for (uint32_t j = kept + tid; j < budget; j += kThreads) {
        pages_out[j] = PK_NO_SLOT;
        weight_out[j] = 0.0f;
    }
    if (evicted) {
        __syncthreads();
        const uint32_t gone = n - kept;
        const uint32_t whole = (reinterpret_cast<uintptr_t>(evicted) & 15) == 0 ? stride / 4 : 0;
        for (uint32_t j = tid; j < whole; j += kThreads) {
            uint4 u = reinterpret_cast<const uint4 *>(order)[j];
            if (4 * j + 3 >= gone) {
                if (4 * j >= gone) u.x = PK_NO_SLOT;
                if (4 * j + 1 >= gone) u.y = PK_NO_SLOT;
                if (4 * j + 2 >= gone) u.z = PK_NO_SLOT;
                u.w = PK_NO_SLOT;
            }
            reinterpret_cast<uint4 *>(evicted)[j] = u;
        }
        for (uint32_t j = 4 * whole + tid; j < stride; j += kThreads) evicted[j] = j < gone ? order[j] : PK_NO_SLOT;
    }
    if (tid == 0) kv_len_out[r] = (int32_t)(len - (int64_t)(n - kept) * page_tokens);
}

constexpr int kBins = 2048;

// One CTA per request of any length.  The lightest page that stays is found by a radix
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
    cudaError_t e;
    auto resident = [&](auto kernel, unsigned threads) {
        return pk_launch_smem(kernel, R, threads, ((size_t)page_stride * 4 + 15) & ~(size_t)15, s, pages, weight, kv_len,
                              (uint32_t)page_stride, page_tokens, budget, sinks, recent, pages_out, weight_out,
                              kv_len_out, evicted, status);
    };
    // Rows that a CTA's registers hold, by the smallest shape that does (512 rows of 8192 pages, 1024 to keep: 34 us
    // against 92 us by histogram; 64 rows of 128 pages, 4 a thread against 16: 5 against 8 us); longer ones by
    // histogram, whose passes read the row again.
    if (page_stride <= 256 * 4)
        e = resident(k_evict_resident<256, 4>, 256);
    else if (page_stride <= 256 * 16)
        e = resident(k_evict_resident<256, 16>, 256);
    else if (page_stride <= 512 * 16)
        e = resident(k_evict_resident<512, 16>, 512);
    else
        e = pk_launch(k_evict_pages<1024>, R, 1024, s, pages, weight, kv_len, page_stride, page_tokens, budget, sinks,
                      recent, pages_out, weight_out, kv_len_out, evicted, status);
    return e != cudaSuccess ? e : cudaGetLastError();
}
