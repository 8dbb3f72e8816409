// pk_kv_host.cpp -- host half of the KV-page calls: argument checks ahead of
// the launches of pk_kv.cu, pk_rotate.cu, pk_attend_prompt.cu,
// pk_attend_chunk.cu, pk_attend_cache.cu and pk_evict_pages.cu; the table of a rotation.
#include <cuda_runtime_api.h>

#include <cfloat>
#include <cmath>
#include <initializer_list>

#include "pk_internal.h"

namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int cuda_rc(cudaError_t e) { return e == cudaSuccess ? PK_OK : PK_ERR_CUDA; }

// A scale that multiplies values: finite and positive.
bool good_scale(float x) { return std::isfinite(x) && x > 0.0f; }

// A factor of scores whose exponents are taken to base 2, in 32 bits.
bool good_score_scale(double x) { return std::fabs(x * 1.4426950408889634) <= FLT_MAX; }  // false for NaN

bool good_cache(const pk_kv_cache *kv) {
    return kv && kv->pool_dev && aligned(kv->pool_dev, 16) && kv->n_slots >= 1 && kv->n_slots <= 0xffffffffull &&
           pk_kv_page_bytes(kv->page_tokens, kv->kv_heads, kv->head_dim) != 0 && good_scale(kv->k_scale) &&
           good_scale(kv->v_scale);
}

// rows * heads of 16-bit rows of 64 or 128 values; the largest offset must fit 62 bits.
bool good_heads(const pk_heads *h, uint64_t rows, uint32_t heads) {
    if (!h) return false;
    if (rows == 0) return true;
    const int64_t lim = (int64_t)1 << 61;
    return h->p && aligned(h->p, 16) && h->tok_stride >= 0 && h->head_stride >= 0 && h->tok_stride % 8 == 0 &&
           h->head_stride % 8 == 0 && (uint64_t)h->tok_stride <= (uint64_t)lim / (rows + 1) &&
           h->head_stride <= lim / ((int64_t)heads + 1);
}

// An output must not write one value twice: one stride steps over a row, the other over all that the first one spans.
bool good_out(const pk_heads *h, uint64_t rows, uint32_t heads, uint32_t head_dim) {
    if (!good_heads(h, rows, heads)) return false;
    if (rows == 0) return true;
    const int64_t d = head_dim, ts = h->tok_stride, hs = h->head_stride;
    if ((heads > 1 && hs < d) || (rows > 1 && ts < d)) return false;
    return heads == 1 || rows == 1 || ts >= hs * ((int64_t)heads - 1) + d || hs >= ts * ((int64_t)rows - 1) + d;
}

int kv_move(bool write, const pk_kv_cache *kv, uint32_t dtype, const pk_heads *k, const pk_heads *v,
            uint64_t n_tokens, const int64_t *tok_off_dev, const int32_t *start_dev, uint32_t R,
            const uint32_t *pages_dev, uint64_t page_stride, int32_t *status_dev, pk_stream stream) {
    if (!good_cache(kv) || dtype > PK_FP16) return PK_ERR_ARG;
    if (!aligned(tok_off_dev, 8) || !aligned(start_dev, 4) || !aligned(pages_dev, 4) || !aligned(status_dev, 4))
        return PK_ERR_ARG;
    if (write ? (!good_heads(k, n_tokens, kv->kv_heads) || !good_heads(v, n_tokens, kv->kv_heads))
              : (!good_out(k, n_tokens, kv->kv_heads, kv->head_dim) ||
                 !good_out(v, n_tokens, kv->kv_heads, kv->head_dim)))
        return PK_ERR_ARG;
    if (n_tokens >= 1ull << 32 || page_stride >= 1ull << 31) return PK_ERR_ARG;
    if (R == 0 || n_tokens == 0) return PK_OK;
    if (!tok_off_dev || !start_dev || (page_stride && !pages_dev)) return PK_ERR_ARG;
    return cuda_rc(pk_launch_kv_move(write, *kv, dtype, *k, *v, n_tokens, tok_off_dev, start_dev, R, pages_dev,
                                     page_stride, status_dev, reinterpret_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

size_t pk_kv_page_bytes(uint32_t page_tokens, uint32_t kv_heads, uint32_t head_dim) {
    if (page_tokens < 16 || page_tokens > 32768 || page_tokens % 16 || kv_heads < 1 || kv_heads > 1024 ||
        (head_dim != 64 && head_dim != 128))
        return 0;
    return (size_t)page_tokens * kv_heads * (head_dim + head_dim / 8);
}

int pk_kv_write(const pk_kv_cache *kv, uint32_t dtype, const pk_heads *k, const pk_heads *v, uint64_t n_tokens,
                const int64_t *tok_off_dev, const int32_t *start_dev, uint32_t R, const uint32_t *pages_dev,
                uint64_t page_stride, int32_t *status_dev, pk_stream stream) {
    return kv_move(true, kv, dtype, k, v, n_tokens, tok_off_dev, start_dev, R, pages_dev, page_stride, status_dev,
                   stream);
}

int pk_kv_read(const pk_kv_cache *kv, uint32_t dtype, const pk_heads *k, const pk_heads *v, uint64_t n_tokens,
               const int64_t *tok_off_dev, const int32_t *start_dev, uint32_t R, const uint32_t *pages_dev,
               uint64_t page_stride, int32_t *status_dev, pk_stream stream) {
    return kv_move(false, kv, dtype, k, v, n_tokens, tok_off_dev, start_dev, R, pages_dev, page_stride, status_dev,
                   stream);
}

size_t pk_attend_prompt_scratch_bytes(uint32_t R) { return ((size_t)R + 1) * 8 + 64; }

int pk_attend_prompt(uint32_t dtype, const pk_heads *q, const pk_heads *k, const pk_heads *v, const pk_heads *out,
                     float *lse_dev, uint64_t n_q, uint64_t n_k, const int64_t *q_off_dev, const int64_t *k_off_dev,
                     uint32_t R, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, float scale,
                     void *scratch_dev, size_t scratch_bytes, int32_t *status_dev, pk_stream stream) {
    if (dtype > PK_FP16 || (head_dim != 64 && head_dim != 128) || !good_score_scale(scale)) return PK_ERR_ARG;
    if (kv_heads == 0 || q_heads == 0 || q_heads % kv_heads || q_heads > 65536) return PK_ERR_ARG;
    if (n_q > 0x7fff0000ull || n_k > 0x7fff0000ull) return PK_ERR_ARG;  // a tile's end still fits 31 bits
    if (!good_heads(q, n_q, q_heads) || !good_heads(k, n_k, kv_heads) || !good_heads(v, n_k, kv_heads) ||
        !good_out(out, n_q, q_heads, head_dim))
        return PK_ERR_ARG;
    for (const pk_heads *h : {q, k, v})  // what a tensor map takes: less than 2^40 bytes
        if (h->tok_stride >= (int64_t)1 << 39 || h->head_stride >= (int64_t)1 << 39) return PK_ERR_ARG;
    if (!aligned(lse_dev, 4) || !aligned(q_off_dev, 8) || !aligned(k_off_dev, 8) || !aligned(scratch_dev, 16) ||
        !aligned(status_dev, 4))
        return PK_ERR_ARG;
    if (R == 0 || n_q == 0) return PK_OK;
    if (!q_off_dev || !k_off_dev || !scratch_dev || scratch_bytes < pk_attend_prompt_scratch_bytes(R) ||
        pk_attend_prompt_items(n_q, R, q_heads, kv_heads) > 0x7fffffffull)
        return PK_ERR_ARG;
    return cuda_rc(pk_launch_attend_prompt(dtype, *q, *k, *v, *out, lse_dev, n_q, n_k, q_off_dev, k_off_dev, R,
                                           q_heads, kv_heads, head_dim, scale, scratch_dev, status_dev,
                                           reinterpret_cast<cudaStream_t>(stream)));
}

// The shapes that both the scratch size and the launch depend on.
static bool good_attend(const pk_kv_cache *kv, uint32_t R, uint32_t n_q, uint32_t q_heads, uint64_t page_stride) {
    return kv && pk_kv_page_bytes(kv->page_tokens, kv->kv_heads, kv->head_dim) != 0 && n_q >= 1 && n_q <= 65536 &&
           q_heads >= 1 && q_heads <= 65536 && q_heads % kv->kv_heads == 0 &&
           (uint64_t)R * n_q * q_heads < 1ull << 31 && page_stride * kv->page_tokens < 1ull << 31 &&
           page_stride < 1ull << 31;
}

// A window that no request can outgrow is none; windows are positions, below 2^31 as they are.
static bool good_window(uint32_t window, uint32_t sinks) { return window < 1u << 31 && sinks < 1u << 31; }
static uint32_t window_within(const pk_kv_cache &kv, uint64_t page_stride, uint32_t window) {
    return window < page_stride * kv.page_tokens ? window : 0;
}

size_t pk_attend_cache_window_scratch_bytes(const pk_kv_cache *kv, uint32_t R, uint32_t n_q, uint32_t q_heads,
                                            uint64_t page_stride, int weigh, uint32_t window, uint32_t sinks) {
    if (!good_attend(kv, R, n_q, q_heads, page_stride) || !good_window(window, sinks)) return 0;
    const uint64_t need = pk_attend_cache_scratch_bytes_impl(*kv, R, n_q, q_heads, page_stride, weigh != 0,
                                                             window_within(*kv, page_stride, window), sinks);
    return need == UINT64_MAX ? 0 : (size_t)need;
}

size_t pk_attend_cache_scratch_bytes(const pk_kv_cache *kv, uint32_t R, uint32_t n_q, uint32_t q_heads,
                                     uint64_t page_stride, int weigh) {
    return pk_attend_cache_window_scratch_bytes(kv, R, n_q, q_heads, page_stride, weigh, 0, 0);
}

int pk_attend_cache_window(const pk_kv_cache *kv, uint32_t dtype, const pk_heads *q, const pk_heads *out, float *lse_dev,
                           uint32_t R, uint32_t n_q, uint32_t q_heads, float scale, uint32_t window, uint32_t sinks,
                           const int32_t *kv_len_dev, const uint32_t *pages_dev, uint64_t page_stride,
                           float *page_weight_dev, void *scratch_dev, size_t scratch_bytes, int32_t *status_dev,
                           pk_stream stream) {
    if (!good_cache(kv) || dtype > PK_FP16 || !good_score_scale((double)scale * kv->k_scale)) return PK_ERR_ARG;
    if (!good_attend(kv, R, n_q, q_heads, page_stride) || !good_window(window, sinks)) return PK_ERR_ARG;
    const uint64_t rows = (uint64_t)R * n_q;
    if (!good_heads(q, rows, q_heads) || !good_out(out, rows, q_heads, kv->head_dim)) return PK_ERR_ARG;
    if (!aligned(lse_dev, 4) || !aligned(kv_len_dev, 4) || !aligned(pages_dev, 4) || !aligned(page_weight_dev, 4) ||
        !aligned(scratch_dev, 16) || !aligned(status_dev, 4))
        return PK_ERR_ARG;
    if (R == 0) return PK_OK;
    if (!kv_len_dev || (page_stride && !pages_dev)) return PK_ERR_ARG;
    window = window_within(*kv, page_stride, window);
    const uint64_t need = pk_attend_cache_scratch_bytes_impl(*kv, R, n_q, q_heads, page_stride, page_weight_dev, window, sinks);
    if (need == UINT64_MAX || scratch_bytes < need || (need && !scratch_dev)) return PK_ERR_ARG;
    return cuda_rc(pk_launch_attend_cache(*kv, dtype, *q, *out, lse_dev, R, n_q, q_heads, scale, kv_len_dev,
                                          pages_dev, page_stride, page_weight_dev, window, sinks, scratch_dev,
                                          status_dev, reinterpret_cast<cudaStream_t>(stream)));
}

int pk_attend_cache(const pk_kv_cache *kv, uint32_t dtype, const pk_heads *q, const pk_heads *out, float *lse_dev,
                    uint32_t R, uint32_t n_q, uint32_t q_heads, float scale, const int32_t *kv_len_dev,
                    const uint32_t *pages_dev, uint64_t page_stride, float *page_weight_dev, void *scratch_dev,
                    size_t scratch_bytes, int32_t *status_dev, pk_stream stream) {
    return pk_attend_cache_window(kv, dtype, q, out, lse_dev, R, n_q, q_heads, scale, 0, 0, kv_len_dev, pages_dev,
                                  page_stride, page_weight_dev, scratch_dev, scratch_bytes, status_dev, stream);
}

// The shapes that both the scratch size and the launch depend on.
static bool good_chunk(const pk_kv_cache *kv, uint32_t R, uint64_t n_q, uint32_t q_heads, uint64_t page_stride,
                       uint32_t window, uint32_t sinks) {
    return kv && pk_kv_page_bytes(kv->page_tokens, kv->kv_heads, kv->head_dim) != 0 && n_q <= 0x7fff0000ull &&
           R < 1u << 31 && q_heads >= 1 && q_heads <= 65536 && q_heads % kv->kv_heads == 0 && n_q * q_heads < 1ull << 34 &&
           page_stride < 1ull << 31 && page_stride * kv->page_tokens <= 0x7fff0000ull && good_window(window, sinks);
}

size_t pk_attend_chunk_scratch_bytes(const pk_kv_cache *kv, uint32_t dtype, uint64_t n_q, uint32_t R, uint32_t q_heads,
                                     uint64_t page_stride, uint32_t window, uint32_t sinks) {
    if (dtype > PK_FP16 || !good_chunk(kv, R, n_q, q_heads, page_stride, window, sinks)) return 0;
    const uint64_t need = pk_attend_chunk_scratch_bytes_impl(*kv, dtype, R, n_q, q_heads, page_stride,
                                                             window_within(*kv, page_stride, window), sinks);
    return need == UINT64_MAX ? 0 : (size_t)need;
}

int pk_attend_chunk(const pk_kv_cache *kv, uint32_t dtype, const pk_heads *q, const pk_heads *out, float *lse_dev,
                    uint64_t n_q, const int64_t *q_off_dev, uint32_t R, uint32_t q_heads, float scale, uint32_t window,
                    uint32_t sinks, const int32_t *kv_len_dev, const uint32_t *pages_dev, uint64_t page_stride,
                    void *scratch_dev, size_t scratch_bytes, int32_t *status_dev, pk_stream stream) {
    if (!good_cache(kv) || dtype > PK_FP16 || !good_score_scale((double)scale * kv->k_scale)) return PK_ERR_ARG;
    if (!good_chunk(kv, R, n_q, q_heads, page_stride, window, sinks)) return PK_ERR_ARG;
    if (!good_heads(q, n_q, q_heads) || !good_out(out, n_q, q_heads, kv->head_dim)) return PK_ERR_ARG;
    if (q->tok_stride >= (int64_t)1 << 39 || q->head_stride >= (int64_t)1 << 39) return PK_ERR_ARG;  // a tensor map's
    if (!aligned(lse_dev, 4) || !aligned(q_off_dev, 8) || !aligned(kv_len_dev, 4) || !aligned(pages_dev, 4) ||
        !aligned(scratch_dev, 32) || !aligned(status_dev, 4))
        return PK_ERR_ARG;
    if (R == 0 || n_q == 0) return PK_OK;
    if (!q_off_dev || !kv_len_dev || (page_stride && !pages_dev) || !scratch_dev) return PK_ERR_ARG;
    window = window_within(*kv, page_stride, window);
    const uint64_t need = pk_attend_chunk_scratch_bytes_impl(*kv, dtype, R, n_q, q_heads, page_stride, window, sinks);
    if (need == UINT64_MAX || scratch_bytes < need) return PK_ERR_ARG;
    return cuda_rc(pk_launch_attend_chunk(*kv, dtype, *q, *out, lse_dev, n_q, q_off_dev, R, q_heads, scale, window, sinks,
                                          kv_len_dev, pages_dev, page_stride, scratch_dev, status_dev,
                                          reinterpret_cast<cudaStream_t>(stream)));
}

static const double kTurn = 6.283185307179586476925286766559;  // 2 pi

static bool good_turns(uint32_t rotary_dim, double base, double factor, double context, double low, double high,
                       const uint64_t *turns) {
    return turns && rotary_dim >= 16 && rotary_dim <= 128 && rotary_dim % 16 == 0 && base > 1.0 && std::isfinite(base) &&
           factor >= 1.0 && std::isfinite(factor) && context >= 0.0 && std::isfinite(context) && low >= 0.0 && high > low &&
           std::isfinite(high);
}

// Part `stays` of f as it is, the rest divided.
static uint64_t turns_of(double f, double factor, double stays) {
    return (uint64_t)std::ldexp((stays * f + (1.0 - stays) * f / factor) / kTurn, 64);
}

int pk_rotary_turns(uint32_t rotary_dim, double base, double factor, double context, double low, double high,
                    uint64_t *turns) {
    if (!good_turns(rotary_dim, base, factor, context, low, high, turns)) return PK_ERR_ARG;
    for (uint32_t i = 0; i < rotary_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rotary_dim);
        double stays = 0.0;
        if (context > 0.0) stays = std::fmin(1.0, std::fmax(0.0, (context * f / kTurn - low) / (high - low)));
        turns[i] = turns_of(f, factor, stays);
    }
    return PK_OK;
}

int pk_rotary_turns_by_index(uint32_t rotary_dim, double base, double factor, double context, double low, double high,
                             uint64_t *turns) {
    if (!good_turns(rotary_dim, base, factor, context, low, high, turns) || context == 0.0 || low == 0.0) return PK_ERR_ARG;
    auto index = [&](double n) { return rotary_dim * std::log(context / (kTurn * n)) / (2.0 * std::log(base)); };
    const double first = std::fmax(std::floor(index(high)), 0.0), last = std::fmin(std::ceil(index(low)), rotary_dim - 1.0);
    if (last < first) return PK_ERR_ARG;
    for (uint32_t i = 0; i < rotary_dim / 2; ++i)
        turns[i] = turns_of(std::pow(base, -2.0 * i / rotary_dim), factor,
                            i <= first ? 1.0 : i >= last ? 0.0 : (last - i) / (last - first));
    return PK_OK;
}

int pk_rotate(uint32_t dtype, const pk_heads *q, const pk_heads *k, const pk_heads *q_out, const pk_heads *k_out,
              uint64_t n_tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, const pk_rotary *rotary,
              const void *q_weight_dev, const void *k_weight_dev, float eps, const int64_t *tok_off_dev,
              const int32_t *start_dev, uint32_t R, int32_t *status_dev, pk_stream stream) {
    if (dtype > PK_FP16 || (head_dim != 64 && head_dim != 128) || (uint64_t)q_heads + kv_heads > 65536) return PK_ERR_ARG;
    if (!rotary || rotary->rotary_dim < 16 || rotary->rotary_dim > head_dim || rotary->rotary_dim % 16 ||
        rotary->interleaved > 1 || !std::isfinite(rotary->amplitude) || !rotary->turns_dev ||
        !aligned(rotary->turns_dev, 16) || !std::isnormal(eps) || eps < 0.0f)
        return PK_ERR_ARG;
    if (n_tokens >= 1ull << 32) return PK_ERR_ARG;
    // heads of none: no rows to look at
    if (!good_heads(q, q_heads ? n_tokens : 0, q_heads) || !good_heads(k, kv_heads ? n_tokens : 0, kv_heads) ||
        !good_out(q_out, q_heads ? n_tokens : 0, q_heads, head_dim) ||
        !good_out(k_out, kv_heads ? n_tokens : 0, kv_heads, head_dim))
        return PK_ERR_ARG;
    if (!aligned(q_weight_dev, 16) || !aligned(k_weight_dev, 16) || !aligned(tok_off_dev, 8) || !aligned(start_dev, 4) ||
        !aligned(status_dev, 4))
        return PK_ERR_ARG;
    if (R == 0 || n_tokens == 0 || q_heads + kv_heads == 0) return PK_OK;
    if (!tok_off_dev || !start_dev) return PK_ERR_ARG;
    return cuda_rc(pk_launch_rotate(dtype, *q, *k, *q_out, *k_out, n_tokens, q_heads, kv_heads, head_dim, *rotary,
                                    q_weight_dev, k_weight_dev, eps, tok_off_dev, start_dev, R, status_dev,
                                    reinterpret_cast<cudaStream_t>(stream)));
}

int pk_evict_pages(const uint32_t *pages_dev, const float *weight_dev, const int32_t *kv_len_dev, uint32_t R,
                   uint64_t page_stride, uint32_t page_tokens, uint32_t budget, uint32_t sinks, uint32_t recent,
                   uint32_t *pages_out_dev, float *weight_out_dev, int32_t *kv_len_out_dev, uint32_t *evicted_dev,
                   int32_t *status_dev, pk_stream stream) {
    if (page_tokens == 0 || recent == 0 || (uint64_t)sinks + recent > budget || budget >= 1u << 31 ||
        page_stride >= 1ull << 31)
        return PK_ERR_ARG;
    for (const void *p : {(const void *)pages_dev, (const void *)weight_dev, (const void *)kv_len_dev,
                          (const void *)pages_out_dev, (const void *)weight_out_dev, (const void *)kv_len_out_dev,
                          (const void *)evicted_dev, (const void *)status_dev})
        if (!aligned(p, 4)) return PK_ERR_ARG;
    if (R == 0) return PK_OK;
    if (!kv_len_dev || !pages_out_dev || !weight_out_dev || !kv_len_out_dev ||
        (page_stride && (!pages_dev || !weight_dev)))
        return PK_ERR_ARG;
    return cuda_rc(pk_launch_evict_pages(pages_dev, weight_dev, kv_len_dev, R, page_stride, page_tokens, budget,
                                         sinks, recent, pages_out_dev, weight_out_dev, kv_len_out_dev, evicted_dev,
                                         status_dev, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
