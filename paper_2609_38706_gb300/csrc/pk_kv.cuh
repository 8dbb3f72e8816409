// pk_kv.cuh -- the 4-bit page format (pk.h) on the device: granule offsets and
// the conversions between 16-bit values, e2m1 codes and e4m3 scales.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace pk {

constexpr uint32_t kGranTokens = 16;

// Byte offsets inside a granule (16 tokens of one KV head).
template <int D>
struct Granule {
    static constexpr uint32_t kRow = D / 2;     // code bytes of a token
    static constexpr uint32_t kScales = D / 16; // scale bytes of a token
    static constexpr uint32_t kK = 0;
    static constexpr uint32_t kV = kGranTokens * kRow;
    static constexpr uint32_t kKs = 2 * kGranTokens * kRow;
    static constexpr uint32_t kVs = kKs + kGranTokens * kScales;
    static constexpr uint32_t kBytes = kVs + kGranTokens * kScales;  // 2304 (D = 128), 1152 (D = 64)
};

// A block's 32 bytes, in one access where they start on a 32-byte boundary (two
// halves of a sector by separate instructions cost the L2 two requests: reading
// 64 x 2048 tokens back 119 -> 93 us).
__device__ __forceinline__ void load32(const uint16_t *p, bool wide, uint4 (&v)[2]) {
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y),
                       "=r"(v[1].z), "=r"(v[1].w)
                     : "l"(p)
                     : "memory");
    } else {
        v[0] = __ldcg(reinterpret_cast<const uint4 *>(p));
        v[1] = __ldcg(reinterpret_cast<const uint4 *>(p) + 1);
    }
}
__device__ __forceinline__ void store32(uint16_t *p, bool wide, const uint32_t (&w)[8]) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// Two e2m1 codes from two floats, to nearest even, saturating; lo in bits 0-3.
__device__ __forceinline__ uint32_t e2m1_pair(float lo, float hi) {
    uint32_t r;
    asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n cvt.u32.u8 %0, t;\n}" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// e4m3 byte of x >= 0, to nearest even, saturating at 448.
__device__ __forceinline__ uint32_t e4m3_byte(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
    return r & 0xff;
}

// Two e4m3 bytes as two halves (exact); byte 0 in the low half.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t two_bytes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two_bytes));
    return r;
}

__device__ __forceinline__ float e4m3_to_float(uint32_t byte) {
    const uint32_t h = e4m3_to_half2(byte & 0xff);
    return __low2float(*reinterpret_cast<const __half2 *>(&h));
}

// The four code pairs of a 32-bit word as halves (exact).
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// 16-bit types by pk.h's dtype numbers.
template <uint32_t DT>
struct Elem;
template <>
struct Elem<PK_BF16> {
    static constexpr uint32_t kInfBits = 0x7f80;
    static __device__ __forceinline__ float2 to2(uint32_t w) {
        return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w));
    }
    static __device__ __forceinline__ uint32_t from2(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ float to1(uint16_t h) {
        return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(&h));
    }
};
template <>
struct Elem<PK_FP16> {
    static constexpr uint32_t kInfBits = 0x7c00;
    static __device__ __forceinline__ float2 to2(uint32_t w) {
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    }
    static __device__ __forceinline__ uint32_t from2(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ float to1(uint16_t h) {
        return __half2float(*reinterpret_cast<const __half *>(&h));
    }
};

}  // namespace pk
