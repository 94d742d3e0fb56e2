// The 8-bit cache shared by the store, commit and attention kernels (library-internal).
//
// A pool holds 8-bit floats (e4m3 or e5m2), [num_pages, Hkv, page_size, 128] by strides, and next to it one float32
// scale per block of `scale_block` tokens and head: value = code * scale[page, head, (token in page) / scale_block].
// The store chooses powers of two: an 8-bit float keeps its relative precision at any scale, so nothing is lost
// against a scale that maps the largest value onto the largest code, dividing by the scale is exact, and re-encoding
// a row for a larger scale is exact too unless it falls below the type's smallest normal number.
#pragma once
#include <stdint.h>
#include "war.h"

constexpr int kKvBf16 = 0, kKvE4M3 = 1, kKvE5M2 = 2;
constexpr float kSmallestScale = 7.8886090522101181e-31f;      // 2^-100: its reciprocal is a normal number

#ifdef __CUDACC__
namespace quant {

// The smallest power of two s with a <= most * s, at least kSmallestScale; 0 for a = 0.  a >= 0; infinity counts as the
// largest finite number.  Both types' largest value is 1.75 * 2^k (k = 8 or 15), so only a's exponent and the comparison
// of its fraction with 0.75 matter: exact.
__device__ __forceinline__ float pow2_scale(float a, int kv) {
    if (!(a > 0.f)) return 0.f;
    const uint32_t u = min(__float_as_uint(a), 0x7f7fffffu);
    const int e = (int)(u >> 23) - (kv == kKvE4M3 ? 8 : 15) + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased exponent of s
    return fmaxf(__uint_as_float((uint32_t)max(e, 1) << 23), kSmallestScale);
}

// two floats to two codes (round to nearest even, beyond the range to the largest value; NaN stays NaN): lo in bits 0-7
__device__ __forceinline__ uint32_t encode2(float lo, float hi, int kv) {
    uint16_t r;
    if (kv == kKvE4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// two codes (bits 0-7 and 8-15) as half2 bits: every value of both types is a half
__device__ __forceinline__ uint32_t decode2_half(uint32_t codes, int kv) {
    uint32_t r;
    const uint16_t c = (uint16_t)codes;
    if (kv == kKvE4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
    else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"(c));
    return r;
}
__device__ __forceinline__ float2 decode2(uint32_t codes, int kv) {
    const uint32_t h = decode2_half(codes, kv);
    float2 f;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}\n" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
// eight codes re-encoded for another scale
__device__ __forceinline__ uint2 recode8(uint2 c, float ratio, int kv) {
    uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = decode2(w[i] & 0xffffu, kv), b = decode2(w[i] >> 16, kv);
        w[i] = encode2(a.x * ratio, a.y * ratio, kv) | (encode2(b.x * ratio, b.y * ratio, kv) << 16);
    }
    return make_uint2(w[0], w[1]);
}

}  // namespace quant
#endif

// Host-side checks of the 8-bit cache's description, shared by the entry points.
inline bool war_quant_block_ok(int page_size, int block) {
    return (block == 8 || block == 16 || block == 32 || block == 64 || block == 128) && page_size >= block && page_size % block == 0;
}
// Strides in elements: rows of 128 contiguous elements that start on 16-byte boundaries.
inline bool war_rows_aligned(const int64_t* s, int element_bytes) {
    if (s[3] != 1) return false;
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (s[i] * element_bytes) % 16 != 0) return false;
    return true;
}
