// The 8-bit cache as the attention kernels see it (library-internal).
#pragma once
#include <math_constants.h>
#include "war_attn_plan.cuh"

struct AttnQuantPools {
    const uint8_t *k, *v;                 // codes, [page, head, token, 128] by strides
    const float *kscale, *vscale;         // [page, head, page_size / block]
    long long ks[3], vs[3];               // strides (page, head, token) in bytes
    int kv, block;                        // type of the codes, tokens per scale
};

// The tensor-core kernels: up to kQuantFewRows query rows per kv head, and more.  fused: one launch, the kernel plans for
// itself and merges split units itself.
constexpr int kQuantFewRows = 32;
war_status_t war_attn_quant_launch_few(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
                                       const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* parent,
                                       const war_attn_params_t* p, const AttnWorkspace& w, bool fused,
                                       void* out, float* lse, int* status_word, cudaStream_t s);
war_status_t war_attn_quant_launch_many(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
                                        const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* parent,
                                        const war_attn_params_t* p, const AttnWorkspace& w, bool fused,
                                        void* out, float* lse, int* status_word, cudaStream_t s);

#ifdef __CUDACC__
// What a row's weights are relative to.  The tensor cores get p * (V's scale), p = exp2(x - m), and what these lose is relative
// to the largest that the row's reference m has to allow for.  So m follows the largest x + lv of the keys that the row sees,
// lv = log2(V's scale / v_ref), not the largest x: a key of little weight, or one that the row does not see, takes no
// precision from the others however large its scale is.  The sum of the p goes by the same m and needs them as 32-bit numbers (2^-126 to
// 2^128), which bounds lv: v_ref = 2^25 leaves room for scales from 2^-60 to 2^125 next to each other (the store's are at
// most 2^120), and a unit that begins with a tile of smaller ones takes 2^-35, for 2^-120 to 2^65.
constexpr float kLeastLv = -85.f;
constexpr float kVRefLarge = 33554432.f, kVRefSmall = 2.9103830456733704e-11f;
__device__ __forceinline__ float v_relative(float scale, float v_ref) { return fminf(scale, v_ref * 0x1p100f) * (1.f / v_ref); }
__device__ __forceinline__ float v_log(float relative) { return fmaxf(__log2f(relative), kLeastLv); }
// A sum whose reference grows by 2^d, given 2^(-d / 2): d may be 185 (from the least lv to the most), where 2^-d is no 32-bit number
// any more but the sum of p up to 2^88 times that is.
__device__ __forceinline__ float half_step(float sum, float root) { return sum * root * root; }
// A group's (reference, sum) with the sum between 1 and 2: such references are logarithms of sums and can be compared between
// groups and parts, whatever scales they were worked out with.  Returns the power of two that the sum was multiplied by.
__device__ __forceinline__ float normal_sum(float& m, float& sum) {
    if (!(sum > 0.f && sum < CUDART_INF_F)) return 1.f;                                   // no keys, or a row that is NaN
    const int e = min(max((int)(__float_as_uint(sum) >> 23), 1), 253) - 127;
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    m += (float)e;
    sum *= down;
    return down;
}
#endif
