// The 8-bit cache as the attention kernels see it (library-internal).
#pragma once
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
