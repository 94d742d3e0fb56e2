// Verify attention over the 8-bit cache: argument checks, the choice of the path and the plain CUDA-core kernel (kept as
// the A/B reference of the tensor-core kernels in war_verify_attn_quant_few.cu and _many.cu).  The plan, the split of a request
// over thread blocks and the merge of its parts are those of the bf16 cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include "war_common.cuh"
#include "war_quant.cuh"
#include "war_attn_quant.cuh"
#include "war_attn_fused_plan.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;
constexpr int kSub = 16;

// One thread per query row; K and V codes are staged as halves (every code is one), their scales beside them, and V's
// logarithms (see war_attn_quant.cuh).
__global__ void __launch_bounds__(128)
attn_quant_simple_kernel(const __nv_bfloat16* __restrict__ q, const AttnQuantPools pools, const int32_t* __restrict__ page_table,
                         const int32_t* __restrict__ prefix_len, int N, int Hq, int Hkv, int G, int page_size, int max_pages,
                         long long num_pages, float scale_log2, AttnWorkspace w, __nv_bfloat16* __restrict__ out,
                         float* __restrict__ lse, int* status_word) {
    __shared__ __align__(16) uint32_t sK[kTile][64];
    __shared__ __align__(16) uint32_t sV[kTile][64];
    __shared__ float s_scale[2][kTile], s_lv[kTile];
    __shared__ int s_unit;
    const int tid = threadIdx.x;
    while (true) {
        __syncthreads();
        if (tid == 0) s_unit = atomicAdd(&w.counters[0], 1);
        __syncthreads();
        const int u = s_unit;
        if (u >= w.counters[1]) break;
        const AttnUnit un = w.units[u];
        const int i = un.req;
        const int n = w.req[i].n_nodes;
        const int R = G * n;
        const int pl = prefix_len[i];
        const int L = pl + n;
        const int r = un.rb * kRowBlock + tid;
        const bool active = r < R;
        const int j = active ? r / G : 0, g = active ? r % G : 0;
        const size_t qrow = ((size_t)i * N + j) * Hq + un.kvh * G + g;
        __nv_bfloat162 qv[64];
        {
            const uint4* src = reinterpret_cast<const uint4*>(q + qrow * 128);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                uint4 x = active ? src[c] : make_uint4(0, 0, 0, 0);
                qv[4 * c + 0] = *reinterpret_cast<__nv_bfloat162*>(&x.x);
                qv[4 * c + 1] = *reinterpret_cast<__nv_bfloat162*>(&x.y);
                qv[4 * c + 2] = *reinterpret_cast<__nv_bfloat162*>(&x.z);
                qv[4 * c + 3] = *reinterpret_cast<__nv_bfloat162*>(&x.w);
            }
        }
        const uint64_t anc = active ? w.anc[(size_t)i * N + j] : 0ull;
        float m = -CUDART_INF_F, l = 0.f;
        float acc[128];
#pragma unroll
        for (int d = 0; d < 128; ++d) acc[d] = 0.f;
        const int k_begin = un.tile_begin * kTileKeys;
        const int k_end = min(un.tile_end * kTileKeys, L);
        for (int kt = k_begin; kt < k_end; kt += kTile) {
            __syncthreads();
            for (int x = tid; x < kTile * 16 * 2; x += 128) {           // 8 codes a piece, 16 pieces a row
                const int which = x / (kTile * 16), y = x % (kTile * 16);
                const int row = y / 16, piece = y % 16;
                const int pos = kt + row;
                uint2 val = make_uint2(0, 0);
                float sc = 0.f;
                if (pos < k_end) {
                    long long page = page_table[(size_t)i * max_pages + pos / page_size];
                    if (page < 0 || page >= num_pages) { war_set_device_status(status_word, WAR_ERR_BAD_PAGE); page = 0; }
                    const long long* st = which ? pools.vs : pools.ks;
                    const uint8_t* pool = which ? pools.v : pools.k;
                    const int in_page = pos % page_size;
                    val = *reinterpret_cast<const uint2*>(pool + page * st[0] + un.kvh * st[1] + (long long)in_page * st[2] + piece * 8);
                    sc = (which ? pools.vscale : pools.kscale)[(page * Hkv + un.kvh) * (page_size / pools.block) + in_page / pools.block];
                }
                uint32_t* dst = &(which ? sV : sK)[row][piece * 4];
                dst[0] = quant::decode2_half(val.x & 0xffffu, pools.kv); dst[1] = quant::decode2_half(val.x >> 16, pools.kv);
                dst[2] = quant::decode2_half(val.y & 0xffffu, pools.kv); dst[3] = quant::decode2_half(val.y >> 16, pools.kv);
                if (piece == 0) {
                    s_scale[which][row] = sc;
                    if (which) s_lv[row] = v_log(v_relative(sc, kVRefLarge));
                }
            }
            __syncthreads();
            if (!active) continue;
            for (int sub = 0; sub < kTile; sub += kSub) {
                float s[kSub];
                float tmax = -CUDART_INF_F;
#pragma unroll
                for (int kk = 0; kk < kSub; ++kk) {
                    const int pos = kt + sub + kk;
                    const __half2* krow = reinterpret_cast<const __half2*>(&sK[sub + kk][0]);
                    float a = 0.f;
#pragma unroll
                    for (int d = 0; d < 64; ++d) {
                        const float2 kf = __half22float2(krow[d]);
                        const float2 qf = __bfloat1622float2(qv[d]);
                        a = fmaf(qf.x, kf.x, a);
                        a = fmaf(qf.y, kf.y, a);
                    }
                    const bool vis = pos < pl || (pos < k_end && ((anc >> (pos - pl)) & 1ull));
                    s[kk] = vis ? a * s_scale[0][sub + kk] * scale_log2 : -CUDART_INF_F;
                    tmax = fmaxf(tmax, s[kk] + s_lv[sub + kk]);
                }
                if (tmax == -CUDART_INF_F) continue;
                const float m_new = fmaxf(m, tmax);
                const float corr = exp2f(0.5f * (m - m_new));
                l = half_step(l, corr);
#pragma unroll
                for (int d = 0; d < 128; ++d) acc[d] = half_step(acc[d], corr);
                m = m_new;
#pragma unroll
                for (int kk = 0; kk < kSub; ++kk) {
                    const float p = exp2f(s[kk] - m);
                    l += p;
                    const float pv = p * s_scale[1][sub + kk];
                    const __half2* vrow = reinterpret_cast<const __half2*>(&sV[sub + kk][0]);
#pragma unroll
                    for (int d = 0; d < 64; ++d) {
                        const float2 vf = __half22float2(vrow[d]);
                        acc[2 * d] = fmaf(pv, vf.x, acc[2 * d]);
                        acc[2 * d + 1] = fmaf(pv, vf.y, acc[2 * d + 1]);
                    }
                }
            }
        }
        if (active) {
            const float down = normal_sum(m, l);
            if (un.n_chunks == 1) {
                const float inv = down / l;
                __nv_bfloat162* dst = reinterpret_cast<__nv_bfloat162*>(out + qrow * 128);
#pragma unroll
                for (int d = 0; d < 64; ++d) dst[d] = __floats2bfloat162_rn(acc[2 * d] * inv, acc[2 * d + 1] * inv);
                if (lse) lse[qrow] = (m + log2f(l)) * kLn2;
            } else {
                float* po = w.part_o + ((size_t)u * w.rows + tid) * 128;
#pragma unroll
                for (int d = 0; d < 128; ++d) po[d] = acc[d] * down;
                w.part_ml[((size_t)u * w.rows + tid) * 2] = m;
                w.part_ml[((size_t)u * w.rows + tid) * 2 + 1] = l;
            }
        }
    }
}

war_status_t check_params(const war_attn_quant_params_t* q) {
    if (!q) return WAR_ERR_INVALID_ARG;
    const war_attn_params_t* p = &q->attn;
    if (p->B < 0 || p->N < 1 || p->N > 64 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->max_pages_per_req < 0 ||
        p->num_pages < 0 || p->kernel < 0 || p->kernel > 2 || !(p->scale > 0.f) || (q->kv_type != kKvE4M3 && q->kv_type != kKvE5M2))
        return WAR_ERR_INVALID_ARG;
    if (p->D != 128 || (p->page_size != 8 && p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128))
        return WAR_ERR_UNSUPPORTED;
    if (!war_quant_block_ok(p->page_size, q->scale_block)) return WAR_ERR_UNSUPPORTED;
    if ((p->Hq / p->Hkv) * p->N > 512 || p->B > kMaxPlanB || (long long)p->B * p->N * p->Hq >= (1ll << 31)) return WAR_ERR_UNSUPPORTED;
    if ((long long)p->max_pages_per_req * p->page_size >= (1ll << 30)) return WAR_ERR_UNSUPPORTED;    // contexts below 2^30 tokens
    if (!war_rows_aligned(p->k_strides, 1) || !war_rows_aligned(p->v_strides, 1)) return WAR_ERR_UNSUPPORTED;
    return WAR_OK;
}

}  // namespace

extern "C" size_t war_verify_attn_quant_workspace_bytes(const war_attn_quant_params_t* q) {
    if (check_params(q) != WAR_OK) return 0;
    return war_attn_workspace_layout(&q->attn, nullptr).bytes;
}

extern "C" war_status_t war_verify_attn_quant(const void* d_q, const void* d_kpool, const void* d_vpool, const float* d_kscale,
                                              const float* d_vscale, const int32_t* d_page_table, const int32_t* d_prefix_len,
                                              const int32_t* d_num_nodes, const int32_t* d_parent, const war_attn_quant_params_t* qp,
                                              void* d_workspace, void* d_out, float* d_lse, war_stream_t stream) {
    war_status_t st = check_params(qp);
    if (st != WAR_OK) return st;
    const war_attn_params_t* p = &qp->attn;
    if (p->B == 0) return WAR_OK;
    if (!d_q || !d_kpool || !d_vpool || !d_kscale || !d_vscale || !d_page_table || !d_prefix_len || !d_num_nodes || !d_parent ||
        !d_workspace || !d_out || p->num_pages == 0)
        return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_q | (uintptr_t)d_out | (uintptr_t)d_kpool | (uintptr_t)d_vpool) & 15))
        return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    const AttnWorkspace w = war_attn_workspace_layout(p, d_workspace);
    const int n_sm = war_attn_sm_count();
    if (n_sm <= 0) return WAR_ERR_CUDA;
    AttnQuantPools pools;
    pools.k = (const uint8_t*)d_kpool; pools.v = (const uint8_t*)d_vpool; pools.kscale = d_kscale; pools.vscale = d_vscale;
    for (int i = 0; i < 3; ++i) { pools.ks[i] = p->k_strides[i]; pools.vs[i] = p->v_strides[i]; }
    pools.kv = qp->kv_type; pools.block = qp->scale_block;
    const auto launch = p->Hq / p->Hkv * p->N <= kQuantFewRows ? war_attn_quant_launch_few : war_attn_quant_launch_many;
    if (p->kernel == 0 && war_attn_fused_ok(p, w.row_blocks, n_sm))
        return launch(d_q, pools, d_page_table, d_prefix_len, d_num_nodes, d_parent, p, w, true, d_out, d_lse,
                                           status_word, stream);
    st = war_attn_launch_plan(d_prefix_len, d_num_nodes, d_parent, p, w, n_sm, status_word, stream);
    if (st != WAR_OK) return st;
    if (p->kernel == 1) {
        const int G = p->Hq / p->Hkv;
        attn_quant_simple_kernel<<<n_sm * 4, 128, 0, stream>>>((const __nv_bfloat16*)d_q, pools, d_page_table, d_prefix_len, p->N, p->Hq,
                                                              p->Hkv, G, p->page_size, p->max_pages_per_req, (long long)p->num_pages,
                                                              p->scale * kLog2e, w, (__nv_bfloat16*)d_out, d_lse, status_word);
        WAR_LAUNCH_CHECK();
    } else {
        st = launch(d_q, pools, d_page_table, d_prefix_len, d_num_nodes, d_parent, p, w, false, d_out, d_lse,
                                         status_word, stream);
        if (st != WAR_OK) return st;
    }
    return war_attn_launch_combine(p, w, d_out, d_lse, stream);
}
