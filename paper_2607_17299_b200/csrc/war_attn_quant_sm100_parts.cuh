// Parts of the two tensor-core kernels over the 8-bit cache (library-internal): copies, MMA and TMEM wrappers, bounded waits,
// kernel arguments, tensor maps.
#pragma once
#include "war_quant.cuh"
#include "war_attn_quant.cuh"
#include "war_attn_sm100_parts.cuh"

namespace {

struct QuantKernelArgs {
    const __nv_bfloat16* q;
    const int32_t* page_table;
    const int32_t* prefix_len;
    __nv_bfloat16* out;
    float* lse;
    int* status_word;
    AttnWorkspace w;
    AttnQuantPools pools;
    long long num_pages;
    float scale_log2;
    int N, Hq, Hkv, G, page_size, max_pages;
    int page_shift, block_shift, bpp_shift;
    uint32_t kv_e5m2;
    const int32_t* num_nodes;
    const int32_t* parent;
    int B;
    unsigned long long call;
};

// One (page, head) of a pool: tensor (d, token, head, page), 128 bytes x page_size.
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, int head, int page, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(head), "r"(page) : "memory");
}
__device__ __forceinline__ void tma_load_page_hint(uint32_t dst, const CUtensorMap* map, int head, int page, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %3, %4, %5}], [%2], %6;"
        ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(head), "r"(page), "l"(policy) : "memory");
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// arrives on the barrier once this thread's copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// kind::f8f6f4, fp32 accumulators, 128 x n x 32; type 0 = e4m3, 1 = e5m2 of A and of B
__device__ __forceinline__ uint32_t umma_idesc8(uint32_t n, uint32_t a_type, uint32_t b_type, uint32_t a_mn_major, uint32_t b_mn_major) {
    return (1u << 4) | (a_type << 7) | (b_type << 10) | (a_mn_major << 15) | (b_mn_major << 16) | ((n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// The bounded wait of war_sm100_prims.cuh in a dozen instructions (the main loops stand in the instruction cache, and a
// tile has eight waits): gives up after kWaitBudgetNs or when another waiter of the CTA has.
__device__ __forceinline__ uint32_t timer_lo() {
    uint32_t t;
    asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
    return t;
}
// mbarrier.try_wait with a time hint: the warp is suspended until the phase completes or about that time has passed.
__device__ __forceinline__ bool mbar_try_wait_long(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(1000000u) : "memory");
    return ok != 0;
}
template <class BarsT>
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, BarsT* bars, int* status_word) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint32_t t0 = timer_lo();
    while (!mbar_try_wait_long(bar, parity)) {
        if (*(volatile int*)&bars->abort_flag) return false;
        if (timer_lo() - t0 > (uint32_t)kWaitBudgetNs) {
            war_set_device_status(status_word, WAR_ERR_TIMEOUT);
            *(volatile int*)&bars->abort_flag = 1;
            return false;
        }
    }
    return true;
}

// One arrival for a whole warp: 32 lanes arriving on one barrier queue up behind each other.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void st_shared8(uint32_t at, uint32_t x, uint32_t y) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// the larger magnitude of two packed bf16, as bits
__device__ __forceinline__ uint32_t mag2(uint32_t w) { return max(w & 0x7fffu, (w >> 16) & 0x7fffu); }

// Four scaled weights (two pairs, each divided by 256) as high (e4m3) and low (e5m2) codes, four of each.  The pipe that
// holds the 8-bit conversions is the busiest but one here, so both codes are cut out of halves: a half of x / 256 holds in
// its bits 7 to 14 the e4m3 code of x (the two exponent biases differ by 8), rounded by adding half a step before the cut;
// the remainder is exact, and its e5m2 code is a half's upper byte, rounded the same way.  Together they hold x to 2^-7.8 of
// itself, or to 2^-13.8 where it is below 2^-6 (the high part's step is 2^-9 there, and the low part holds the rest to 2^-3).
__device__ __forceinline__ void split_weights(float2 x01, float2 x23, uint32_t& high, uint32_t& low) {
    asm("{\n.reg .b32 y0, y1, h0, h1, d0, d1, s0, s1;\n"
        "cvt.rn.f16x2.f32 y0, %3, %2;\n"
        "cvt.rn.f16x2.f32 y1, %5, %4;\n"
        "add.u32 h0, y0, 0x00400040;\n"
        "add.u32 h1, y1, 0x00400040;\n"
        "and.b32 h0, h0, 0x7f807f80;\n"
        "and.b32 h1, h1, 0x7f807f80;\n"
        "sub.rn.f16x2 d0, y0, h0;\n"
        "sub.rn.f16x2 d1, y1, h1;\n"
        "mul.rn.f16x2 d0, d0, %6;\n"
        "mul.rn.f16x2 d1, d1, %6;\n"
        "add.u32 s0, h0, h0;\n"
        "add.u32 s1, h1, h1;\n"
        "add.u32 d0, d0, 0x00800080;\n"
        "add.u32 d1, d1, 0x00800080;\n"
        "prmt.b32 %0, s0, s1, 0x7531;\n"
        "prmt.b32 %1, d0, d1, 0x7531;\n}\n"
        : "=r"(high), "=r"(low) : "f"(x01.x), "f"(x01.y), "f"(x23.x), "f"(x23.y), "r"(0x5c005c00u));
}

// from the scales of a group's first tile, one a lane
__device__ __forceinline__ float v_reference(float scale) {
    const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(scale));         // (not negative: ordered as integers)
    return top == 0 || top >= 0x21800000u ? kVRefLarge : kVRefSmall;                      // (2^-60)
}

// A pool as (d, token, head, page) with its own strides and a box of one (page, head).
bool make_pool_map(CUtensorMap* map, const void* pool, long long num_pages, int Hkv, int page_size, const long long* s) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    const cuuint64_t dims[4] = {128, (cuuint64_t)page_size, (cuuint64_t)Hkv, (cuuint64_t)num_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)s[2], (cuuint64_t)s[1], (cuuint64_t)s[0]};
    const cuuint32_t box[4] = {128, (cuuint32_t)page_size, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(pool), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// What both kernels are launched with; false: the pools have no tensor map.
inline bool quant_kernel_args(const void* q, const AttnQuantPools& pools, const int32_t* page_table, const int32_t* prefix_len,
                              const int32_t* num_nodes, const int32_t* parent, const war_attn_params_t* p, const AttnWorkspace& w,
                              bool fused, void* out, float* lse, int* status_word, QuantKernelArgs* a, CUtensorMap* k_map,
                              CUtensorMap* v_map) {
    if (!make_pool_map(k_map, pools.k, p->num_pages, p->Hkv, p->page_size, pools.ks) ||
        !make_pool_map(v_map, pools.v, p->num_pages, p->Hkv, p->page_size, pools.vs))
        return false;
    a->q = (const __nv_bfloat16*)q; a->page_table = page_table; a->prefix_len = prefix_len;
    a->out = (__nv_bfloat16*)out; a->lse = lse; a->status_word = status_word; a->w = w; a->pools = pools;
    a->num_pages = p->num_pages; a->scale_log2 = p->scale * kLog2e;
    a->N = p->N; a->Hq = p->Hq; a->Hkv = p->Hkv; a->G = p->Hq / p->Hkv; a->page_size = p->page_size; a->max_pages = p->max_pages_per_req;
    a->page_shift = log2_of(p->page_size); a->block_shift = log2_of(pools.block); a->bpp_shift = a->page_shift - a->block_shift;
    a->kv_e5m2 = pools.kv == kKvE5M2;
    a->num_nodes = num_nodes; a->parent = parent; a->B = p->B; a->call = fused ? war_attn_next_call() : 0;
    return true;
}

}  // namespace
