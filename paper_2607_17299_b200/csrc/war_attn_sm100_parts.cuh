// Parts of the tensor-core verify attention that do not depend on the cache's type: ancestor masks, the counting of split
// units' partial results and their merge, tensor maps (library-internal, device code).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>
#include "war_common.cuh"
#include "war_attn_plan.cuh"
#include "war_attn_fused_plan.cuh"
#include "war_sm100_prims.cuh"

// Number of a launch of the one-launch path, for the arrival counters below.
unsigned long long war_attn_next_call();

namespace {
using namespace sm100;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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

// Has the phase completed?  (mbarrier.try_wait may hold the thread for a while, test_wait never does.)
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}

// One arrival for a whole warp: 32 lanes arriving on one barrier queue up behind each other.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}

// What the three roles need to know about a unit, wherever the plan lives.
struct UnitView {
    int req, kvh, rb, tile_begin, tile_end, n_chunks, chunk, n_nodes;
    int slot;                            // index of this unit's partial in the workspace
    int slot_base, slot_stride, bump;    // fused-plan variant: partial of chunk c is slot_base + c * slot_stride (+ bump for c == 0)
    int page0, n_keys, visible, rows, slot0, part0, part_rows;      // shared-prefix variant: see SharedUnit (rows: end of the unit's rows)
};

// Ancestor-or-self bit masks of one tree, by one warp: lane l holds slots l and l + 32.  After round r a slot's mask
// covers its 2^r nearest ancestors-or-self and its pointer is the 2^r-th ancestor (the root points at itself).
// Returns the mask of slot j (any j < n per lane).  The tree has been validated (parent[s] in [0, s) for 0 < s < n).
__device__ __forceinline__ uint64_t shfl_u64(uint64_t v, int src) {
    const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)v, src);
    const uint32_t hi = __shfl_sync(0xffffffffu, (uint32_t)(v >> 32), src);
    return ((uint64_t)hi << 32) | lo;
}
// parent[s] must lie in [0, s) for every slot 0 < s < n (lane l holds the entries of slots l and l + 32)
__device__ __forceinline__ bool tree_is_malformed(int q0, int q1, int n, int lane) {
    const int j0 = lane, j1 = lane + 32;
    const bool bad = (j0 > 0 && j0 < n && (q0 < 0 || q0 >= j0)) || (j1 < n && (q1 < 0 || q1 >= j1));
    return __any_sync(0xffffffffu, bad);
}
__device__ __forceinline__ uint64_t warp_ancestor_mask(int q0, int q1, int n, int j, int lane) {
    const int j0 = lane, j1 = lane + 32;
    int p0 = (j0 > 0 && j0 < n) ? q0 : 0;
    int p1 = (j1 < n) ? q1 : 0;
    uint64_t a0 = 1ull << j0, a1 = 1ull << j1;
    // (rolled loops: this runs once per unit, from code that is usually not in the instruction cache)
    if (n <= 32) {
#pragma unroll 1
        for (int r = 0; r < 5; ++r) {
            const uint64_t b = shfl_u64(a0, p0);
            const int q = __shfl_sync(0xffffffffu, p0, p0);
            a0 |= b; p0 = q;
        }
    } else {
#pragma unroll 1
        for (int r = 0; r < 6; ++r) {
            const uint64_t b00 = shfl_u64(a0, p0 & 31), b01 = shfl_u64(a1, p0 & 31);
            const uint64_t b10 = shfl_u64(a0, p1 & 31), b11 = shfl_u64(a1, p1 & 31);
            const int q00 = __shfl_sync(0xffffffffu, p0, p0 & 31), q01 = __shfl_sync(0xffffffffu, p1, p0 & 31);
            const int q10 = __shfl_sync(0xffffffffu, p0, p1 & 31), q11 = __shfl_sync(0xffffffffu, p1, p1 & 31);
            a0 |= p0 >= 32 ? b01 : b00;
            a1 |= p1 >= 32 ? b11 : b10;
            p0 = p0 >= 32 ? q01 : q00;
            p1 = p1 >= 32 ? q11 : q10;
        }
    }
    const uint64_t m0 = shfl_u64(a0, j & 31), m1 = shfl_u64(a1, j & 31);
    return j >= 32 ? m1 : m0;
}

// Arrival counters of split (request, kv head, row block) triples (fused-plan variant).  A word holds
// (call number << 16) | arrivals (one per unit, at most kFusedMaxChunks).  The call number (48 bits, never 0, a new
// one for every launch made by this process) makes a word written by an earlier call, or never written at all, read
// as "no arrivals yet", so nothing has to be cleared before a launch; the CTA that merges a triple writes 0 back, so
// a captured launch (whose call number is frozen in the graph) can be replayed.  (A word that was never written
// equals the current call number by accident with probability 2^-48.)
__device__ __forceinline__ void count_arrival(unsigned long long* p, unsigned long long call) {
    const unsigned long long old = atomicAdd(p, 1ull);
    if ((old >> 16) == call) return;                         // the usual case after a triple's first arrival
    // The word was not this call's: the increment above went to a stale word and does not count.  Either make the
    // word this call's with one arrival, or, if somebody else has done so meanwhile, add this arrival to it.
    unsigned long long cur = old + 1ull;
    while (true) {
        if ((cur >> 16) == call) { atomicAdd(p, 1ull); return; }
        const unsigned long long prev = atomicCAS(p, cur, (call << 16) | 1ull);
        if (prev == cur) return;
        cur = prev;
    }
}
// The same count that also says how many of this call's arrivals there are now, this one included.
__device__ __noinline__ int count_arrival_ranked(unsigned long long* p, unsigned long long call) {
    const unsigned long long old = atomicAdd(p, 1ull);
    if ((old >> 16) == call) return (int)(old & 0xffffull) + 1;
    unsigned long long cur = old + 1ull;
    while (true) {
        if ((cur >> 16) == call) return (int)(atomicAdd(p, 1ull) & 0xffffull) + 1;
        const unsigned long long prev = atomicCAS(p, cur, (call << 16) | 1ull);
        if (prev == cur) return 1;
        cur = prev;
    }
}
// Bounded wait (one thread) until `target` arrivals of this call have been counted in p[0]; then the word is cleared.
// When `parts` CTAs merge the triple, each a share of its rows, every one of them waits here; they count themselves
// in *seen once they have seen the arrivals, and the last one to do so clears both words.
template <class BarsT>
__device__ __forceinline__ bool wait_arrivals(unsigned long long* p, unsigned long long* seen, unsigned long long call, int target, int parts, BarsT* bars, int* status_word) {
    auto there = [&]() -> bool {
        unsigned long long v;
        asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
        return (v >> 16) == call && (int)(v & 0xffffull) >= target;
    };
    if (!there()) {
        const unsigned long long t0 = global_timer_ns();
        unsigned spins = 0;
        while (!there()) {
            if ((++spins & 63u) == 0) {
                if (*(volatile int*)&bars->abort_flag) return false;
                if (global_timer_ns() - t0 > kWaitBudgetNs) {
                    war_set_device_status(status_word, WAR_ERR_TIMEOUT);
                    atomicExch(&bars->abort_flag, 1);
                    return false;
                }
            }
        }
    }
    __threadfence();
    if (parts > 1) {
        if (count_arrival_ranked(seen, call) < parts) return true;
        *(volatile unsigned long long*)seen = 0ull;
    }
    *(volatile unsigned long long*)p = 0ull;
    return true;
}

// Merge of the partial results of one split (request, kv head, row block) by the CTA that ran its chunk 0
// (fused-plan variant), once all units of the CTA are done and the ring and the Q tile are idle.  The eight softmax
// warps call it together.  Rows are taken in groups small enough that every chunk's rows of a group fit the ring at
// once: one thread issues a bulk copy per chunk for the partial outputs (ring) and one for the (max, sum) pairs (Q
// tile), everybody waits for the bytes, then every warp takes rows of the group, four at a time: row maximum over
// the chunks, then the chunks in chunk order with the arithmetic of attn_combine_kernel, so the bits do not depend
// on who merges.  Loops are rolled on purpose: this code runs once or twice per launch from a cold instruction cache.
// `phase` counts the groups this CTA has merged so far (the parity of both barriers).
struct MergeArgs {
    const float* part_o; const float* part_ml;
    __nv_bfloat16* out; float* lse; int* status_word;
    int rows, G, N, Hq;
    int req, kvh, rb, n_nodes, n_chunks, slot_base, slot_stride, bump;
    int part, parts, share;              // this CTA merges share `part` of `parts`: rows [part * share, + share), share even
    unsigned long long* arrivals; unsigned long long* seen; unsigned long long call;
};
template <int kRingBytes, class BarsT>
__device__ __noinline__ bool merge_partials(const MergeArgs m, uint8_t* ring, uint8_t* q_tile, BarsT* bars, uint32_t* phase_io) {
    const int tid = threadIdx.x, w8 = tid >> 5, lane = tid & 31;
    const int R = m.G * m.n_nodes;
    const int rows_valid = min(kRowBlock, R - m.rb * kRowBlock);
    const int nch = m.n_chunks;
    uint32_t phase = *phase_io;
    const int rows_g = min(kRowBlock, (kRingBytes / (nch * 512)) & ~1);     // even, >= 2 (nch <= kFusedMaxChunks)
    const float* s_o = (const float*)ring;
    const float2* s_ml = (const float2*)q_tile;
    int r_lo = 0, r_hi = rows_valid;
    if (m.parts > 1) {
        r_lo = m.part * m.share; r_hi = min(rows_valid, r_lo + m.share);
        if (r_lo >= r_hi) {                   // nothing falls to this share; it still takes part in clearing the counter
            if (tid == 0 && !wait_arrivals(m.arrivals, m.seen, m.call, nch, m.parts, bars, m.status_word)) return false;
            return true;
        }
    }
    for (int row0 = r_lo; row0 < r_hi; row0 += rows_g, ++phase) {
        const int rg = min(rows_g, (r_hi - row0 + 1) & ~1);                           // rows copied (even; the workspace has them)
        if (tid == 0) {
            // every chunk has left its partial
            if (row0 == r_lo && !wait_arrivals(m.arrivals, m.seen, m.call, nch, m.parts, bars, m.status_word)) { *phase_io = phase; return false; }
            // the previous group's readers are done with the buffers
            if (phase > 0 && !mbar_wait(&bars->merge_free, (phase - 1) & 1u, bars, m.status_word)) { *phase_io = phase; return false; }
            mbar_arrive_expect_tx(&bars->merge_full, (uint32_t)(nch * rg * (512 + 8)));
            for (int c = 0; c < nch; ++c) {
                const size_t slot = (size_t)(m.slot_base + c * m.slot_stride + (c == 0 ? m.bump : 0));
                const size_t at = slot * m.rows + row0;
                bulk_load(smem_u32(s_o + (size_t)c * rg * 128), m.part_o + at * 128, (uint32_t)rg * 512u, &bars->merge_full);
                bulk_load(smem_u32(s_ml + (size_t)c * rg), m.part_ml + at * 2, (uint32_t)rg * 8u, &bars->merge_full);
            }
        }
        if (!mbar_wait(&bars->merge_full, phase & 1u, bars, m.status_word)) { *phase_io = phase; return false; }
        // a warp takes four rows at a time, eight lanes per row, each lane four float4 of the row (columns 4*sub + 32*k):
        // sixteen independent accumulators per lane, and a load instruction reads four whole 128-byte segments
        const int sub = lane & 7;
        for (int rbase = w8 * 4; rbase < rg; rbase += 32) {
            const int r = rbase + (lane >> 3);
            const bool live = r < rg && row0 + r < r_hi;
            const int rr = live ? r : 0;
            float M = -CUDART_INF_F;
#pragma unroll 1
            for (int c = 0; c < nch; ++c) M = fmaxf(M, s_ml[c * rg + rr].x);
            float l = 0.f;
            float4 acc[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int c = 0; c < nch; ++c) {
                const float2 ml = s_ml[c * rg + rr];
                const float4* src = reinterpret_cast<const float4*>(s_o + ((size_t)c * rg + rr) * 128) + sub;
                const float sc = ml.x == -CUDART_INF_F ? 0.f : exp2f(ml.x - M);
                l = fmaf(ml.y, sc, l);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float4 o = src[8 * k];
                    acc[k].x = fmaf(o.x, sc, acc[k].x); acc[k].y = fmaf(o.y, sc, acc[k].y);
                    acc[k].z = fmaf(o.z, sc, acc[k].z); acc[k].w = fmaf(o.w, sc, acc[k].w);
                }
            }
            if (live) {
                const int gr = m.rb * kRowBlock + row0 + r;
                const int j = gr / m.G, g = gr - j * m.G;
                const size_t row = ((size_t)m.req * m.N + j) * m.Hq + m.kvh * m.G + g;
                const float inv = 1.f / l;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 h0 = __floats2bfloat162_rn(acc[k].x * inv, acc[k].y * inv), h1 = __floats2bfloat162_rn(acc[k].z * inv, acc[k].w * inv);
                    uint2 packed;
                    packed.x = *reinterpret_cast<const uint32_t*>(&h0);
                    packed.y = *reinterpret_cast<const uint32_t*>(&h1);
                    *reinterpret_cast<uint2*>(m.out + row * 128 + (sub + 8 * k) * 4) = packed;
                }
                if (m.lse && sub == 0) m.lse[row] = (M + log2f(l)) * kLn2;
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->merge_free);
    }
    *phase_io = phase;
    return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
            qres != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return nullptr;
        }
        fn = (EncodeTiledFn)p;
    }
    return fn;
}

// A head-major pool [num_pages, Hkv, page_size, 128] bf16 seen as blocks of (page, head): [blocks][token/8][d/64][token%8][d%64].
// A token-major pool (page, token, head, d) seen as (d, token, head, page) with a box of 64 dims x all tokens of one head.
bool make_pool_map(CUtensorMap* map, const void* pool, long long num_pages, int Hkv, int page_size, int token_major) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    if (token_major) {
        const cuuint64_t dims[4] = {128, (cuuint64_t)page_size, (cuuint64_t)Hkv, (cuuint64_t)num_pages};
        const cuuint64_t strides[3] = {(cuuint64_t)Hkv * 256, 256, (cuuint64_t)page_size * Hkv * 256};
        const cuuint32_t box[4] = {64, (cuuint32_t)page_size, 1, 1};
        return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    const cuuint64_t dims[5] = {64, 8, 2, (cuuint64_t)(page_size / 8), (cuuint64_t)(num_pages * Hkv)};
    const cuuint64_t strides[4] = {256, 128, 2048, (cuuint64_t)page_size * 256};
    const cuuint32_t box[5] = {64, 8, 2, (cuuint32_t)(page_size / 8), 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(pool), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
