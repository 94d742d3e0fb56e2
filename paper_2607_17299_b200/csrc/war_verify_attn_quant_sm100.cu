// Tensor-core verify attention over the 8-bit cache for sm_100a.  The skeleton is that of war_verify_attn_sm100.cu (work
// units, warp roles, a ring of TMA-filled slots, two softmax groups with an accumulator each, one launch for up to 64
// requests); what differs is the arithmetic, because the cache's bytes go to the tensor cores as they are:
//
//   S = Qh K' + Ql K'      q (scaled by a power of two per row) = Qh + Ql, both e4m3: eight kind::f8f6f4 products of 32 dims
//   p = exp2(S * (row's constant * K's scale of the key's block) - m)
//   O += Ph V' + Pl V'     p * (V's scale of the key's block) = Ph + Pl, e4m3 and e5m2: eight products of 32 keys
//
// Converting the cache to 16 bits on chip instead would move every element through shared memory three more times (read,
// written twice as wide, read twice as wide by the tensor cores), 192 of the 128 bytes an SM moves a cycle; splitting the
// small operands keeps the tensor work of the bf16 kernel per key (sixteen products of 64 cycles a tile) and its precision.
// A tile of 128 keys is 16 KB of K and 16 KB of V, rows of 128 bytes in the 128-byte swizzle, for either memory order: one
// tensor map (d, token, head, page) with the pool's own strides, one copy per (page, head).
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>
#include <mutex>
#include "war_common.cuh"
#include "war_quant.cuh"
#include "war_attn_quant.cuh"
#include "war_attn_sm100_parts.cuh"

namespace {

constexpr int kSlots = 11;
constexpr int kSlotBytes = 16384;
constexpr int kThreads = 384;                      // three warpgroups: softmax 0, softmax 1, {producer, MMA, signaller, spare}
constexpr int kRegsSoftmax = 224;
constexpr int kRegsOther = 48;
constexpr uint32_t kTmemCols = 512;
// The largest scaled weight is 2^kRescaleThreshold (a stale maximum) * 2 (V's scale against its reference) * kWeightTop = 448,
// the largest e4m3 value.
constexpr float kRescaleThreshold = 2.0f;          // log2 units
constexpr float kWeightTop = 56.f;
constexpr float kTinyScale = 1.1754943508222875e-38f;   // a scale of 0 must not turn a masked -inf into NaN

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int kOffQ = 0;                            // high parts, then low parts
constexpr int kOffRing = 32768;
constexpr int kOffBar = kOffRing + kSlots * kSlotBytes;
constexpr int kOffStats = kOffBar + 512;
constexpr int kOffFused = kOffStats + 1536;
constexpr int kSmemBytes = kOffFused + 768 + 1024;
constexpr int kMaxChunks = kSlots * kSlotBytes / 1024;    // the merge needs two rows of every chunk in the ring
static_assert(sizeof(FusedPlan) <= 768, "plan table of the fused-plan variant");
static_assert(kSmemBytes <= 232448, "shared memory");
static_assert(sizeof(FusedPlanScratch) <= kSlots * kSlotBytes, "the plan scratch lives in the idle ring");
static_assert(kThreads == kFusedThreads, "fused_plan::make is written for the attention kernel's block size");
static_assert(kThreads * 168 >= 256 * kRegsSoftmax + 128 * kRegsOther, "the hand-over draws on the registers of the launch");

struct Bars {
    uint64_t full[kSlots], empty[kSlots];
    uint64_t s_ready[2], p_ready[2], pv_done[2];
    uint64_t q_ready, stats_ready, epi_done;
    uint64_t part_out, merge_full, merge_free;
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// Ring sequence numbers as in the bf16 kernel: K0, K1, V0, K2, V1, ..., K(T-1), V(T-2), V(T-1).
__device__ __forceinline__ uint32_t seq_k(uint32_t ld0, int t) { return t == 0 ? ld0 : ld0 + 2u * t - 1u; }
__device__ __forceinline__ uint32_t seq_v(uint32_t ld0, int t, int T) { return t == T - 1 ? ld0 + 2u * T - 1u : ld0 + 2u * t + 2u; }

struct KernelArgs {
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
    int page_shift, block_shift, bpp_shift, kv_e5m2;
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

// kind::f8f6f4, fp32 accumulators, 128 x 128 x 32; type 0 = e4m3, 1 = e5m2 of A and of B
__device__ __forceinline__ uint32_t umma_idesc8(uint32_t a_type, uint32_t b_type, uint32_t b_mn_major) {
    return (1u << 4) | (a_type << 7) | (b_type << 10) | (b_mn_major << 16) | (16u << 17) | (8u << 24);
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_f8_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// the larger magnitude of two packed bf16, as bits
__device__ __forceinline__ uint32_t mag2(uint32_t w) { return max(w & 0x7fffu, (w >> 16) & 0x7fffu); }

// Two weights as high (e4m3) and low (e5m2) parts, two codes each.  Through halves: 11 bits hold what 4 + 3 bits and the
// sign of the remainder can, and the remainder is exact in them.
__device__ __forceinline__ void split_weights(float2 x, uint32_t& high, uint32_t& low) {
    uint16_t h, l;
    asm("{\n.reg .b32 x, b, d;\n"
        "cvt.rn.f16x2.f32 x, %3, %2;\n"
        "cvt.rn.satfinite.e4m3x2.f16x2 %0, x;\n"
        "cvt.rn.f16x2.e4m3x2 b, %0;\n"
        "sub.rn.f16x2 d, x, b;\n"
        "cvt.rn.satfinite.e5m2x2.f16x2 %1, d;\n}\n"
        : "=h"(h), "=h"(l) : "f"(x.x), "f"(x.y));
    high = h; low = l;
}

// kFused: see attn_sm100_kernel.
template <bool kFused>
__global__ void __launch_bounds__(kThreads, 1)
attn_quant_sm100_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const KernelArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars* bars = (Bars*)(smem + kOffBar);
    float* stats = (float*)(smem + kOffStats);       // group 1's max, sum and weight of its O per row, for the merge
    const FusedPlan* plan = (const FusedPlan*)(smem + kOffFused);
    const uint32_t sQ = smem_u32(smem + kOffQ), sRing = smem_u32(smem + kOffRing);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int n_units = 0, list_first = 0, list_end = 0;
    bool contiguous = false;
    if (!kFused) {
        n_units = a.w.counters[1];
        // k-th unit of this CTA: its own contiguous list, or the snake deal of the longest-first list
        contiguous = a.w.counters[3] != 0 && gridDim.x <= (unsigned)kMaxPlanCtas;
        list_first = contiguous ? a.w.cta_first[blockIdx.x] : 0; list_end = contiguous ? a.w.cta_first[blockIdx.x + 1] : 0;
    }
    auto unit_at = [&](int k) -> int {
        if (contiguous) return list_first + k < list_end ? list_first + k : n_units;
        return snake_unit(k, blockIdx.x, gridDim.x);
    };
    // next unit of this CTA (false: no more); every warp role walks the list with its own cursor
    auto fetch = [&](fused_plan::Cursor& cur, UnitView& un) -> bool {
        if (kFused) {
            fused_plan::Unit f;
            if (!fused_plan::next_unit(plan, cur, a.B, a.Hkv, a.G, f)) return false;
            un.req = f.req; un.kvh = f.kvh; un.rb = f.rb; un.n_nodes = f.n_nodes;
            un.tile_begin = f.tile_begin; un.tile_end = f.tile_end; un.n_chunks = f.n_chunks; un.chunk = f.chunk;
            un.slot_base = f.slot_base; un.slot_stride = f.slot_stride; un.bump = f.bump;
            un.slot = f.slot_base + f.chunk * f.slot_stride + (f.chunk == 0 ? f.bump : 0);
            return true;
        }
        const int u = unit_at(cur.k++);
        if (u >= n_units) return false;
        const AttnUnit x = a.w.units[u];
        un.req = x.req; un.kvh = x.kvh; un.rb = x.rb; un.tile_begin = x.tile_begin; un.tile_end = x.tile_end;
        un.n_chunks = x.n_chunks; un.chunk = x.chunk; un.n_nodes = a.w.req[x.req].n_nodes;
        un.slot = u; un.slot_base = 0; un.slot_stride = 0; un.bump = 0;
        return true;
    };
    const int pages_per_tile = kTileKeys / a.page_size;
    const uint32_t page_bytes = (uint32_t)a.page_size * 128u;

    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(&bars->full[i], 1); mbar_init(&bars->empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars->s_ready[i], 1); mbar_init(&bars->p_ready[i], 128); mbar_init(&bars->pv_done[i], 1); }
        mbar_init(&bars->q_ready, 256);
        mbar_init(&bars->stats_ready, 128);
        mbar_init(&bars->epi_done, 128);
        mbar_init(&bars->part_out, 128);
        mbar_init(&bars->merge_full, 1);
        mbar_init(&bars->merge_free, 8);
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (kFused) {
        // this CTA's units, worked out here (the ring is idle until the first unit starts)
        fused_plan::make<kMaxChunks>(a.prefix_len, a.num_nodes, a.B, a.N, a.Hkv, a.G, a.page_size, a.max_pages,
                         (FusedPlanScratch*)(smem + kOffRing), (FusedPlan*)(smem + kOffFused), a.status_word);
    }
    if (kFused) fence_async_proxy();                       // the plan's scratch is about to be overwritten by tensor copies
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    // columns: [0,128) S/P of group 0, [128,256) S/P of group 1, [256,384) O of group 0, [384,512) O of group 1

    // register hand-over between warpgroups: the third warpgroup gives registers up, the softmax warpgroups take them
    // (each instruction is executed by all four warps of its warpgroup, and the role code stays inside that branch)
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 8) {
        // ------------------------------------------------------------------ producer
        // One-launch variant (64 requests or fewer), one row block per kv head: every K/V line is read once per call,
        // by one CTA, and is marked to leave L2 first, so that the stream does not push out what the step reads again
        // (the index the draft kernel probes, page tables, the kernels' own code).  With several row blocks the
        // siblings share K/V through L2 and the lines keep the default policy; so do the large batches of the
        // three-launch variant, where the mark bought nothing and cost 2-3 %.
        const bool stream_once = kFused && a.w.row_blocks == 1;
        const uint64_t evict_first = kFused ? l2_policy_evict_first() : 0ull;
        uint32_t ld = 0;
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int i = un.req;
            const int L = a.prefix_len[i] + un.n_nodes;
            const int total_pages = (L + a.page_size - 1) / a.page_size;
            const int32_t* pt = a.page_table + (size_t)i * a.max_pages;
            const int T = un.tile_end - un.tile_begin;
            auto page_of = [&](int t) -> int {                   // this lane's page id in local tile t (-1: none)
                if (t >= T || lane >= pages_per_tile) return -1;
                const int pi = (un.tile_begin + t) * pages_per_tile + lane;
                return pi < total_pages ? pt[pi] : -1;
            };
            auto load = [&](int t, int page, bool is_v) -> bool {
                const uint32_t slot = ld % kSlots, phase = (ld / kSlots) & 1u;
                ++ld;
                bool w = mbar_wait(&bars->empty[slot], phase ^ 1u, bars, a.status_word);
                w = __all_sync(0xffffffffu, w);
                if (!w) return false;
                const int n_valid = min(pages_per_tile, total_pages - (un.tile_begin + t) * pages_per_tile);
                if (lane == 0) mbar_arrive_expect_tx(&bars->full[slot], (uint32_t)n_valid * page_bytes);
                __syncwarp();
                if (lane < n_valid) {
                    long long pg = page;
                    if (pg < 0 || pg >= a.num_pages) { war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE); pg = 0; }
                    const CUtensorMap* map = is_v ? &v_map : &k_map;
                    if (stream_once) tma_load_page_hint(sRing + slot * kSlotBytes + lane * page_bytes, map, un.kvh, (int)pg, &bars->full[slot], evict_first);
                    else tma_load_page(sRing + slot * kSlotBytes + lane * page_bytes, map, un.kvh, (int)pg, &bars->full[slot]);
                }
                return true;
            };
            int pg_cur = page_of(0), pg_nxt = page_of(1);
            ok = load(0, pg_cur, false);                                    // K0
            for (int t = 0; t < T && ok; ++t) {
                const int pg_nn = page_of(t + 2);                            // page ids two tiles ahead, off the critical path
                if (t + 1 < T) ok = load(t + 1, pg_nxt, false);              // K(t+1)
                if (ok) ok = load(t, pg_cur, true);                          // V(t)
                pg_cur = pg_nxt; pg_nxt = pg_nn;
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ MMA issuer
        uint32_t ld0 = 0, cg[2] = {0, 0}, units_done = 0;
        // operand types of one product: the 8-bit parts of q and of the weights against the cache's codes
        const uint32_t kv = (uint32_t)a.kv_e5m2;
        const uint32_t idesc_s = umma_idesc8(0, kv, 0), idesc_hi = umma_idesc8(0, kv, 1), idesc_lo = umma_idesc8(1, kv, 1);
        // every tile is rows of 128 bytes, 8-row groups 1 KB apart: Q and K as K-major operands, V as an MN-major one
        constexpr uint32_t hi = umma_desc_hi(1024);
        const uint32_t q_lo = umma_desc_lo(sQ, 16), ring_lo = umma_desc_lo(sRing, 16);
        auto mma_s = [&](uint32_t d_s, uint32_t k_lo) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {                             // 32 dims at a time: high parts of q, then low parts
                const uint32_t at = (uint32_t)(ks & 3) * 2u;
                umma_f8(d_s, pack64(q_lo + (uint32_t)(ks >> 2) * (16384u >> 4) + at, hi), pack64(k_lo + at, hi), idesc_s, ks > 0);
            }
        };
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int T = un.tile_end - un.tile_begin;
            auto issue_s = [&](int t) -> bool {
                const uint32_t sq = seq_k(ld0, t), slot = sq % kSlots, g = t & 1;
                if (!mbar_wait(&bars->full[slot], (sq / kSlots) & 1u, bars, a.status_word)) return false;
                tc_fence_after();
                if (lane == 0) {
                    mma_s(tmem + g * 128u, ring_lo + slot * (kSlotBytes >> 4));
                    umma_commit(&bars->s_ready[g]);
                    umma_commit(&bars->empty[slot]);
                }
                __syncwarp();
                return true;
            };
            ok = mbar_wait(&bars->q_ready, units_done & 1u, bars, a.status_word);
            if (ok) ok = issue_s(0);
            if (ok && T > 1) ok = issue_s(1);
            for (int t = 0; t < T && ok; ++t) {
                const uint32_t g = t & 1, tg = cg[g] + (uint32_t)(t >> 1);
                const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                const bool has_s = t + 2 < T;                        // S(t+2) goes out in the same burst as PV(t)
                const uint32_t sq_k = has_s ? seq_k(ld0, t + 2) : 0u, slot_k = sq_k % kSlots;
                ok = mbar_wait(&bars->p_ready[g], tg & 1u, bars, a.status_word) &&
                     mbar_wait(&bars->full[slot], (sq / kSlots) & 1u, bars, a.status_word);
                if (ok && has_s) ok = mbar_wait(&bars->full[slot_k], (sq_k / kSlots) & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t v_lo = ring_lo + slot * (kSlotBytes >> 4), d_o = tmem + 256u + g * 128u, a_p = tmem + g * 128u;
                    const uint32_t acc0 = t > 1 ? 1u : 0u;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {                     // 32 keys at a time: high and low parts of the weights
                        const uint64_t v_desc = pack64(v_lo + (uint32_t)ks * (4096u >> 4), hi);
                        umma_f8_ts(d_o, a_p + (uint32_t)ks * 8u, v_desc, idesc_hi, ks > 0 ? 1u : acc0);
                        umma_f8_ts(d_o, a_p + 32u + (uint32_t)ks * 8u, v_desc, idesc_lo, 1u);
                    }
                    if (has_s) {
                        // sixteen MMAs back to back; the completion signals follow the burst (the one the softmax group
                        // waits for first)
                        mma_s(tmem + g * 128u, ring_lo + slot_k * (kSlotBytes >> 4));
                        umma_commit(&bars->s_ready[g]);
                    }
                    umma_commit(&bars->pv_done[g]);
                    umma_commit(&bars->empty[slot]);
                    if (has_s) umma_commit(&bars->empty[slot_k]);
                }
                __syncwarp();
            }
            cg[0] += (uint32_t)(T + 1) >> 1;
            cg[1] += (uint32_t)T >> 1;
            ld0 += 2u * T;
            ++units_done;
        }
    } else if (kFused && warp == 10) {
        // ------------------------------------------------------------------ signaller (fused-plan variant)
        // Counts every split unit of this CTA whose partial result is out, for the CTA that merges the triple.  The
        // softmax warps only arrive on a barrier; the device-wide fence and the atomic sit here, off their path.
        uint32_t outs = 0;
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            if (un.n_chunks == 1) continue;
            const int32_t* prow = a.parent + (size_t)un.req * a.N;
            const int q0 = lane < a.N ? prow[lane] : 0, q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            if (tree_is_malformed(q0, q1, un.n_nodes, lane)) continue;          // (no partial is written for it)
            ok = mbar_wait(&bars->part_out, outs & 1u, bars, a.status_word);
            ++outs;
            if (ok && lane == 0) {
                __threadfence();
                count_arrival(&a.w.pair_count[(un.req * a.Hkv + un.kvh) * a.w.row_blocks + un.rb], a.call);
            }
            __syncwarp();
        }
    }
    } else {
        // ------------------------------------------------------------------ softmax groups, one thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int grp = warp >> 2;
        const int quad = warp & 3;
        const int row = quad * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        const uint32_t tS = tmem + grp * 128u + lane_addr;          // S, later P, of this group
        const uint32_t tO = tmem + 256u + grp * 128u + lane_addr;
        uint32_t ld0 = 0, cgm = 0, cg_other = 0, units_done = 0;    // cgm: tiles this group has processed so far
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int u = un.slot;
            const int i = un.req;
            const int n = un.n_nodes;
            const int R = a.G * n;
            const int pl = a.prefix_len[i];
            const int L = pl + n;
            const int gr = un.rb * kRowBlock + row;
            const bool in_tree = gr < R;
            const int j = in_tree ? gr / a.G : 0, g = in_tree ? gr % a.G : 0;
            const size_t qrow = ((size_t)i * a.N + j) * a.Hq + un.kvh * a.G + g;
            const int T = un.tile_end - un.tile_begin;
            // fused-plan variant: the plan has looked at num_nodes and prefix_len only; the tree itself is checked
            // below, by every warp that is about to use it (all come to the same verdict).  Its parent row is
            // requested here, ahead of the Q rows, and looked at after them.
            int q0 = 0, q1 = 0;
            if (kFused) {
                const int32_t* prow = a.parent + (size_t)i * a.N;
                q0 = lane < a.N ? prow[lane] : 0; q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            }
            // group 1 may not touch Q, O or its statistics before group 0 has finished the previous unit's epilogue
            if (grp == 1 && units_done > 0) {
                ok = mbar_wait(&bars->epi_done, (units_done - 1) & 1u, bars, a.status_word);
                if (!ok) break;
            }
            // The row's largest magnitude fixes a power of two that puts it into [128, 256); the scaled row is the sum of a
            // high part, rounded to e4m3, and a low part, the remainder rounded to e4m3: exact for elements above 2^-9 of
            // the largest.  Each group writes one 64-wide half of both (swizzled K-major).
            float row_scale;
            {
                const uint4* src = reinterpret_cast<const uint4*>(a.q + qrow * 128);
                uint4 x[8];
                uint32_t top = 0;                                           // bf16 magnitudes compare as integers
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const uint4 y = in_tree ? src[c ^ (grp ? 0 : 8)] : make_uint4(0, 0, 0, 0);      // the other half first
                    top = max(top, max(max(mag2(y.x), mag2(y.y)), max(mag2(y.z), mag2(y.w))));
                    if (c >= 8) x[c - 8] = y;
                }
                const int e = (int)(top >> 7);                              // biased exponent of the largest
                const uint32_t up = top == 0 ? 127u : (uint32_t)min(254 + 7 - e, 254);              // 2^(7 - exponent)
                const float f = __uint_as_float(up << 23);
                row_scale = top >= 0x7f80u ? CUDART_NAN_F : a.scale_log2 / f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {                               // 16 dims a piece
                    uint32_t h4[4], l4[4];
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint4 y = x[2 * c + v];
                        const uint32_t w4[4] = {y.x, y.y, y.z, y.w};
                        uint32_t h2[4], l2[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float lo = __uint_as_float(w4[i] << 16) * f, hi = __uint_as_float(w4[i] & 0xffff0000u) * f;
                            h2[i] = quant::encode2(lo, hi, kKvE4M3);
                            const float2 back = quant::decode2(h2[i], kKvE4M3);
                            l2[i] = quant::encode2(lo - back.x, hi - back.y, kKvE4M3);
                        }
                        h4[2 * v] = h2[0] | (h2[1] << 16); h4[2 * v + 1] = h2[2] | (h2[3] << 16);
                        l4[2 * v] = l2[0] | (l2[1] << 16); l4[2 * v + 1] = l2[2] | (l2[3] << 16);
                    }
                    const uint32_t dst = sQ + (uint32_t)row * 128u + (uint32_t)(((grp * 4 + c) ^ (row & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(h4[0]), "r"(h4[1]), "r"(h4[2]), "r"(h4[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 16384u), "r"(l4[0]), "r"(l4[1]), "r"(l4[2]), "r"(l4[3]) : "memory");
                }
            }
            fence_async_proxy();
            mbar_arrive(&bars->q_ready);
            // A malformed tree makes its units run with no live row: nothing is written for the request.
            bool tree_ok = true;
            if (kFused) {
                tree_ok = !tree_is_malformed(q0, q1, n, lane);
                if (!tree_ok && lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_TREE);
            }
            const bool valid = in_tree && tree_ok;
            const bool warp_valid = __any_sync(0xffffffffu, valid);
            uint64_t anc;
            if (kFused) {
                anc = tree_ok ? warp_ancestor_mask(q0, q1, n, j, lane) : 0ull;
                if (!valid) anc = 0ull;
            } else {
                anc = valid ? a.w.anc[(size_t)i * a.N + j] : 0ull;
            }
            float m_used = -CUDART_INF_F, l = 0.f;
            // Scales of a tile: lane l < 16 holds K's for its 8-key group l, lane 16 + l V's; page ids are requested two of
            // the group's tiles ahead, the scales themselves one ahead.  Groups past the request's end get 1
            // and 0 (their own scales may be anything, and V's reference follows the live ones).
            const float* scales = lane < 16 ? a.pools.kscale : a.pools.vscale;
            auto scale_page = [&](int t) -> int {
                const int pos = (un.tile_begin + t) * kTileKeys + (lane & 15) * 8;
                return t < T && pos < L ? a.page_table[(size_t)i * a.max_pages + (pos >> a.page_shift)] : -1;
            };
            auto scale_at = [&](int t, int page) -> float {
                const int pos = (un.tile_begin + t) * kTileKeys + (lane & 15) * 8;
                if (t >= T || pos >= L) return lane < 16 ? 1.f : 0.f;
                const long long pg = page < 0 || page >= a.num_pages ? 0 : page;
                return scales[((pg * a.Hkv + un.kvh) << a.bpp_shift) + ((pos & (a.page_size - 1)) >> a.block_shift)];
            };
            float sc_next = scale_at(grp, scale_page(grp));
            int page_next = scale_page(grp + 2);
            float v_ref = 0.f;                                             // power of two that V's scales are taken relative to
            for (int t = grp; t < T && ok; t += 2, ++cgm) {
                const float sc = sc_next;
                sc_next = scale_at(t + 2, page_next);
                page_next = scale_page(t + 4);
                const int key0 = (un.tile_begin + t) * kTileKeys;
                const bool need_mask = key0 + kTileKeys > pl;
                ok = mbar_wait(&bars->s_ready[grp], cgm & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();
                if (warp_valid) {
                    // the whole row of S comes into registers once
                    uint32_t r[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, r + c * 32);
                    tmem_wait_ld();
                    if (need_mask) {
                        // Which of the tile's 128 keys this row sees, as a bit mask built once: the first d keys are
                        // prefix (all visible), key d + a is tree slot a (visible when a is the row's slot or an ancestor;
                        // the ancestor mask has no bit at or above num_nodes, so keys past the request's end are out).
                        // Two instructions per element afterwards: this path runs once per (request, kv head) and its
                        // code, fetched cold, competes with the main loop for the instruction cache.
                        const int d = pl - key0;                                  // < 128 here
                        unsigned long long lo, hi;
                        if (d >= 64) { lo = ~0ull; hi = ((1ull << (d - 64)) - 1ull) | (anc << (d - 64)); }
                        else if (d > 0) { lo = ((1ull << d) - 1ull) | (anc << d); hi = anc >> (64 - d); }
                        else { lo = d > -64 ? anc >> (-d) : 0ull; hi = 0ull; }
                        const uint32_t w[4] = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (!((w[e >> 5] >> (e & 31)) & 1u)) r[e] = 0xff800000u;     // -inf
                    }
                    // V's scales relative to a power of two that follows the largest one seen: a factor below 2
                    const float sv_top = __uint_as_float(__reduce_max_sync(0xffffffffu, lane < 16 ? 0u : __float_as_uint(sc)));
                    float v_corr = 1.f;
                    if (sv_top >= 2.f * v_ref) {
                        const float ref = __uint_as_float(max(__float_as_uint(sv_top) & 0x7f800000u, 0x0c800000u));   // at least 2^-102
                        v_corr = v_ref / ref;
                        v_ref = ref;
                    }
                    const float sv = sc * (kWeightTop / v_ref);            // lanes 16 to 31
                    float mx = -CUDART_INF_F;
#pragma unroll
                    for (int g8 = 0; g8 < 16; ++g8) {                      // 8 keys with one scale: three-input max, then the scale
                        const uint32_t* x = r + g8 * 8;
                        const float m0 = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
                        const float m1 = max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5]));
                        const float m2 = max3(m0, __uint_as_float(x[6]), __uint_as_float(x[7]));
                        mx = fmaxf(mx, fmaxf(m1, m2) * fmaxf(__shfl_sync(0xffffffffu, sc, g8) * row_scale, kTinyScale));
                    }
                    float corr = 1.f;
                    bool rescale = v_corr != 1.f;
                    if (mx > m_used + kRescaleThreshold || (m_used == -CUDART_INF_F && mx > -CUDART_INF_F)) {
                        corr = exp2f(m_used - mx);                 // 0 when nothing was accumulated yet
                        l *= corr;
                        m_used = mx;
                        rescale = true;
                    }
                    rescale = rescale && t > grp;                  // O of this group holds earlier tiles of the unit
                    corr *= v_corr;
                    const float neg_m = m_used == -CUDART_INF_F ? 0.f : -m_used;
                    // p = exp2(s * scales - m) goes into the sum as it is; p * (V's scale) goes to the tensor cores as a high
                    // part, rounded to e4m3, and a low part, the remainder rounded to e5m2 (as exact, and it reaches further
                    // down): together within 2^-8 of it, and 2^-23 of the largest weight for the smallest
                    float2 l4[4] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
                    const float2 nm2 = make_float2(neg_m, neg_m);
                    uint32_t ph[32], pw[32];
#pragma unroll
                    for (int g8 = 0; g8 < 16; ++g8) {
                        const float ks = fmaxf(__shfl_sync(0xffffffffu, sc, g8) * row_scale, kTinyScale);
                        const float vs = __shfl_sync(0xffffffffu, sv, 16 + g8);
                        const float2 ks2 = make_float2(ks, ks), vs2 = make_float2(vs, vs);
                        uint32_t h2[4], w2[4];
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int e = g8 * 8 + 2 * v;
                            const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), ks2, nm2);
                            const float2 pp = make_float2(fast_exp2(x.x), fast_exp2(x.y));          // exp2(-inf) = 0
                            l4[v] = __fadd2_rn(l4[v], pp);
                            split_weights(__fmul2_rn(pp, vs2), h2[v], w2[v]);
                        }
                        ph[2 * g8] = h2[0] | (h2[1] << 16); ph[2 * g8 + 1] = h2[2] | (h2[3] << 16);
                        pw[2 * g8] = w2[0] | (w2[1] << 16); pw[2 * g8 + 1] = w2[2] | (w2[3] << 16);
                    }
                    l += ((l4[0].x + l4[0].y) + (l4[1].x + l4[1].y)) + ((l4[2].x + l4[2].y) + (l4[3].x + l4[3].y));
                    if (__any_sync(0xffffffffu, rescale)) {
                        // O of this group is stable once its previous P V product has completed
                        ok = mbar_wait(&bars->pv_done[grp], (cgm - 1) & 1u, bars, a.status_word);
                        ok = __all_sync(0xffffffffu, ok);
                        if (ok) {
                            tc_fence_after();
                            const float f = rescale ? corr : 1.f;
#pragma unroll 1                                                    // (rare: kept small, see the mask path above)
                            for (int c = 0; c < 4; ++c) {
                                uint32_t o[32];
                                tmem_ld32(tO + c * 32, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st32(tO + c * 32, o);
                            }
                        }
                    }
                    tmem_st32(tS, ph);
                    tmem_st32(tS + 32, pw);
                    tmem_wait_st();
                }
                if (!ok) break;
                // the unit's last tile may hold rows past the request's last key: zero their V (P is exactly 0 there,
                // but 0 x NaN garbage would still poison the product)
                if (key0 + kTileKeys > L) {
                    const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                    ok = mbar_wait(&bars->full[slot], (sq / kSlots) & 1u, bars, a.status_word);
                    if (!ok) break;
                    if (row >= L - key0) {
                        const uint32_t base = sRing + slot * kSlotBytes + (uint32_t)row * 128u;
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + c * 16u), "r"(0) : "memory");
                    }
                    fence_async_proxy();
                }
                tc_fence_before();
                mbar_arrive(&bars->p_ready[grp]);
            }
            if (!ok) break;
            if (row_scale != row_scale) l = row_scale;                     // NaN or infinity among the row's queries
            const uint32_t mine = (uint32_t)(T + 1 - grp) >> 1, theirs = (uint32_t)(T + grp) >> 1;   // tiles of this unit per group
            const bool fused_split = kFused && un.n_chunks != 1;
            if (grp == 1) {
                stats[row] = m_used; stats[128 + row] = l; stats[256 + row] = v_ref * (1.f / kWeightTop);
                mbar_arrive(&bars->stats_ready);
            } else {
                // epilogue: both groups' last products, then merge (max, sum, O) of the two groups and store
                ok = mbar_wait(&bars->pv_done[0], (cgm - 1) & 1u, bars, a.status_word) &&
                     mbar_wait(&bars->stats_ready, units_done & 1u, bars, a.status_word);
                if (ok && theirs > 0) ok = mbar_wait(&bars->pv_done[1], (cg_other + theirs - 1) & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();
                if (warp_valid) {
                    const float m1 = theirs > 0 ? stats[row] : -CUDART_INF_F, l1 = theirs > 0 ? stats[128 + row] : 0.f;
                    const float M = fmaxf(m_used, m1);
                    const float w0 = m_used == -CUDART_INF_F ? 0.f : exp2f(m_used - M);
                    const float w1 = m1 == -CUDART_INF_F ? 0.f : exp2f(m1 - M);
                    const float lsum = l * w0 + l1 * w1;
                    const bool split = un.n_chunks != 1;
                    float f0 = split ? w0 : (lsum == 0.f ? 0.f : w0 / lsum), f1 = split ? w1 : (lsum == 0.f ? 0.f : w1 / lsum);
                    f0 *= v_ref * (1.f / kWeightTop); f1 *= theirs > 0 ? stats[256 + row] : 0.f;       // what O is relative to
                    const bool use1 = theirs > 0;                  // uniform: O of group 1 is stale when it had no tile
#pragma unroll 1                                                    // (once per unit: kept small, see the mask path above)
                    for (int c = 0; c < 8; ++c) {
                        uint32_t o0[16], o1[16];
                        tmem_ld16(tO + c * 16, o0);
                        if (use1) tmem_ld16(tO + 128u + c * 16, o1);
                        tmem_wait_ld();
                        float x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            x[e] = __uint_as_float(o0[e]) * f0;
                            if (use1) x[e] = fmaf(__uint_as_float(o1[e]), f1, x[e]);
                        }
                        if (valid) {
                            if (!split) {
                                uint4* dst = reinterpret_cast<uint4*>(a.out + qrow * 128 + c * 16);
#pragma unroll
                                for (int v = 0; v < 2; ++v) {
                                    uint32_t w4[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const __nv_bfloat162 h = __floats2bfloat162_rn(x[v * 8 + 2 * e], x[v * 8 + 2 * e + 1]);
                                        w4[e] = *reinterpret_cast<const uint32_t*>(&h);
                                    }
                                    dst[v] = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                                }
                            } else {
                                float4* dst = reinterpret_cast<float4*>(a.w.part_o + ((size_t)u * a.w.rows + row) * 128 + c * 16);
#pragma unroll
                                for (int v = 0; v < 4; ++v) dst[v] = make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]);
                            }
                        }
                    }
                    if (valid) {
                        if (!split) {
                            if (a.lse) a.lse[qrow] = (M + log2f(lsum)) * kLn2;
                        } else {
                            a.w.part_ml[((size_t)u * a.w.rows + row) * 2] = M;
                            a.w.part_ml[((size_t)u * a.w.rows + row) * 2 + 1] = lsum;
                        }
                    }
                }
                tc_fence_before();
                mbar_arrive(&bars->epi_done);
                if (fused_split && tree_ok) mbar_arrive(&bars->part_out);     // this thread's share of the partial is written
            }
            (void)mine;
            cg_other += theirs;
            ld0 += 2u * T;
            ++units_done;
        }
        if (kFused && ok) {
            // ---- merges of split (request, kv head, row block) triples, by all eight softmax warps.  Contiguous
            // split: every CTA has at most one, the pair its last unit began.  Snake deal: the triples of all split
            // requests are dealt to the CTAs in turn, so the work at the end of the kernel is spread over all SMs.
            // Nothing waits for this CTA any more (its own partials are out), so waiting here cannot close a cycle. ----
            uint32_t merge_phase = 0;
            int share = kRowBlock;
            auto merge_one = [&](const UnitView& un, int part, int parts) -> bool {
                MergeArgs m;
                m.part = part; m.parts = parts; m.share = share;
                m.part_o = a.w.part_o; m.part_ml = a.w.part_ml; m.out = a.out; m.lse = a.lse; m.status_word = a.status_word;
                m.rows = a.w.rows; m.G = a.G; m.N = a.N; m.Hq = a.Hq;
                m.req = un.req; m.kvh = un.kvh; m.rb = un.rb; m.n_nodes = un.n_nodes; m.n_chunks = un.n_chunks;
                m.slot_base = un.slot_base; m.slot_stride = un.slot_stride; m.bump = un.bump;
                m.arrivals = &a.w.pair_count[(un.req * a.Hkv + un.kvh) * a.w.row_blocks + un.rb]; m.call = a.call;
                m.seen = &a.w.pair_seen[(un.req * a.Hkv + un.kvh) * a.w.row_blocks + un.rb];
                const bool done = merge_partials<kSlots * kSlotBytes>(m, smem + kOffRing, smem + kOffQ, bars, &merge_phase);
                return done;
            };
            auto tree_bad = [&](int req, int n) -> bool {              // a malformed tree left no partials
                const int32_t* prow = a.parent + (size_t)req * a.N;
                const int q0 = lane < a.N ? prow[lane] : 0, q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
                return tree_is_malformed(q0, q1, n, lane);
            };
            if (plan->mode == 1) {
                fused_plan::cursor_init(plan, cur);
                while (ok) {
                    UnitView un;
                    if (!fetch(cur, un)) break;
                    if (un.n_chunks == 1 || un.chunk != 0 || tree_bad(un.req, un.n_nodes)) continue;
                    ok = merge_one(un, 0, 1);
                }
            } else {
                // With few split triples every one is merged by two, four or eight CTAs, a share of its rows each: a
                // triple of many chunks is up to a megabyte that one SM would bring in and walk through in several
                // rounds.  Shares of at least 16 rows, on at most half of the CTAs (measured: 1 and 2 requests
                // with 128-row trees 74 -> 47 and 75 -> 64 us per call, 2 and 3 requests with 32-row trees 64 -> 60
                // and 71 -> 68; more shares than that bought nothing or cost a microsecond).
                const int n_split = plan->n_used, rows_blk = plan->t_all;
                int parts = 1, lg = 0;
                while (parts < 8 && 4 * parts * n_split <= (int)gridDim.x && rows_blk >= 32 * parts) { parts *= 2; ++lg; }
                share = (((rows_blk + parts - 1) >> lg) + 1) & ~1;
                int dealt = 0;                                         // shares of split requests before this one
#pragma unroll 1
                for (int p = 0; p < a.B && ok; ++p) {
                    const int i = plan->pos_req[p];
                    const int nc = plan->u.s.nc[i], n = plan->n[i];
                    if (nc <= 1 || n == 0) continue;
                    const int rbs = (a.G * n + kRowBlock - 1) / kRowBlock, per = a.Hkv * rbs, shares = per * parts;
                    int k = ((int)blockIdx.x - dealt) % (int)gridDim.x;
                    if (k < 0) k += gridDim.x;
                    dealt += shares;
                    if (k >= shares || tree_bad(i, n)) continue;
#pragma unroll 1
                    for (; k < shares && ok; k += gridDim.x) {
                        const int part = k / per, tr = k - part * per;       // the shares of a triple sit `per` CTAs apart
                        UnitView un;
                        un.req = i; un.kvh = tr / rbs; un.rb = tr - un.kvh * rbs; un.n_nodes = n; un.n_chunks = nc; un.chunk = 0;
                        un.tile_begin = un.tile_end = 0; un.slot = 0;
                        un.slot_base = (int)plan->u.s.pos_base[p] + tr; un.slot_stride = per; un.bump = 0;
                        ok = merge_one(un, part, parts);
                    }
                }
            }
        }
    }
    // ---------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
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

// The tensor maps of a call depend only on the pools' addresses and shapes, so the last few are kept (by value: a map holds
// an address and strides, nothing of the contents).
struct PoolMapKey {
    const void *k, *v; long long num_pages, s[6]; int Hkv, page_size, dev;
    bool operator==(const PoolMapKey& o) const {
        for (int i = 0; i < 6; ++i) if (s[i] != o.s[i]) return false;
        return k == o.k && v == o.v && num_pages == o.num_pages && Hkv == o.Hkv && page_size == o.page_size && dev == o.dev;
    }
};
struct PoolMaps { PoolMapKey key; CUtensorMap k_map, v_map; bool used; };
constexpr int kMapCacheEntries = 8;
std::mutex g_map_lock;
PoolMaps g_map_cache[kMapCacheEntries];

bool pool_maps(const PoolMapKey& key, CUtensorMap* k_map, CUtensorMap* v_map) {
    std::lock_guard<std::mutex> g(g_map_lock);
    for (int e = 0; e < kMapCacheEntries; ++e) {
        if (g_map_cache[e].used && g_map_cache[e].key == key) {
            const PoolMaps hit = g_map_cache[e];
            for (int m = e; m > 0; --m) g_map_cache[m] = g_map_cache[m - 1];
            g_map_cache[0] = hit;
            *k_map = hit.k_map; *v_map = hit.v_map;
            return true;
        }
    }
    PoolMaps fresh;
    fresh.key = key; fresh.used = true;
    if (!make_pool_map(&fresh.k_map, key.k, key.num_pages, key.Hkv, key.page_size, key.s) ||
        !make_pool_map(&fresh.v_map, key.v, key.num_pages, key.Hkv, key.page_size, key.s + 3))
        return false;
    for (int m = kMapCacheEntries - 1; m > 0; --m) g_map_cache[m] = g_map_cache[m - 1];
    g_map_cache[0] = fresh;
    *k_map = fresh.k_map; *v_map = fresh.v_map;
    return true;
}

constexpr int kMaxDevices = 64;
std::once_flag g_dev_once[kMaxDevices];
war_status_t g_dev_status[kMaxDevices];

war_status_t device_setup(int dev) {
    std::call_once(g_dev_once[dev], [dev]() {
        g_dev_status[dev] = WAR_ERR_CUDA;
        if (cudaFuncSetAttribute(attn_quant_sm100_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        if (cudaFuncSetAttribute(attn_quant_sm100_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

}  // namespace

war_status_t war_attn_quant_launch_sm100(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
                                         const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* parent,
                                         const war_attn_params_t* p, const AttnWorkspace& w, bool fused,
                                         void* out, float* lse, int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int grid = war_attn_sm_count();
    if (grid <= 0) return WAR_ERR_CUDA;
    CUtensorMap k_map, v_map;
    PoolMapKey key{pools.k, pools.v, p->num_pages, {}, p->Hkv, p->page_size, dev};
    for (int i = 0; i < 3; ++i) { key.s[i] = pools.ks[i]; key.s[3 + i] = pools.vs[i]; }
    if (!pool_maps(key, &k_map, &v_map)) return WAR_ERR_UNSUPPORTED;
    KernelArgs a;
    a.q = (const __nv_bfloat16*)q; a.page_table = page_table; a.prefix_len = prefix_len;
    a.out = (__nv_bfloat16*)out; a.lse = lse; a.status_word = status_word; a.w = w; a.pools = pools;
    a.num_pages = p->num_pages; a.scale_log2 = p->scale * kLog2e;
    a.N = p->N; a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.page_size = p->page_size; a.max_pages = p->max_pages_per_req;
    a.page_shift = log2_of(p->page_size); a.block_shift = log2_of(pools.block); a.bpp_shift = a.page_shift - a.block_shift;
    a.kv_e5m2 = pools.kv == kKvE5M2;
    a.num_nodes = num_nodes; a.parent = parent; a.B = p->B; a.call = fused ? war_attn_next_call() : 0;
    if (fused) attn_quant_sm100_kernel<true><<<grid, kThreads, kSmemBytes, s>>>(k_map, v_map, a);
    else attn_quant_sm100_kernel<false><<<grid, kThreads, kSmemBytes, s>>>(k_map, v_map, a);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
}
