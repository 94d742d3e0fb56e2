// Tensor-core verify attention over the 8-bit cache for sm_100a, for calls with more than 32 query rows per kv head
// (war_verify_attn_quant_few.cu has the others).  The skeleton is that of war_verify_attn_sm100.cu (work units, warp roles, a
// ring of TMA-filled slots, two softmax groups with an accumulator each, one launch for up to 64 requests); what differs is
// the arithmetic, because the cache's bytes go to the tensor cores as they are:
//
//   S = Qh K' + Ql K'      q (scaled by a power of two per row) = Qh + Ql, both e4m3: eight kind::f8f6f4 products of 32 dims
//   p = exp2(S * (row's constant * K's scale of the key's block) - m)
//   O += Ph V' + Pl V'     p * (V's scale of the key's block) = Ph + Pl, e4m3 and e5m2: eight products of 32 keys; the row's
//                          reference m follows these, not the p alone (see war_attn_quant.cuh)
//
// Splitting the small operands keeps the tensor work of the bf16 kernel per key (sixteen products of 64 cycles a tile).  Converting the
// cache to 16 bits on chip instead would move every element through shared memory three more times (read, written twice as
// wide, read twice as wide by the tensor cores): 192 KB a tile, 1500 cycles, above the 1400 that HBM needs for a tile but
// below the 3400 that this kernel takes; it has not been tried here.
// A tile of 128 keys is 16 KB of K and 16 KB of V, rows of 128 bytes in the 128-byte swizzle, for either memory order: one
// tensor map (d, token, head, page) with the pool's own strides, one copy per (page, head).  The scales of a tile travel
// with it, sixteen 4-byte asynchronous copies for K and for V, so that no softmax warp waits for global memory.
//
// A tile is worked on in halves of 64 keys: while a group's softmax warps have one half, P V and the next tile's S of the other
// are on the tensor cores, so the next S is ready when they come to it (571 us against 598 with whole tiles, same GPU).
//
// Measured next to the bf16 kernel on the same keys and GPU: this one is the slower one, with half the bytes.  32 requests of 16K to
// 32K keys, 128 rows per kv head (1.60 GB): 577 us against 499; 64 requests, 64 rows (2.02 GB): 624 against 594; 4 requests of up to
// 131072 keys, 96 rows, e5m2 (0.40 GB): 197 against 156; 128 requests, 512 rows in four row blocks (1.19 GB): 1980 against 1310.
// 577 us are 2.8 TB/s and 700 TFLOP/s of the two products (each operand in two parts: twice that on the pipe).  Bound by the
// softmax warps: 11 instructions an element, two warps a scheduler, 47 % of the issue slots and 30 % of the tensor pipe used (8
// requests).  TMEM has no room for a third group's S next to two O.  Sixteen softmax
// warps, two threads a row, were slower in lockstep (754 us) and with the reference handed from half to half (639 us): what
// they gain in overlap they lose in instructions for agreeing on it and in registers.
#include <mutex>
#include <type_traits>
#include "war_attn_quant_sm100_parts.cuh"

namespace {

constexpr int kSlots = 11;
constexpr int kSlotBytes = 16384;
constexpr int kThreads = 384;                      // three warpgroups: softmax 0, softmax 1, {K producer, MMA 0, MMA 1, V producer}
constexpr int kRegsSoftmax = 224;
constexpr int kRegsOther = 48;
constexpr int kWarpLoadK = 8, kWarpMma = 9, kWarpLoadV = 11;        // (group g's issuer is warp kWarpMma + g)
constexpr uint32_t kTmemCols = 512;
// The largest weight is 2^kRescaleThreshold (a stale reference) * kWeightTop = 448, the largest e4m3 value.  (3 and 56 take as
// long and lose two bits of the smallest weights; with 32 rows and less, where a group renews all rows at once, 1 takes 11 %.)
constexpr float kRescaleThreshold = 1.0f;          // log2 units
constexpr float kWeightTop = 224.f;
constexpr float kTinyScale = 1.1754943508222875e-38f;   // a scale of 0 must not turn a masked -inf into NaN

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int kOffQ = 0;                            // high parts, then low parts
constexpr int kOffRing = 32768;
constexpr int kOffBar = kOffRing + kSlots * kSlotBytes;
constexpr int kOffStats = kOffBar + 512;
constexpr int kOffScales = kOffStats + 3 * 256 * 4;        // [tile of the CTA & 15][K, V][8-key group]
constexpr int kOffLv = kOffScales + 2048;                  // [softmax warp][V's scales: log2, relative][8-key group of its tile]
constexpr int kOffFused = kOffLv + 8 * 32 * 4;
constexpr int kSmemBytes = kOffFused + 768 + 1024;
// Scales are kept for 16 tiles.  While a tile y is unfinished, the slots of V of y, y + 2, y + 4 ... and of K of y + 2, y + 4 ...
// stay taken once they are loaded (one issuer serves these tiles in order): half of the loads from there on, so with kSlots
// slots no producer gets past y + 2 + kSlots.
constexpr int kScaleTiles = 16;
static_assert(2 + kSlots < kScaleTiles, "scales of an unfinished tile stay");
constexpr int kMaxChunks = kSlots * kSlotBytes / 1024;    // the merge needs two rows of every chunk in the ring
static_assert(sizeof(FusedPlan) <= 768, "plan table of the fused-plan variant");
static_assert(kSmemBytes <= 232448, "shared memory");
static_assert(sizeof(FusedPlanScratch) <= kSlots * kSlotBytes, "the plan scratch lives in the idle ring");
static_assert(kThreads == kFusedThreads, "fused_plan::make is written for the attention kernel's block size");
static_assert(kThreads * 168 >= 256 * kRegsSoftmax + 128 * kRegsOther, "the hand-over draws on the registers of the launch");

struct Bars {
    uint64_t full[kSlots], empty[kSlots];
    uint64_t s_ready[2][2], p_ready[2][2], pv_done[2][2];     // [group][half of a tile]
    uint64_t scales[kScaleTiles];        // a tile's scales are there (16 lanes of either producer)
    uint64_t exch;                       // the epilogue's exchange buffer has been written / read
    uint64_t q_ready, stats_ready, epi_done;
    uint64_t part_out, merge_full, merge_free;
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// Ring sequence numbers as in the bf16 kernel: K0, K1, V0, K2, V1, ..., K(T-1), V(T-2), V(T-1).
__device__ __forceinline__ uint32_t seq_k(uint32_t ld0, int t) { return t == 0 ? ld0 : ld0 + 2u * t - 1u; }
__device__ __forceinline__ uint32_t seq_v(uint32_t ld0, int t, int T) { return t == T - 1 ? ld0 + 2u * T - 1u : ld0 + 2u * t + 2u; }

__device__ __forceinline__ void umma_f8_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_zero8(uint32_t taddr) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%1], {%0, %0, %0, %0, %0, %0, %0, %0};" ::"r"(0), "r"(taddr) : "memory");
}

// kFused: see attn_sm100_kernel.
template <bool kFused>
__global__ void __launch_bounds__(kThreads, 1)
attn_quant_many_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const QuantKernelArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars* bars = (Bars*)(smem + kOffBar);
    float* st_m = (float*)(smem + kOffStats);        // [group][lane] maximum,
    float* st_l = st_m + 256;                        // sum,
    float* st_w = st_l + 256;                        // and what O is relative to, for the merge
    float* s_scale = (float*)(smem + kOffScales);
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
    // A load has landed.  Parities tell a phase from the next one only, and whoever waits here does not see every load of a slot:
    // if another issuer's load before this is still on its way, its phase would pass for this one.  So that one has to be
    // consumed first.  (It has been issued by then: the caller has seen a later load of its producer land, or the unit
    // before is through; so the load before that is consumed and the wait on `empty` cannot take one phase for another.)
    auto landed = [&](uint32_t sq) -> bool {
        const uint32_t slot = sq % kSlots, phase = (sq / kSlots) & 1u;
        return wait_for(&bars->empty[slot], phase ^ 1u, bars, a.status_word) && wait_for(&bars->full[slot], phase, bars, a.status_word);
    };
    const int pages_per_tile = kTileKeys / a.page_size;
    const uint32_t page_bytes = (uint32_t)a.page_size * 128u;

    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(&bars->full[i], 1); mbar_init(&bars->empty[i], 1); }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bars->s_ready[0][i], 1); mbar_init(&bars->p_ready[0][i], 4); mbar_init(&bars->pv_done[0][i], 1);
        }
        for (int i = 0; i < kScaleTiles; ++i) mbar_init(&bars->scales[i], 32);
        mbar_init(&bars->q_ready, 8);
        mbar_init(&bars->stats_ready, 8);
        mbar_init(&bars->epi_done, 4);
        mbar_init(&bars->exch, 4);
        mbar_init(&bars->part_out, 4);
        mbar_init(&bars->merge_full, 1);
        mbar_init(&bars->merge_free, 8);
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpMma) {
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
    const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
    // columns: [0,128) S/P of group 0, a half tile in each half, [128,256) S/P of group 1, [256,384) O of group 0, [384,512) O of group 1

    // register hand-over between warpgroups: the third warpgroup gives registers up, the softmax warpgroups take them
    // (each instruction is executed by all four warps of its warpgroup, and the role code stays inside that branch)
    if (warp >= kWarpLoadK) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kWarpLoadK || warp == kWarpLoadV) {
        // ------------------------------------------------------------------ producers of K and of V
        // (one lane issues one copy, and a warp's copies go out one after the other, about 60 ns each: with pages of 16
        // tokens a single warp brought in 6 TB/s / 1.35)
        // One-launch variant (64 requests or fewer), one row block per kv head: every K/V line is read once per call,
        // by one CTA, and is marked to leave L2 first, so that the stream does not push out what the step reads again
        // (the index the draft kernel probes, page tables, the kernels' own code).  With several row blocks the
        // siblings share K/V through L2 and the lines keep the default policy; so do the large batches of the
        // three-launch variant, where the mark bought nothing and cost 2-3 %.
        const bool stream_once = kFused && a.w.row_blocks == 1;
        const uint64_t evict_first = kFused ? l2_policy_evict_first() : 0ull;
        const bool is_v = warp == kWarpLoadV;
        const CUtensorMap* map = is_v ? &v_map : &k_map;
        const float* scales = is_v ? a.pools.vscale : a.pools.kscale;
        uint32_t ld0 = 0;
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
            auto load = [&](int t, int page) -> bool {
                const uint32_t ld = is_v ? seq_v(ld0, t, T) : seq_k(ld0, t);
                const uint32_t slot = ld % kSlots, phase = (ld / kSlots) & 1u;
                bool w = wait_for(&bars->empty[slot], phase ^ 1u, bars, a.status_word);
                w = __all_sync(0xffffffffu, w);
                if (!w) return false;
                const int n_valid = min(pages_per_tile, total_pages - (un.tile_begin + t) * pages_per_tile);
                if (lane == 0) mbar_arrive_expect_tx(&bars->full[slot], (uint32_t)n_valid * page_bytes);
                __syncwarp();
                // the tile's scales, one of its 16 groups of 8 keys a lane; groups past the request's end get 1 (K) and 0 (V):
                // their own may be anything, and V's reference follows the live ones
                long long spg = __shfl_sync(0xffffffffu, page, (lane & 15) * 8 >> a.page_shift);
                if (lane < 16) {
                    const uint32_t tile = ld0 / 2 + t;
                    uint64_t* bar = &bars->scales[tile & (kScaleTiles - 1)];
                    float* dst = s_scale + (tile & (kScaleTiles - 1)) * 32 + (is_v ? 16 : 0) + lane;
                    const int pos = (un.tile_begin + t) * kTileKeys + lane * 8;
                    if (pos < L) {
                        if (spg < 0 || spg >= a.num_pages) spg = 0;
                        cp_async4(smem_u32(dst), scales + ((spg * a.Hkv + un.kvh) << a.bpp_shift) + ((pos & (a.page_size - 1)) >> a.block_shift));
                        cp_async_arrive(bar);
                    } else {
                        *dst = is_v ? 0.f : 1.f;
                        mbar_arrive(bar);
                    }
                }
                if (lane < n_valid) {
                    long long pg = page;
                    if (pg < 0 || pg >= a.num_pages) { war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE); pg = 0; }
                    if (stream_once) tma_load_page_hint(sRing + slot * kSlotBytes + lane * page_bytes, map, un.kvh, (int)pg, &bars->full[slot], evict_first);
                    else tma_load_page(sRing + slot * kSlotBytes + lane * page_bytes, map, un.kvh, (int)pg, &bars->full[slot]);
                }
                return true;
            };
            int pg_cur = page_of(0), pg_nxt = page_of(1);
            for (int t = 0; t < T && ok; ++t) {
                const int pg_nn = page_of(t + 2);                            // page ids two tiles ahead, off the critical path
                ok = load(t, pg_cur);
                pg_cur = pg_nxt; pg_nxt = pg_nn;
            }
            ld0 += 2u * T;
        }
    } else {
        // ------------------------------------------------------------------ MMA issuers, a warp (one lane of it) per group
        // The tensor pipe takes only a few products in advance, so a single issuer stands still until its burst is nearly
        // through and then leaves the pipe idle while it looks at the next tile's barriers; with two, one looks while the
        // other's products run.  They take turns burst by burst: mixed bursts would both end late.  Group 1's issuer also
        // counts the split units of this CTA whose partial result is out (fused-plan variant).
        const int g = warp - kWarpMma;
        uint32_t ld0 = 0, cg = 0, units_done = 0, outs = 0;
        // operand types of one product: the 8-bit parts of q and of the weights against the cache's codes
        const uint32_t idesc_s = umma_idesc8(64, 0, a.kv_e5m2, 0, 0), idesc_hi = umma_idesc8(128, 0, a.kv_e5m2, 0, 1),
                       idesc_lo = umma_idesc8(128, 1, a.kv_e5m2, 0, 1);
        // every tile is rows of 128 bytes, 8-row groups 1 KB apart: Q and K as K-major operands, V as an MN-major one
        constexpr uint32_t hi = umma_desc_hi(1024);
        const uint32_t q_lo = umma_desc_lo(sQ, 16), ring_lo = umma_desc_lo(sRing, 16);
        const uint32_t d_s = tmem + (uint32_t)g * 128u, d_o = d_s + 256u;           // S and later P, O of this group
        auto mma_s = [&](uint32_t slot, int half) {
            const uint32_t k_lo = ring_lo + slot * (kSlotBytes >> 4) + (uint32_t)half * (8192u >> 4);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)                               // 32 dims at a time: high parts of q, then low parts
                umma_f8(d_s + (uint32_t)half * 64u, pack64(q_lo + (uint32_t)(ks >> 2) * (16384u >> 4) + (ks & 3) * 2u, hi), pack64(k_lo + (ks & 3) * 2u, hi), idesc_s, ks > 0);
            umma_commit(&bars->s_ready[g][half]);
        };
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int T = un.tile_end - un.tile_begin;
            const bool split = kFused && g == 1 && un.n_chunks != 1;
            int q0 = 0, q1 = 0;
            if (split) {
                const int32_t* prow = a.parent + (size_t)un.req * a.N;
                q0 = lane < a.N ? prow[lane] : 0; q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            }
            ok = wait_for(&bars->q_ready, units_done & 1u, bars, a.status_word);
            if (ok && g < T) {
                const uint32_t sq = seq_k(ld0, g), slot = sq % kSlots;
                ok = landed(sq);
                if (ok) {
                    tc_fence_after();
                    if (lane == 0) { mma_s(slot, 0); mma_s(slot, 1); umma_commit(&bars->empty[slot]); }
                    __syncwarp();
                }
            }
            for (int t = g; t < T && ok; t += 2, ++cg) {
                const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                const bool has_s = t + 2 < T;                        // S(t+2) of a half goes out behind its P V(t)
                const uint32_t sq_k = has_s ? seq_k(ld0, t + 2) : 0u, slot_k = sq_k % kSlots;
                ok = landed(sq);
                if (ok && has_s) ok = landed(sq_k);
#pragma unroll 1
                for (int half = 0; half < 2 && ok; ++half) {
                    ok = wait_for(&bars->p_ready[g][half], cg & 1u, bars, a.status_word);
                    if (!ok) break;
                    tc_fence_after();
                    if (lane == 0) {
                        const uint32_t v_lo = ring_lo + slot * (kSlotBytes >> 4) + (uint32_t)half * (8192u >> 4), d_p = d_s + (uint32_t)half * 64u;
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks) {                 // 32 keys at a time: high and low parts of the weights
                            const uint64_t v_desc = pack64(v_lo + (uint32_t)ks * (4096u >> 4), hi);
                            umma_f8_ts(d_o, d_p + (uint32_t)ks * 8u, v_desc, idesc_hi, ks > 0 || half > 0 || t > 1);
                            umma_f8_ts(d_o, d_p + 16u + (uint32_t)ks * 8u, v_desc, idesc_lo, 1u);
                        }
                        umma_commit(&bars->pv_done[g][half]);
                        if (half) umma_commit(&bars->empty[slot]);
                        if (has_s) {
                            mma_s(slot_k, half);
                            if (half) umma_commit(&bars->empty[slot_k]);
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
            }
            ld0 += 2u * T;
            ++units_done;
            if (ok && split && !tree_is_malformed(q0, q1, un.n_nodes, lane)) {       // (no partial is written for a malformed one)
                // The softmax warps only arrive on a barrier; the device-wide fence and the atomic sit here.  The next unit's
                // queries are on their way meanwhile.
                ok = wait_for(&bars->part_out, outs & 1u, bars, a.status_word);
                ++outs;
                if (ok && lane == 0) {
                    __threadfence();
                    count_arrival(&a.w.pair_count[(un.req * a.Hkv + un.kvh) * a.w.row_blocks + un.rb], a.call);
                }
                __syncwarp();
            }
        }
    }
    } else {
        // ------------------------------------------------------------------ softmax groups, one thread per row
        // With at most 64 rows in the block the rows stand twice among the 128 lanes, and a copy takes only half of the keys,
        // with its own maximum and its own O: the weights of the other keys are zero in its lanes.  So a thread has 64 or 32
        // keys of a row at a time, and all four schedulers work.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int grp = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;                            // TMEM lane
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        const uint32_t tS = tmem + grp * 128u + lane_addr;          // S, later P, of this group
        const uint32_t tO = tmem + 256u + grp * 128u + lane_addr;
        uint32_t ld0 = 0, cgm = 0, cg_other = 0, units_done = 0, exch = 0;      // cgm: tiles this group has processed so far
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int i = un.req;
            const int n = un.n_nodes;
            const int R = a.G * n;
            const int pl = a.prefix_len[i];
            const int L = pl + n;
            const bool twice = R - un.rb * kRowBlock <= 64;
            const int copy = twice ? row >> 6 : 0;
            const int r_l = twice ? row & 63 : row;                      // row in the block
            const int gr = un.rb * kRowBlock + r_l;
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
            // nobody may touch Q or the statistics before group 0 has finished the previous unit's epilogue
            if (units_done > 0) {
                ok = wait_for(&bars->epi_done, (units_done - 1) & 1u, bars, a.status_word);
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
                        for (int k = 0; k < 4; ++k) {
                            const float lo = __uint_as_float(w4[k] << 16) * f, hi = __uint_as_float(w4[k] & 0xffff0000u) * f;
                            h2[k] = quant::encode2(lo, hi, kKvE4M3);
                            const float2 back = quant::decode2(h2[k], kKvE4M3);
                            l2[k] = quant::encode2(lo - back.x, hi - back.y, kKvE4M3);
                        }
                        h4[2 * v] = h2[0] | (h2[1] << 16); h4[2 * v + 1] = h2[2] | (h2[3] << 16);
                        l4[2 * v] = l2[0] | (l2[1] << 16); l4[2 * v + 1] = l2[2] | (l2[3] << 16);
                    }
                    const uint32_t dst = sQ + (uint32_t)row * 128u + (uint32_t)(((grp * 4 + c) ^ (row & 7)) << 4);
                    st_shared16(dst, h4[0], h4[1], h4[2], h4[3]);
                    st_shared16(dst + 16384u, l4[0], l4[1], l4[2], l4[3]);
                }
            }
            fence_async_proxy();
            warp_arrive(&bars->q_ready, lane);
            // A malformed tree makes its units run with no live row: nothing is written for the request.
            bool tree_ok = true;
            if (kFused) {
                tree_ok = !tree_is_malformed(q0, q1, n, lane);
                if (!tree_ok && lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_TREE);
            }
            const bool valid = in_tree && tree_ok;
            const bool warp_valid = twice ? tree_ok : (bool)__any_sync(0xffffffffu, valid);      // (the copies meet in the epilogue)
            uint64_t anc;
            if (kFused) {
                anc = tree_ok ? warp_ancestor_mask(q0, q1, n, j, lane) : 0ull;
                if (!valid) anc = 0ull;
            } else {
                anc = valid ? a.w.anc[(size_t)i * a.N + j] : 0ull;
            }
            float m_used = -CUDART_INF_F, l = 0.f;
            float v_ref = 1.f;                                             // power of two that V's scales are taken relative to
            float* const s_lv = (float*)(smem + kOffLv) + warp * 32;      // log2 of V's scales, and the scales, relative to v_ref
            // Half a tile's share of this thread: kCols keys.
            auto step = [&](int t, int half, auto cols_c) -> bool {
                constexpr int kCols = decltype(cols_c)::value;
                const int c0 = half * 64 + (kCols == 32 ? copy * 32 : 0);  // first key of the tile that is this thread's
                const int key0 = (un.tile_begin + t) * kTileKeys;
                const uint32_t ti = ld0 / 2 + t;
                const float* const sc = s_scale + (ti & (kScaleTiles - 1)) * 32;
                if (half == 0) {
                    if (!wait_for(&bars->scales[ti & (kScaleTiles - 1)], (ti / kScaleTiles) & 1u, bars, a.status_word)) return false;
                    const float sv = sc[16 + (lane & 15)];
                    if (t == grp) v_ref = v_reference(sv);
                    const float rel = v_relative(sv, v_ref);
                    __syncwarp();                                          // (the tile before has been read)
                    if (lane < 16) { s_lv[lane] = v_log(rel); s_lv[16 + lane] = rel * (kWeightTop / 256.f); }    // (split_weights wants x / 256)
                    __syncwarp();
                }
                if (!wait_for(&bars->s_ready[grp][half], cgm & 1u, bars, a.status_word)) return false;
                tc_fence_after();
                // the thread's part of the row of S comes into registers once
                uint32_t r[kCols];
#pragma unroll
                for (int c = 0; c < kCols; c += 32) tmem_ld32(tS + c0 + c, r + c);
                tmem_wait_ld();
                if (key0 + c0 + kCols > pl) {
                    // Which of its keys this row sees, as a bit mask built once: the first d are prefix (all visible), key
                    // d + a is tree slot a (visible when a is the row's slot or an ancestor; the ancestor mask has no bit
                    // at or above num_nodes, so keys past the request's end are out).
                    const int d = pl - key0 - c0;                          // < kCols here
                    const unsigned long long see = d > 0 ? ((1ull << d) - 1ull) | (anc << d) : d > -64 ? anc >> (-d) : 0ull;
                    const uint32_t w[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        if (!((w[e >> 5] >> (e & 31)) & 1u)) r[e] = 0xff800000u;     // -inf
                }
                float mx = -CUDART_INF_F;
#pragma unroll
                for (int k = 0; k < kCols / 8; ++k) {                      // 8 keys with one scale: three-input max, then the scales
                    const uint32_t* x = r + k * 8;
                    const float m0 = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
                    const float m1 = max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5]));
                    mx = fmaxf(mx, fmaf(max3(m0, m1, fmaxf(__uint_as_float(x[6]), __uint_as_float(x[7]))), fmaxf(sc[(c0 >> 3) + k] * row_scale, kTinyScale), s_lv[(c0 >> 3) + k]));
                }
                float corr = 1.f;
                bool rescale = false;
                if (mx > m_used + kRescaleThreshold || (m_used == -CUDART_INF_F && mx > -CUDART_INF_F)) {
                    corr = exp2f(0.5f * (m_used - mx));                    // 0 when nothing was accumulated yet; see half_step
                    l = half_step(l, corr);
                    m_used = mx;
                    rescale = true;
                }
                rescale = rescale && (t > grp || half > 0);                // O of this group holds earlier keys of the unit
                const float neg_m = m_used == -CUDART_INF_F ? 0.f : -m_used;
                // p = exp2(s * scales - m) goes into the sum as it is; p * (V's scale) goes to the tensor cores as a high
                // part, rounded to e4m3, and a low part, the remainder rounded to e5m2
                float2 l4[4] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
                const float2 nm2 = make_float2(neg_m, neg_m);
                uint32_t ph[kCols / 4], pw[kCols / 4];
#pragma unroll
                for (int k = 0; k < kCols / 8; ++k) {
                    const float ks = fmaxf(sc[(c0 >> 3) + k] * row_scale, kTinyScale), vs = s_lv[16 + (c0 >> 3) + k];
                    const float2 ks2 = make_float2(ks, ks), vs2 = make_float2(vs, vs);
                    float2 w2[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int e = k * 8 + 2 * v;
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), ks2, nm2);
                        const float2 pp = make_float2(fast_exp2(x.x), fast_exp2(x.y));          // exp2(-inf) = 0
                        l4[v] = __fadd2_rn(l4[v], pp);
                        w2[v] = __fmul2_rn(pp, vs2);
                    }
                    split_weights(w2[0], w2[1], ph[2 * k], pw[2 * k]);
                    split_weights(w2[2], w2[3], ph[2 * k + 1], pw[2 * k + 1]);
                }
                l += ((l4[0].x + l4[0].y) + (l4[1].x + l4[1].y)) + ((l4[2].x + l4[2].y) + (l4[3].x + l4[3].y));
                if (__any_sync(0xffffffffu, rescale)) {
                    // O is stable once the products of the half before are through
                    if (!wait_for(&bars->pv_done[grp][half ^ 1], (half ? cgm : cgm - 1) & 1u, bars, a.status_word)) return false;
                    tc_fence_after();
                    const float f = rescale ? corr : 1.f;
#pragma unroll 1                                                           // (rare: kept small)
                    for (int c = 0; c < 8; ++c) {
                        uint32_t o[16];
                        tmem_ld16(tO + c * 16, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(half_step(__uint_as_float(o[e]), f));
                        tmem_st16(tO + c * 16, o);
                    }
                }
                const uint32_t at = tS + (uint32_t)half * 64u;
                if constexpr (kCols == 64) { tmem_st16(at, ph); tmem_st16(at + 16, pw); }
                else {
                    tmem_st8(at + copy * 8, ph); tmem_st8(at + 16 + copy * 8, pw);
                    const uint32_t z = at + (uint32_t)((copy ^ 1) << 3);   // the other copy's keys weigh nothing in these lanes
                    tmem_zero8(z); tmem_zero8(z + 16);
                }
                tmem_wait_st();
                return true;
            };
            for (int t = grp; t < T && ok; t += 2, ++cgm) {
#pragma unroll 1
                for (int half = 0; half < 2 && ok; ++half) {
                    if (warp_valid) ok = twice ? step(t, half, std::integral_constant<int, 32>()) : step(t, half, std::integral_constant<int, 64>());
                    else {
                        const uint32_t ti = ld0 / 2 + t;                   // (its scales as well: no phase of theirs is passed over)
                        ok = wait_for(&bars->scales[ti & (kScaleTiles - 1)], (ti / kScaleTiles) & 1u, bars, a.status_word) &&
                             wait_for(&bars->s_ready[grp][half], cgm & 1u, bars, a.status_word);
                        tc_fence_after();
                    }
                    if (!ok) break;
                    // the unit's last tile may hold rows past the request's last key: zero their V (P is exactly 0 there,
                    // but 0 x NaN garbage would still poison the product)
                    const int key0 = (un.tile_begin + t) * kTileKeys;
                    if (half == 0 && key0 + kTileKeys > L) {
                        const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                        ok = landed(sq);
                        if (!ok) break;
                        if (row >= L - key0) {
                            const uint32_t base = sRing + slot * kSlotBytes + (uint32_t)row * 128u;
#pragma unroll
                            for (int c = 0; c < 8; ++c) st_shared16(base + c * 16u, 0, 0, 0, 0);
                        }
                        fence_async_proxy();
                    }
                    tc_fence_before();
                    warp_arrive(&bars->p_ready[grp][half], lane);
                }
            }
            if (!ok) break;
            if (row_scale != row_scale) l = row_scale;                     // NaN or infinity among the row's queries
            const uint32_t theirs = (uint32_t)(T + grp) >> 1;              // tiles of this unit that the other group has
            const bool fused_split = kFused && un.n_chunks != 1;
            const float down = normal_sum(m_used, l);
            st_m[grp * 128 + row] = m_used; st_l[grp * 128 + row] = l; st_w[grp * 128 + row] = down * v_ref * (1.f / kWeightTop);
            warp_arrive(&bars->stats_ready, lane);
            if (grp == 0) {
                // epilogue: both groups' last products, then the merge of (max, sum, O) over groups and copies, and the store
                ok = wait_for(&bars->pv_done[0][1], (cgm - 1) & 1u, bars, a.status_word) &&
                     wait_for(&bars->stats_ready, units_done & 1u, bars, a.status_word);
                if (ok && theirs > 0) ok = wait_for(&bars->pv_done[1][1], (cg_other + theirs - 1) & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();
                if (warp_valid) {
                    const bool split = un.n_chunks != 1;
                    float M = -CUDART_INF_F;
                    for (int c = r_l; c < kRowBlock; c += twice ? 64 : 128) M = fmaxf(M, fmaxf(st_m[c], st_m[128 + c]));
                    float lsum = 0.f;
                    for (int c = r_l; c < kRowBlock; c += twice ? 64 : 128) {
                        const float m0 = st_m[c], m1 = st_m[128 + c];
                        lsum += st_l[c] * (m0 == -CUDART_INF_F ? 0.f : exp2f(m0 - M)) + st_l[128 + c] * (m1 == -CUDART_INF_F ? 0.f : exp2f(m1 - M));
                    }
                    if (row_scale != row_scale) lsum = row_scale;
                    const float norm = split ? 1.f : (lsum == 0.f ? 0.f : 1.f / lsum);
                    const float m1 = st_m[128 + row];
                    const float f0 = (m_used == -CUDART_INF_F ? 0.f : exp2f(m_used - M)) * st_w[row] * norm;
                    const float f1 = (m1 == -CUDART_INF_F ? 0.f : exp2f(m1 - M)) * st_w[128 + row] * norm;
                    const bool use1 = theirs > 0;                          // uniform: O of group 1 is stale when it had no tile
                    __nv_bfloat16* const out = a.out + qrow * 128;
                    float* const part = split ? a.w.part_o + ((size_t)un.slot * a.w.rows + r_l) * 128 : nullptr;
                    auto store8 = [&](int col, const float* x) {           // eight columns of this row
                        if (split) {
                            float4* dst = reinterpret_cast<float4*>(part + col);
                            dst[0] = make_float4(x[0], x[1], x[2], x[3]);
                            dst[1] = make_float4(x[4], x[5], x[6], x[7]);
                        } else {
                            uint32_t w4[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
                                w4[e] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            *reinterpret_cast<uint4*>(out + col) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                        }
                    };
                    // exchange buffer (the Q tile, idle by now): 64 columns of 128 lanes, 16-byte pieces swizzled over the lanes
                    float* const xb = (float*)(smem + kOffQ);
#pragma unroll 1                                                           // (once per unit: kept small)
                    for (int c = 0; c < 8; ++c) {
                        const int col = c * 16;
                        uint32_t o0[16], o1[16];
                        tmem_ld16(tO + col, o0);
                        if (use1) tmem_ld16(tO + 128u + col, o1);
                        tmem_wait_ld();
                        float x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            x[e] = __uint_as_float(o0[e]) * f0;
                            if (use1) x[e] = fmaf(__uint_as_float(o1[e]), f1, x[e]);
                        }
                        if (!twice) {
                            if (valid) { store8(col, x); store8(col + 8, x + 8); }
                            continue;
                        }
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            *reinterpret_cast<float4*>(xb + row * 64 + ((((c & 3) * 4 + v) ^ (row & 15)) << 2)) = make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]);
                        if ((c & 3) != 3) continue;
                        // 64 columns are there: the two copies of a row are summed, 32 columns a thread
                        warp_arrive(&bars->exch, lane);
                        if (!wait_for(&bars->exch, exch++ & 1u, bars, a.status_word)) { ok = false; break; }
                        for (int k = 0; k < 4; ++k) {
                            const int p0 = (copy * 4 + k) * 2;             // 16-byte piece
                            float y[8];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float4 s0 = *reinterpret_cast<const float4*>(xb + r_l * 64 + (((p0 + h) ^ (r_l & 15)) << 2));
                                const float4 s1 = *reinterpret_cast<const float4*>(xb + (r_l + 64) * 64 + (((p0 + h) ^ (r_l & 15)) << 2));
                                y[4 * h] = s0.x + s1.x; y[4 * h + 1] = s0.y + s1.y; y[4 * h + 2] = s0.z + s1.z; y[4 * h + 3] = s0.w + s1.w;
                            }
                            if (valid) store8((c >> 2) * 64 + p0 * 4, y);
                        }
                        if (c < 7) {                                       // the buffer is written again
                            warp_arrive(&bars->exch, lane);
                            if (!wait_for(&bars->exch, exch++ & 1u, bars, a.status_word)) { ok = false; break; }
                        }
                    }
                    ok = __all_sync(0xffffffffu, ok);
                    if (valid && copy == 0) {
                        if (!split) {
                            if (a.lse) a.lse[qrow] = (M + log2f(lsum)) * kLn2;
                        } else {
                            a.w.part_ml[((size_t)un.slot * a.w.rows + r_l) * 2] = M;
                            a.w.part_ml[((size_t)un.slot * a.w.rows + r_l) * 2 + 1] = lsum;
                        }
                    }
                }
                if (!ok) break;
                tc_fence_before();
                warp_arrive(&bars->epi_done, lane);
                if (fused_split && tree_ok) warp_arrive(&bars->part_out, lane);     // this warp's share of the partial is written
            }
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
            // the last unit's epilogue is through, and with it both groups' products: the ring is idle
            if (units_done > 0) ok = wait_for(&bars->epi_done, (units_done - 1) & 1u, bars, a.status_word);
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
    if (warp == kWarpMma) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

constexpr int kMaxDevices = 64;
std::once_flag g_dev_once[kMaxDevices];
war_status_t g_dev_status[kMaxDevices];

war_status_t device_setup(int dev) {
    std::call_once(g_dev_once[dev], [dev]() {
        g_dev_status[dev] = WAR_ERR_CUDA;
        for (const auto kernel : {attn_quant_many_kernel<false>, attn_quant_many_kernel<true>})
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

}  // namespace

war_status_t war_attn_quant_launch_many(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
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
    QuantKernelArgs a;
    if (!quant_kernel_args(q, pools, page_table, prefix_len, num_nodes, parent, p, w, fused, out, lse, status_word, &a, &k_map, &v_map))
        return WAR_ERR_UNSUPPORTED;
    if (fused) attn_quant_many_kernel<true><<<grid, kThreads, kSmemBytes, s>>>(k_map, v_map, a);
    else attn_quant_many_kernel<false><<<grid, kThreads, kSmemBytes, s>>>(k_map, v_map, a);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
}
