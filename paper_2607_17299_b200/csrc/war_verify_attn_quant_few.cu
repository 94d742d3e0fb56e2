// Tensor-core verify attention over the 8-bit cache for sm_100a, for calls with at most 32 query rows per kv head
// (war_verify_attn_quant_many.cu has the others).  Work units, the ring of TMA-filled slots and the merge of split requests are
// those of war_verify_attn_sm100.cu; what differs is the arithmetic, because the cache's bytes go to the tensor cores as
// they are, and which operand is the wide one, because a product of 128 rows is wasted on 4 to 32 of them:
//
//   S = K Qh' + K Ql'      128 keys x the rows; q (scaled by a power of two per row) = Qh + Ql, both e4m3
//   p = exp2(S * (row's constant * K's scale of the key's block) - the row's reference)
//   O' += V' Ph + V' Pl    128 dims x the rows; p * (V's scale of the key's block) = Ph + Pl, e4m3 and e5m2; the row's
//                          reference follows these, not the p alone (see war_attn_quant.cuh)
//
// So a softmax thread has one key and all rows, and a tile of 128 keys costs sixteen products of 16 or 32 columns, each bound
// by the 4 KB of K or V that it reads from shared memory.  Rows' maxima lie across the lanes: a tile is worked out relative
// to the reference of the tiles before, the group's four warps vote whether some value exceeds it by more than
// 2^kRescaleThreshold, and only then the maxima are taken and the tile is worked out again (once or twice a unit).
// Converting the cache to 16 bits on chip instead would move every element through shared memory three more times.
// Four groups take tiles in turn, each with its own S, P, O, maxima and sums: one group's chain S -> exponentials -> P is
// about 6000 cycles long against the 1350 in which HBM brings a tile.  They are merged at the end of a unit.
// A tile is 16 KB of K and 16 KB of V, rows of 128 bytes in the 128-byte swizzle, for either memory order: one tensor map
// (d, token, head, page) with the pool's own strides, one copy per (page, head).
//
// Measured next to the bf16 kernel on the same keys and GPU (64 requests of 4096 to 32768 keys, 8 kv heads, 2.02 GB of codes): 16
// rows 368 us (5.5 TB/s, near HBM's bound) against 588, 32 rows 442 to 472 us (4.3 to 4.6 TB/s) against 591.  With 32 rows no unit is
// at its limit (issue slots 42 %, tensor pipe 12 %, DRAM 47 % over 16 requests): the softmax warps' chain is the longest.
// Single tokens (8 requests of 4096 keys, 67 MB): 31 us against 34, of which planning takes 5 and the merge of split requests 6.
// A row per lane, as for more rows, takes 600 us and more for 32 rows; three slots fewer in the ring 10 % more.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>
#include <mutex>
#include <type_traits>
#include "war_common.cuh"
#include "war_attn_quant_sm100_parts.cuh"

namespace {

constexpr int kGroups = 4;
constexpr int kSlots = 11;
constexpr int kSlotBytes = 16384;
constexpr int kThreads = 640;                      // four softmax warpgroups and {K producer, MMA of groups 0 and 2, of 1 and 3, V producer}
constexpr int kRegsLaunch = 96;                     // registers a thread that 640 threads can be launched with
constexpr int kRegsSoftmax = 104;
constexpr int kRegsOther = 64;
constexpr int kSoftWarps = 4 * kGroups;
constexpr int kWarpLoadK = kSoftWarps, kWarpMma = kSoftWarps + 1, kWarpLoadV = kSoftWarps + 3;
constexpr uint32_t kTmemCols = 512;
constexpr int kMaxRows = 32;
// What a unit costs in the split, times the bf16 kernel's tiles: with 32 rows a boundary takes as long as some fifteen tiles of
// 32 KB (64 requests of 8 slots 468 -> 447 us when it came in, 20 requests 158 -> 152; with 16 rows it made 326 us 332).
template <int kRp> constexpr int kUnitCostOf = kRp == 32 ? 3 : 1;
// The largest weight is 2^kRescaleThreshold (a stale reference) * kWeightTop = 448, the largest e4m3 value.
constexpr float kRescaleThreshold = 3.0f;          // log2 units
constexpr float kWeightTop = 56.f;
constexpr float kMargin = 1.f;                      // a new reference lies this far above the maximum
constexpr float kNoMax = 1e30f;                     // stands for minus the maximum of a row that has seen no key yet

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int kOffQ = 0;                            // [high, low parts][32 rows][128 dims]
constexpr int kOffP = 8192;                         // [group][128 keys][high, low parts of 16 or 32 rows]
constexpr int kGroupP = 8192;
constexpr int kOffRing = kOffP + kGroups * kGroupP;
constexpr int kOffBar = kOffRing + kSlots * kSlotBytes;
constexpr int kOffScales = kOffBar + 640;           // [tile of the CTA & 31][K, V][8-key group]
constexpr int kScaleTiles = 32;
constexpr int kOffSoft = kOffScales + kScaleTiles * 128;   // SoftmaxShared
constexpr int kSmemBytes = 232448;
constexpr int kOffFused = kSmemBytes - 1024 - 704;
// Scales are kept for 32 tiles.  While a tile y is unfinished, the slots of V of y, y + 2, y + 4 ... and of K of y + 6, y + 8 ...
// stay taken once they are loaded (one issuer serves these tiles in order): half of the loads from there on, so with kSlots
// slots no producer gets past y + 6 + kSlots.
static_assert(6 + kSlots < kScaleTiles, "scales of an unfinished tile stay");
constexpr int kMergeBytes = kGroups * kGroupP + kSlots * kSlotBytes;   // the weights' buffers and the ring, idle when parts are merged
constexpr int kMaxChunks = kMergeBytes / 1024 < fused_plan::kFusedMaxChunks ? kMergeBytes / 1024 : fused_plan::kFusedMaxChunks;   // two rows of every chunk
static_assert(kMergeBytes / 512 * 8 <= kOffP, "the parts' maxima and sums land in the Q tile");
static_assert(sizeof(FusedPlan) <= 704, "plan table of the fused-plan variant");
static_assert(sizeof(FusedPlanScratch) <= kSlots * kSlotBytes, "the plan scratch lives in the idle ring");
static_assert(kThreads >= kFusedThreads, "fused_plan::make searches with its first kFusedThreads threads");
static_assert(kThreads * kRegsLaunch >= kSoftWarps * 32 * kRegsSoftmax + 128 * kRegsOther, "the hand-over draws on the registers of the launch");

struct Bars {
    uint64_t full[kSlots], empty[kSlots];
    uint64_t s_ready[kGroups], p_ready[kGroups], pv_done[kGroups];
    uint64_t vote[kGroups];              // the four warps of a group have left a word for each other
    uint64_t scales[32];                 // a tile's scales are there (16 lanes of either producer); tile & 31
    uint64_t q_ready, stats_ready, epi_done;
    uint64_t part_out, merge_full, merge_free;
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 640, "barrier block");

// What the softmax warps tell each other.
struct SoftmaxShared {
    alignas(16) float row_scale[kMaxRows];   // scale * log2(e) / the power of two q was scaled by (NaN: the row's result is NaN)
    int q_row[kMaxRows];                 // row of q, out and lse
    unsigned long long anc[kMaxRows];    // tree slots the row sees
    float m[kGroups][kMaxRows], neg_m[kGroups][kMaxRows], corr[kGroups][kMaxRows];
    union {
        float sum[kGroups][4][kMaxRows]; // [group][warp]: the row sums at the end of a unit,
        float most[kGroups][4][kMaxRows];  // a tile's row maxima before
    };
    alignas(16) float f[kGroups][kMaxRows];          // factors of the groups' O in the epilogue
    float v_unit[kGroups];               // what a group's O is relative to
    alignas(16) int viol[2][kGroups][4]; // [tile parity][group][warp]
};
static_assert(kOffSoft + (int)sizeof(SoftmaxShared) <= kOffFused, "shared memory");

// Ring sequence numbers inside a unit of T tiles whose first load has number ld0, in the order the tensor pipe consumes the
// loads: K0, K1, K2, K3, V0, K4, V1, K5, ..., the last four V.
__device__ __forceinline__ uint32_t seq_k(uint32_t ld0, int t) { return ld0 + t + max(0, t - (kGroups - 1)); }
__device__ __forceinline__ uint32_t seq_v(uint32_t ld0, int t, int T) { return ld0 + t + min(T, t + kGroups); }

// descriptor upper word for the 64-byte swizzle
__device__ __forceinline__ constexpr uint32_t umma_desc_hi64(uint32_t sbo_bytes) { return (sbo_bytes >> 4) | (1u << 14) | (4u << 29); }

// One value per row and lane -> one row per lane (row = lane & (kN - 1)), combined over the 32 lanes.
template <int kN, class Op>
__device__ __forceinline__ float reduce_rows(float (&v)[kN], int lane, Op op) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        if (o >= kN) {
#pragma unroll
            for (int i = 0; i < kN; ++i) v[i] = op(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
        } else {
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < o; ++i) {
                const float send = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
                v[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, o));
            }
        }
    }
    return v[0];
}

// kFused: see attn_sm100_kernel.  kRp: rows that the operands are laid out for (16 or 32, the smaller that holds the call's
// trees; one instance per size keeps the code of a launch within the instruction cache).
template <bool kFused, int kRp>
__global__ void __launch_bounds__(kThreads, 1)
attn_quant_few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const QuantKernelArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars* bars = (Bars*)(smem + kOffBar);
    SoftmaxShared* const sh = (SoftmaxShared*)(smem + kOffSoft);
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
        for (int i = 0; i < kGroups; ++i) {
            mbar_init(&bars->s_ready[i], 1); mbar_init(&bars->p_ready[i], 4); mbar_init(&bars->pv_done[i], 1); mbar_init(&bars->vote[i], 4);
        }
        for (int i = 0; i < kScaleTiles; ++i) mbar_init(&bars->scales[i], 32);
        mbar_init(&bars->q_ready, kSoftWarps);
        mbar_init(&bars->stats_ready, kSoftWarps);
        mbar_init(&bars->epi_done, kSoftWarps);
        mbar_init(&bars->part_out, kSoftWarps);
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
        fused_plan::make<kMaxChunks, kUnitCostOf<kRp>>(a.prefix_len, a.num_nodes, a.B, a.N, a.Hkv, a.G, a.page_size, a.max_pages,
                         (FusedPlanScratch*)(smem + kOffRing), (FusedPlan*)(smem + kOffFused), a.status_word);
    }
    if (kFused) fence_async_proxy();                       // the plan's scratch is about to be overwritten by tensor copies
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
    // columns: S of group g at 64 g, its O (high parts, low parts) at 256 + 64 g

    // register hand-over between warpgroups: the last warpgroup gives registers up, the softmax warpgroups take them
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
        // ------------------------------------------------------------------ MMA issuers: groups 0 and 2, groups 1 and 3
        // One lane of each.  The tensor pipe takes only a few products in advance, so a single issuer stands still until its
        // burst is nearly through and then leaves the pipe idle while it looks at the next tile's barriers; with two, one
        // looks while the other's products run.  The second one also counts the split units of this CTA whose partial
        // result is out (fused-plan variant).
        const int w = warp - kWarpMma;
        uint32_t ld0 = 0, tiles_done[2] = {0, 0}, units_done = 0, outs = 0;          // [g >> 1]
        // K, Q and V: rows of 128 bytes in the 128-byte swizzle, 8-row groups 1 KB apart (K and Q K-major, V MN-major);
        // P: rows of 64 bytes in the 64-byte swizzle, MN-major
        constexpr uint32_t hi = umma_desc_hi(1024), hi_p = umma_desc_hi64(512);
        const uint32_t ring_lo = umma_desc_lo(sRing, 16), q_lo = umma_desc_lo(sQ, 16), p_lo = umma_desc_lo(smem_u32(smem + kOffP), 16);
        const uint32_t idesc_s = umma_idesc8(kRp, a.kv_e5m2, 0, 0, 0), idesc_hi = umma_idesc8(kRp, a.kv_e5m2, 0, 1, 1),
                       idesc_lo = umma_idesc8(kRp, a.kv_e5m2, 1, 1, 1);
        auto mma_s = [&](int g, uint32_t slot) {                               // S = K Q high + K Q low, 32 dims at a time
            const uint32_t k_lo = ring_lo + slot * (kSlotBytes >> 4), d_s = tmem + (uint32_t)g * 64u;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_f8(d_s, pack64(k_lo + (ks & 3) * 2u, hi), pack64(q_lo + (ks >> 2) * (kRp * 128u >> 4) + (ks & 3) * 2u, hi), idesc_s, ks > 0);
            umma_commit(&bars->s_ready[g]);
            umma_commit(&bars->empty[slot]);
        };
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int T = un.tile_end - un.tile_begin;
            const bool split = kFused && w == 1 && un.n_chunks != 1;
            int q0 = 0, q1 = 0;
            if (split) {
                const int32_t* prow = a.parent + (size_t)un.req * a.N;
                q0 = lane < a.N ? prow[lane] : 0; q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            }
            ok = wait_for(&bars->q_ready, units_done & 1u, bars, a.status_word);
            for (int g = w; g < kGroups && g < T && ok; g += 2) {
                const uint32_t sq = seq_k(ld0, g), slot = sq % kSlots;
                ok = landed(sq);
                if (!ok) break;
                tc_fence_after();
                if (lane == 0) mma_s(g, slot);
                __syncwarp();
            }
            for (int t = w; t < T && ok; t += 2) {
                const int g = t & (kGroups - 1);
                const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                const bool has_s = t + kGroups < T;                      // the group's next S goes out in the same burst as PV(t)
                const uint32_t sq_k = seq_k(ld0, t + kGroups), slot_k = sq_k % kSlots;
                const uint32_t done = g >= 2 ? tiles_done[1]++ : tiles_done[0]++;
                ok = landed(sq);
                if (ok && has_s) ok = landed(sq_k);
                if (ok) ok = wait_for(&bars->p_ready[g], done & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t v_lo = ring_lo + slot * (kSlotBytes >> 4), d_o = tmem + 256u + (uint32_t)g * 64u;
                    const uint32_t p_g = p_lo + (uint32_t)g * (kGroupP >> 4);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {                     // O += V^T P high + V^T P low, 32 keys at a time
                        const uint64_t v_desc = pack64(v_lo + ks * (4096u >> 4), hi);
                        umma_f8(d_o, v_desc, pack64(p_g + ks * (2048u >> 4), hi_p), idesc_hi, ks > 0 || t >= kGroups);
                        umma_f8(d_o, v_desc, pack64(p_g + ks * (2048u >> 4) + (kRp >> 4), hi_p), idesc_lo, 1u);
                    }
                    if (has_s) mma_s(g, slot_k);
                    umma_commit(&bars->pv_done[g]);
                    umma_commit(&bars->empty[slot]);
                }
                __syncwarp();
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
        // ------------------------------------------------------------------ softmax groups, one thread per key of a tile
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int grp = warp >> 2, quad = warp & 3;
        const int key = quad * 32 + lane;                            // TMEM lane: key of a tile, dimension of O
        const int tid_g = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t tS = t_lane + grp * 64u, tO = t_lane + 256u + grp * 64u;
        const uint32_t p_row = smem_u32(smem + kOffP) + (uint32_t)grp * kGroupP + (uint32_t)key * 64u;
        const uint32_t p_swz = (key >> 1) & 3;
        uint32_t ld0 = 0, cgm = 0, others = 0, units_done = 0, votes = 0;       // cgm: tiles this group has processed so far
        bool ok = true;
        fused_plan::Cursor cur{0, 0, 0};
        if (kFused) fused_plan::cursor_init(plan, cur);
        while (ok) {
            UnitView un;
            if (!fetch(cur, un)) break;
            const int i = un.req;
            const int n = un.n_nodes;
            const int R = a.G * n;                                       // at most kRp: one row block
            const int pl = a.prefix_len[i];
            const int L = pl + n;
            const int T = un.tile_end - un.tile_begin;
            int q0 = 0, q1 = 0;
            if (kFused) {
                const int32_t* prow = a.parent + (size_t)i * a.N;
                q0 = lane < a.N ? prow[lane] : 0; q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            }
            // nobody may touch Q or what the warps tell each other before all are through with the previous unit
            if (units_done > 0) {
                ok = wait_for(&bars->epi_done, (units_done - 1) & 1u, bars, a.status_word);
                if (!ok) break;
            }
            // Queries, sixteen threads a row, eight dims each.  A row's largest magnitude fixes a power of two that puts it into
            // [128, 256); the scaled row is the sum of a high part, rounded to e4m3, and a low part, the remainder rounded to
            // e4m3: exact for elements above 2^-9 of the largest.
            if (tid < 16 * kRp) {
                const int r = tid >> 4, piece = tid & 15;
                const bool in_tree = r < R;
                const int q_row = (i * a.N + (in_tree ? r / a.G : 0)) * a.Hq + un.kvh * a.G + (in_tree ? r % a.G : 0);
                const uint4 x = *(reinterpret_cast<const uint4*>(a.q + (size_t)q_row * 128) + piece);
                uint32_t top = in_tree ? max(max(mag2(x.x), mag2(x.y)), max(mag2(x.z), mag2(x.w))) : 0u;     // bf16 magnitudes compare as integers
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const int e = (int)(top >> 7);                              // biased exponent of the largest
                const uint32_t up = !in_tree ? 0u : top == 0 ? 127u : (uint32_t)min(254 + 7 - e, 254);  // 2^(7 - exponent); rows that are none: 0
                const float f = __uint_as_float(up << 23);
                if (piece == 0) {
                    sh->row_scale[r] = top >= 0x7f80u ? CUDART_NAN_F : in_tree ? a.scale_log2 / f : 0.f;
                    sh->q_row[r] = q_row;
                }
                const uint32_t w4[4] = {x.x, x.y, x.z, x.w};
                uint32_t h2[4], l2[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float lo = __uint_as_float(w4[k] << 16) * f, hi = __uint_as_float(w4[k] & 0xffff0000u) * f;
                    h2[k] = quant::encode2(lo, hi, kKvE4M3);
                    const float2 back = quant::decode2(h2[k], kKvE4M3);
                    l2[k] = quant::encode2(lo - back.x, hi - back.y, kKvE4M3);
                }
                const uint32_t at = sQ + (uint32_t)r * 128u + (uint32_t)(((piece >> 1) ^ (r & 7)) << 4) + (piece & 1) * 8u;
                st_shared8(at, h2[0] | (h2[1] << 16), h2[2] | (h2[3] << 16));
                st_shared8(at + kRp * 128u, l2[0] | (l2[1] << 16), l2[2] | (l2[3] << 16));
            }
            // A malformed tree: nothing is written for the request.
            bool tree_ok = true;
            if (kFused) {
                tree_ok = !tree_is_malformed(q0, q1, n, lane);
                if (!tree_ok && lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_TREE);
            }
            if (warp == 4) {                                                 // tree slots that every row sees
                const int j = lane < R ? lane / a.G : 0;
                unsigned long long anc = 0;
                if (kFused) { if (tree_ok) anc = warp_ancestor_mask(q0, q1, n, j, lane); }
                else anc = a.w.anc[(size_t)i * a.N + j];
                sh->anc[lane] = lane < R ? anc : 0ull;
            }
            if (tid_g < kRp) { sh->m[grp][tid_g] = -CUDART_INF_F; sh->neg_m[grp][tid_g] = kNoMax; }
            fence_async_proxy();
            warp_arrive(&bars->q_ready, lane);
            ok = wait_for(&bars->q_ready, units_done & 1u, bars, a.status_word);
            if (!ok) break;

            float v_ref = 1.f;                                             // power of two that V's scales are taken relative to
            float l[kRp];
#pragma unroll
            for (int r = 0; r < kRp; ++r) l[r] = 0.f;
            for (int t = grp; t < T; t += kGroups, ++cgm) {
                const int key0 = (un.tile_begin + t) * kTileKeys;
                const uint32_t ti = ld0 / 2 + t;
                const float* const sc = s_scale + (ti & (kScaleTiles - 1)) * 32;
                ok = wait_for(&bars->scales[ti & (kScaleTiles - 1)], (ti / kScaleTiles) & 1u, bars, a.status_word);
                if (!ok) break;
                const float ks = sc[key >> 3];
                if (t == grp) v_ref = v_reference(sc[16 + (lane & 15)]);
                const float vs = v_relative(sc[16 + (key >> 3)], v_ref) * (kWeightTop / 256.f);       // (split_weights wants x / 256)
                // Which rows see this thread's key: all (prefix), none (past the request's end), or those with the key's
                // tree slot among their ancestors.
                uint32_t see = ~0u;
                if (key0 + key >= pl) {
                    see = 0u;
                    const int slot = key0 + key - pl;
                    if (slot < n) {
#pragma unroll 1
                        for (int r = 0; r < kRp; ++r) see |= (uint32_t)((sh->anc[r] >> slot) & 1ull) << r;
                    }
                }
                ok = wait_for(&bars->s_ready[grp], cgm & 1u, bars, a.status_word);
                if (!ok) break;
                tc_fence_after();

                // x = S * (row's and key's scales) - the row's reference, -inf where the row does not see the key; p = exp2(x).
                // If some x + lv (p with V's scale, what the tensor cores get) of the group is above kRescaleThreshold the references
                // are renewed and all is worked out again; the group's four warps tell each other while the exponentials are under way.
                float x[kRp];
                const float2 ks2 = make_float2(ks, ks);
                bool viol = false;
#pragma unroll 1
                while (true) {
                    if constexpr (kRp == 32) tmem_ld32(tS, reinterpret_cast<uint32_t*>(x));
                    else tmem_ld16(tS, reinterpret_cast<uint32_t*>(x));
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < kRp; r += 4) {
                        const float4 rs = *reinterpret_cast<const float4*>(&sh->row_scale[r]), rm = *reinterpret_cast<const float4*>(&sh->neg_m[grp][r]);
                        const float2 y0 = __ffma2_rn(make_float2(x[r], x[r + 1]), __fmul2_rn(make_float2(rs.x, rs.y), ks2), make_float2(rm.x, rm.y));
                        const float2 y1 = __ffma2_rn(make_float2(x[r + 2], x[r + 3]), __fmul2_rn(make_float2(rs.z, rs.w), ks2), make_float2(rm.z, rm.w));
                        x[r] = y0.x; x[r + 1] = y0.y; x[r + 2] = y1.x; x[r + 3] = y1.y;
                    }
                    if (key0 + kTileKeys > pl) {
#pragma unroll
                        for (int r = 0; r < kRp; ++r)
                            if (!((see >> r) & 1u)) x[r] = -CUDART_INF_F;
                    }
                    int* const word = sh->viol[cgm & 1u][grp];
                    if (!viol) {
                        float top[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                        for (int r = 0; r < kRp; r += 4) { top[0] = max3(top[0], x[r], x[r + 1]); top[1] = max3(top[1], x[r + 2], x[r + 3]); }
                        const float lv = v_log(vs * (256.f / kWeightTop));
                        const bool mine = __any_sync(0xffffffffu, fmaxf(top[0], top[1]) + lv > kRescaleThreshold);
                        if (lane == 0) word[quad] = mine;
                        warp_arrive(&bars->vote[grp], lane);
                    }
#pragma unroll
                    for (int r = 0; r < kRp; ++r) x[r] = fast_exp2(x[r]);                       // exp2(-inf) = 0
                    if (viol) break;
                    ok = wait_for(&bars->vote[grp], votes++ & 1u, bars, a.status_word);
                    if (!ok) break;
                    const int4 w = *reinterpret_cast<const int4*>(word);
                    viol = (w.x | w.y | w.z | w.w) != 0;
                    if (!viol) break;
                    // ---- the tile's row maxima (of S * scales + lv, read again), and new references for all rows
                    if constexpr (kRp == 32) tmem_ld32(tS, reinterpret_cast<uint32_t*>(x));
                    else tmem_ld16(tS, reinterpret_cast<uint32_t*>(x));
                    tmem_wait_ld();
                    const float lv = v_log(vs * (256.f / kWeightTop));
#pragma unroll
                    for (int r = 0; r < kRp; ++r) x[r] = (see >> r) & 1u ? fmaf(x[r], sh->row_scale[r] * ks, lv) : -CUDART_INF_F;
                    const float most = reduce_rows(x, lane, [](float p, float q) { return fmaxf(p, q); });
                    if (lane < kRp) sh->most[grp][quad][lane] = most;
                    warp_arrive(&bars->vote[grp], lane);
                    ok = wait_for(&bars->vote[grp], votes++ & 1u, bars, a.status_word);
                    if (!ok) break;
                    if (tid_g < kRp) {
                        const int r = tid_g;
                        const float o = fmaxf(fmaxf(sh->most[grp][0][r], sh->most[grp][1][r]), fmaxf(sh->most[grp][2][r], sh->most[grp][3][r]));
                        // (a margin, so that the next one is further off; -inf stays -inf; a NaN row keeps its reference)
                        const float old = sh->m[grp][r], now = fmaxf(o + kMargin, old);
                        sh->m[grp][r] = now;
                        sh->neg_m[grp][r] = now == -CUDART_INF_F ? kNoMax : -now;
                        sh->corr[grp][r] = now == old ? 1.f : exp2f(0.5f * (old - now));    // 0 when nothing was accumulated yet; see half_step
                    }
                    warp_arrive(&bars->vote[grp], lane);
                    ok = wait_for(&bars->vote[grp], votes++ & 1u, bars, a.status_word);
                    if (!ok) break;
#pragma unroll
                    for (int r = 0; r < kRp; r += 4) {
                        const float4 c4 = *reinterpret_cast<const float4*>(&sh->corr[grp][r]);
                        l[r] = half_step(l[r], c4.x); l[r + 1] = half_step(l[r + 1], c4.y); l[r + 2] = half_step(l[r + 2], c4.z); l[r + 3] = half_step(l[r + 3], c4.w);
                    }
                }
                if (!ok) break;
                if (viol && t != grp) {
                    // (S of this tile was committed behind the group's last P V product: O is stable)
#pragma unroll 1
                    for (int c = 0; c < kRp; c += 8) {
                        uint32_t o[8];
                        tmem_ld8(tO + c, o);
                        const float* const f = &sh->corr[grp][c];
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(half_step(__uint_as_float(o[e]), f[e]));
                        tmem_st8(tO + c, o);
                    }
                    tmem_wait_st();
                }
                // p goes into the sums as it is, p * (V's scale) as high and low parts into the P buffer, 2 * kRp bytes a key
                const float2 vs2 = make_float2(vs, vs);
#pragma unroll
                for (int c = 0; c < kRp; c += 16) {
                    uint32_t h4[4], l4[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int r = c + 4 * q;
                        const float2 p0 = make_float2(x[r], x[r + 1]), p1 = make_float2(x[r + 2], x[r + 3]);
                        const float2 s0 = __fadd2_rn(make_float2(l[r], l[r + 1]), p0), s1 = __fadd2_rn(make_float2(l[r + 2], l[r + 3]), p1);
                        l[r] = s0.x; l[r + 1] = s0.y; l[r + 2] = s1.x; l[r + 3] = s1.y;
                        split_weights(__fmul2_rn(p0, vs2), __fmul2_rn(p1, vs2), h4[q], l4[q]);
                    }
                    st_shared16(p_row + (((c >> 4) ^ p_swz) << 4), h4[0], h4[1], h4[2], h4[3]);
                    st_shared16(p_row + ((((c + kRp) >> 4) ^ p_swz) << 4), l4[0], l4[1], l4[2], l4[3]);
                }
                // the request's last tile may hold rows past its last key: zero their V (the weights are exactly 0 there, but
                // 0 x NaN garbage would still poison the product)
                if (key0 + kTileKeys > L) {
                    const uint32_t sq = seq_v(ld0, t, T), slot = sq % kSlots;
                    ok = landed(sq);
                    if (!ok) break;
                    if (key >= L - key0) {
                        const uint32_t base = sRing + slot * kSlotBytes + (uint32_t)key * 128u;
#pragma unroll
                        for (int c = 0; c < 8; ++c) st_shared16(base + c * 16u, 0, 0, 0, 0);
                    }
                }
                fence_async_proxy();
                tc_fence_before();
                warp_arrive(&bars->p_ready[grp], lane);
            }
            if (!ok) break;
            // row sums over the group's keys: of this warp's here, of the four warps by whoever reads them
            {
                const float sum = reduce_rows(l, lane, [](float p, float q) { return p + q; });
                if (lane < kRp) sh->sum[grp][quad][lane] = sum;
            }

            // ---- epilogue: merge of the groups and the store
            if (tid_g == 0) sh->v_unit[grp] = v_ref * (1.f / kWeightTop);
            warp_arrive(&bars->stats_ready, lane);
            ok = wait_for(&bars->stats_ready, units_done & 1u, bars, a.status_word);
            // the last products of the groups that had tiles (this unit's tiles of group g: (T + 3 - g) / 4; `others` holds the
            // counts of earlier units' tiles, a byte's low bit per group)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const uint32_t mine = (uint32_t)(T + kGroups - 1 - g) / kGroups;
                const uint32_t before = (others >> g) & 1u;                // parity of the group's earlier tiles
                if (ok && mine > 0) ok = wait_for(&bars->pv_done[g], (before + mine - 1) & 1u, bars, a.status_word);
                others ^= (mine & 1u) << g;
            }
            if (!ok) break;
            tc_fence_after();
            const bool split = un.n_chunks != 1;
            static_assert(kGroups * 8 == 32, "a lane for every group of eight rows");
            if (quad == 0 && grp * 8 < kRp) {                            // the eight rows this group stores, a lane per row and group
                const int g = lane >> 3, r = grp * 8 + (lane & 7);
                float m = sh->m[g][r], sum = (sh->sum[g][0][r] + sh->sum[g][1][r]) + (sh->sum[g][2][r] + sh->sum[g][3][r]);
                const float down = normal_sum(m, sum);
                float M = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 16));
                const float w = m == -CUDART_INF_F ? 0.f : exp2f(m - M);
                sum *= w;
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                if (sh->row_scale[r] != sh->row_scale[r]) sum = CUDART_NAN_F;           // NaN or infinity among the queries
                const float norm = split ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
                sh->f[g][r] = w * (down * sh->v_unit[g]) * norm;
                if (g == 0 && tree_ok && r < R) {
                    if (!split) {
                        if (a.lse) a.lse[sh->q_row[r]] = (M + log2f(sum)) * kLn2;
                    } else {
                        float* ml = a.w.part_ml + ((size_t)un.slot * a.w.rows + r) * 2;
                        ml[0] = M; ml[1] = sum;
                    }
                }
            }
            warp_arrive(&bars->vote[grp], lane);
            ok = wait_for(&bars->vote[grp], votes++ & 1u, bars, a.status_word);
            if (!ok) break;
            // O^T: this thread has dimension `key` of every row; eight rows at a time, dealt to the groups
            static_assert(kRp <= 8 * kGroups, "eight rows a group");
            const int live = tree_ok ? min(kRp, R) - grp * 8 : 0;
            if (live > 0) {                                                // (once per unit: kept small)
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll 1
                for (int g = 0; g < kGroups && g < T; ++g) {
                    uint32_t x[8];
                    tmem_ld8(t_lane + 256u + g * 64u + grp * 8u, x);
                    const float4 f0 = *reinterpret_cast<const float4*>(&sh->f[g][grp * 8]), f1 = *reinterpret_cast<const float4*>(&sh->f[g][grp * 8 + 4]);
                    const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = fmaf(__uint_as_float(x[e]), f[e], o[e]);
                }
                float* const part = a.w.part_o + ((size_t)un.slot * a.w.rows + grp * 8) * 128 + key;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e >= live) break;
                    if (split) part[e * 128] = o[e];
                    else a.out[(size_t)sh->q_row[grp * 8 + e] * 128 + key] = __float2bfloat16_rn(o[e]);
                }
            }
            tc_fence_before();
            warp_arrive(&bars->epi_done, lane);
            if (kFused && split && tree_ok) warp_arrive(&bars->part_out, lane);     // this warp's share of the partial is written
            ld0 += 2u * T;
            ++units_done;
        }
        if (kFused && ok && warp < 8) {
            // ---- merges of split (request, kv head, row block) triples, by eight of the softmax warps.  Contiguous
            // split: every CTA has at most one, the pair its last unit began.  Snake deal: the triples of all split
            // requests are dealt to the CTAs in turn, so the work at the end of the kernel is spread over all SMs.
            // Nothing waits for this CTA any more (its own partials are out), so waiting here cannot close a cycle. ----
            uint32_t merge_phase = 0;
            // both groups' products are through: the buffers the parts land in are idle
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
                const bool done = merge_partials<kMergeBytes>(m, smem + kOffP, smem + kOffQ, bars, &merge_phase);
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
        for (const auto kernel : {attn_quant_few_kernel<false, 16>, attn_quant_few_kernel<false, 32>, attn_quant_few_kernel<true, 16>,
                                  attn_quant_few_kernel<true, 32>})
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

}  // namespace

war_status_t war_attn_quant_launch_few(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
                                       const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* parent,
                                       const war_attn_params_t* p, const AttnWorkspace& w, bool fused,
                                       void* out, float* lse, int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int grid = war_attn_sm_count(), rows = p->Hq / p->Hkv * p->N;
    if (grid <= 0) return WAR_ERR_CUDA;
    if (rows > kMaxRows) return WAR_ERR_UNSUPPORTED;
    CUtensorMap k_map, v_map;
    QuantKernelArgs a;
    if (!quant_kernel_args(q, pools, page_table, prefix_len, num_nodes, parent, p, w, fused, out, lse, status_word, &a, &k_map, &v_map))
        return WAR_ERR_UNSUPPORTED;
    const auto kernel = rows <= 16 ? (fused ? attn_quant_few_kernel<true, 16> : attn_quant_few_kernel<false, 16>)
                                   : (fused ? attn_quant_few_kernel<true, 32> : attn_quant_few_kernel<false, 32>);
    kernel<<<grid, kThreads, kSmemBytes, s>>>(k_map, v_map, a);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
}
