// Tensor-core attention over shared prefixes for sm_100a, 8-bit cache: the kernel of war_verify_attn_shared_sm100.cu with codes widened
// to halves on the way to the tensor cores.
//
// Every code of both types is a half, so K and V lose nothing.  Q is scaled by a power of two per row (its largest element into [2^14, 2^15)) and
// kept as halves: exact for elements above 2^-29 of the row's largest.  Scales stay outside of the products: K's goes to S, p * (V's
// scale) is rounded to a half (2^-11 of itself, or 2^-32 of the row's largest), with the row's reference as in war_attn_quant.cuh.
// What it costs: 4 prompts of 16K to 32K tokens with 7 rollouts of 32 slots and 4 requests alone, 32 + 8 heads, 637 us the call with e4m3 and as much
// with e5m2 (codes as they are: 721; each for itself 649; bf16 cache 530).  No one unit is the bound: a tile with two row blocks moves 352 KB through
// shared memory (operands 256, codes in 32, out of their slot and in again 64), 2750 cycles at 128 bytes each, which is 250 to 290 us of the call;
// the tensor pipe is 40 % busy, issue slots 51 %.  The rest is the chain of codes, wideners, products and softmax, which has not been taken apart.
// Conversions are not it (e5m2 is widened by moving bytes), nor are the slots for codes (four of them, three for halves: 709 against 656).
// Warp roles:  warps 8 and 11   producers: TMA copies of codes into two slots of 16 KB; the first one also brings the scales
//              warps 12-15      wideners: 16 KB of codes -> a 32 KB slot of the ring, rows of V past the part's last key zeroed
//              warps 9 and 10   MMA issuers, warps 0-3 and 4-7 softmax groups: as there
#include <mutex>
#include <type_traits>
#include "war_attn_quant_sm100_parts.cuh"
#include "war_attn_shared.cuh"

namespace {

constexpr int kSlots = 4, kStages = 2;                             // of halves, of codes
constexpr int kSlotBytes = 32768;
constexpr int kStageBytes = 16384;
constexpr int kLoadBars = 8, kStageBars = 4, kScaleTiles = 6;
constexpr int kThreads = 512;
constexpr int kRegsSoftmax = 200, kRegsOther = 56;                  // register budgets after the hand-over below
constexpr int kWarpLoad0 = 8, kWarpMma = 9, kWarpLoad1 = 11, kWarpWiden = 12;   // (group g's issuer is warp kWarpMma + g)
constexpr uint32_t kTmemCols = 512;
constexpr int kWidenDeep = 2;                                       // pieces of 16 codes that a widener asks for at once
constexpr int kAhead = 2;                                           // units whose numbers a CTA holds
constexpr float kRescaleThreshold = 8.0f;                           // log2 units

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int kOffQ = 0;                                            // two blocks of 128 rows
constexpr int kOffRing = 65536;
constexpr int kOffStage = kOffRing + kSlots * kSlotBytes;
constexpr int kOffScales = kOffStage + kStages * kStageBytes;       // [tile][K: 16 groups of 8 keys, V: 16]
constexpr int kOffLv = kOffScales + kScaleTiles * 128;              // [group][tile by turns][log2 of V's scales, and the scales, relative to v_ref]
constexpr int kOffBar = kOffLv + 512;
constexpr int kSmemBytes = kOffBar + 640 + 1024;
// where the groups share rows, the second block of Q is free: the rows' scales, and what group 1 leaves for the merge
constexpr int kOffRowScale = kOffQ + 32768, kOffStats = kOffRowScale + 512;
// The largest weight is 2^kRescaleThreshold (a stale reference) * kWeightTop = 2^15.
constexpr float kWeightTop = 128.f;
constexpr float kTinyScale = 1.1754943508222875e-38f;               // a scale of 0 must not turn a masked -inf into NaN
static_assert(kSmemBytes <= 232448, "shared memory");
static_assert(kThreads * 128 >= 256 * (kRegsSoftmax + kRegsOther), "the hand-over draws on the registers of the launch");

struct Bars {
    uint64_t full[kLoadBars];                                       // one arrival of each widener
    uint64_t empty[kLoadBars];                                      // two arrivals, one of each issuer or both of one
    uint64_t codes_full[kStageBars], codes_empty[kStageBars];       // two arrivals, one of each producer; one of each widener
    uint64_t scales[kScaleTiles];                                   // 32 arrivals, one a scale
    uint64_t s_ready[2][2], p_ready[2][2];                          // [group][half of a tile]
    uint64_t pv_done[2][2];                                         // of a group's last tile in a unit (else the next S says it)
    uint64_t q_ready, stats_ready, unit_done;
    uint64_t next_full[kAhead], next_free[kAhead];                  // numbers of the CTA's units, in the order they are run
    int next[kAhead];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 640, "barrier block");

// Load n of the CTA (see load_k) has codes in slot n % 2 and halves in slot n % 4 of the ring; its barriers are numbers n % 4 and n % 8, as in
// war_verify_attn_shared_sm100.cu.
// Scales are written without a wait for their ring.  Those of tile t + 1 come behind load K(t + 1), number 2t + 1 of its unit, for which the wideners
// are through with load 2t - 1 and so the issuers with load 2t - 5 and all before it, V(t - 4) among them: the softmax warps are past tile t - 4.
// A unit's first scales come behind the last load of the unit before, which says as much for the tile four back.  Five tiles would do.
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}
// two packed bf16 times f as halves
__device__ __forceinline__ uint32_t halves2(uint32_t w, float f) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(__uint_as_float(w & 0xffff0000u) * f), "f"(__uint_as_float(w << 16) * f));
    return r;
}
// 16 codes to halves (a code of e5m2 is a half's upper byte)
template <bool kE5M2>
__device__ __forceinline__ void widen16(const uint4& c, uint32_t* h) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (kE5M2) { h[2 * k] = __byte_perm(w[k], 0, 0x1404); h[2 * k + 1] = __byte_perm(w[k], 0, 0x3424); }
        else { h[2 * k] = quant::decode2_half(w[k] & 0xffffu, kKvE4M3); h[2 * k + 1] = quant::decode2_half(w[k] >> 16, kKvE4M3); }
    }
}

// Two elements of a softmax row, whose keys have the same scales: p = exp2(x * scale - m), added to a pair of sums in 32 bits, and p * vs as
// packed halves.
__device__ __forceinline__ void weights2(uint32_t x0, uint32_t x1, uint64_t scale2, uint64_t neg_m2, uint64_t vs2, uint64_t& sum2, uint32_t& packed) {
    asm("{\n.reg .b64 x, y;\n.reg .f32 a, b;\n"
        "mov.b64 x, {%2, %3};\n"
        "fma.rn.f32x2 x, x, %4, %5;\n"
        "mov.b64 {a, b}, x;\n"
        "ex2.approx.ftz.f32 a, a;\n"
        "ex2.approx.ftz.f32 b, b;\n"
        "mov.b64 y, {a, b};\n"
        "add.rn.f32x2 %1, %1, y;\n"
        "mul.rn.f32x2 y, y, %6;\n"
        "mov.b64 {a, b}, y;\n"
        "cvt.rn.f16x2.f32 %0, b, a;\n}\n"
        : "=r"(packed), "+l"(sum2) : "r"(x0), "r"(x1), "l"(scale2), "l"(neg_m2), "l"(vs2));
}

struct SharedQuantArgs {
    const __nv_bfloat16* q;
    const int32_t* page_table;
    const uint2* units;
    const SharedPart* parts;
    int* counters;
    const int* slot_map;
    const int32_t* parent;
    float *part_ml, *part_o;
    __nv_bfloat16* out;
    float* lse;
    int* status_word;
    const float *kscale, *vscale;
    long long num_pages;
    float scale_log2;
    int N, Hq, Hkv, G, page_size, max_pages, page_shift, block_shift, bpp_shift;
};

template <bool kE5M2>
__global__ void __launch_bounds__(kThreads, 1)
attn_shared_quant_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const SharedQuantArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars* bars = (Bars*)(smem + kOffBar);
    float* const s_row_scale = (float*)(smem + kOffRowScale);
    float4* const stats = (float4*)(smem + kOffStats);              // group 1's (max, sum, what O is relative to) per row
    float* const s_scale = (float*)(smem + kOffScales);
    const uint32_t sQ = smem_u32(smem + kOffQ), sRing = smem_u32(smem + kOffRing), sStage = smem_u32(smem + kOffStage);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // Every lane of a warp waits and all go on or none does (a wait that runs out must not split a warp).
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait_for(bar, parity, bars, a.status_word)); };
    // The CTA's k-th unit (false: no more).  Units are sorted, the longest first, and every CTA takes the next one when its loads are
    // through, so that CTAs with short units run more of them.  Producer 0 draws the numbers, the other warps read them here.
    auto unit_at = [&](int k, SharedUnit& un) -> bool {
        const int at = k % kAhead;
        if (!wait(&bars->next_full[at], (k / kAhead) & 1u)) return false;
        const int u = *(volatile int*)&bars->next[at];
        warp_arrive(&bars->next_free[at], lane);
        if (u < 0) return false;
        un = shared_unit(a.units, a.parts, u, a.Hkv, kSharedBlock);
        return true;
    };
    auto landed = [&](uint32_t load) -> bool { return wait(&bars->full[load % kLoadBars], (load / kLoadBars) & 1u); };
    auto landed_now = [&](uint32_t load) -> bool { return __all_sync(0xffffffffu, mbar_test(&bars->full[load % kLoadBars], (load / kLoadBars) & 1u)); };
    const int pages_per_tile = kTileKeys / a.page_size;
    const uint32_t page_bytes = (uint32_t)a.page_size * 128u;

    if (tid == 0) {
        for (int i = 0; i < kLoadBars; ++i) { mbar_init(&bars->full[i], 4); mbar_init(&bars->empty[i], 2); }
        for (int i = 0; i < kStageBars; ++i) { mbar_init(&bars->codes_full[i], 2); mbar_init(&bars->codes_empty[i], 4); }
        for (int i = 0; i < kScaleTiles; ++i) mbar_init(&bars->scales[i], 32);
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bars->s_ready[0][i], 1); mbar_init(&bars->p_ready[0][i], 4); mbar_init(&bars->pv_done[0][i], 1);
        }
        mbar_init(&bars->q_ready, 8);
        mbar_init(&bars->stats_ready, 4);
        mbar_init(&bars->unit_done, 8);
        for (int i = 0; i < kAhead; ++i) { mbar_init(&bars->next_full[i], 1); mbar_init(&bars->next_free[i], 15); }
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    war_wait_before();                                              // the plan
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
    // columns: [0,128) S of group 0, a half tile in each half, P over the first 32 of it; [128,256) of group 1; [256,384) O of group 0, [384,512) of 1

    // register hand-over between warpgroups, as in war_verify_attn_sm100.cu
    if (warp >= kWarpLoad0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kWarpLoad0 || warp == kWarpLoad1) {
        // ------------------------------------------------------------------ producers: both make every load, half of its pages each
        // (one lane issues one copy, and a warp's copies go out one after the other, about 60 ns each.  A warp for K and one for V
        // would not do here: with two slots the one could get a round of barriers ahead of the other, and parities would mislead it.)
        const int half = warp == kWarpLoad1;
        const int piece = 2 * lane + half;                          // this lane's page of a tile
        uint32_t ld = 0, tile0 = 0;
        bool ok = true;
        SharedUnit un;
        const int n_units = a.counters[1];
        int drawn = blockIdx.x;                                     // (lane 0 of producer 0) the number of the next unit
        auto take = [&](int k) -> bool {
            if (half == 1) return unit_at(k, un);
            const int at = k % kAhead, u = __shfl_sync(0xffffffffu, drawn < n_units ? drawn : -1, 0);
            if (!wait(&bars->next_free[at], ((k / kAhead) & 1u) ^ 1u)) return false;
            if (lane == 0) {
                *(volatile int*)&bars->next[at] = u;
                mbar_arrive(&bars->next_full[at]);
                if (u >= 0) drawn = (int)gridDim.x + atomicAdd(a.counters, 1);
            }
            __syncwarp();
            if (u < 0) return false;
            un = shared_unit(a.units, a.parts, u, a.Hkv, kSharedBlock);
            return true;
        };
        for (int k = 0; ok && take(k); ++k) {
            const int total_pages = (un.part.n_keys + a.page_size - 1) / a.page_size;
            const int32_t* pt = a.page_table + (size_t)un.part.req * a.max_pages + un.part.page0;
            const int T = un.tile_end - un.tile_begin;
            auto page_of = [&](int t) -> int {                      // this lane's page id in local tile t (-1: none)
                if (t >= T || piece >= pages_per_tile) return -1;
                const int pi = (un.tile_begin + t) * pages_per_tile + piece;
                return pi < total_pages ? pt[pi] : -1;
            };
            // the tile's scales, one of its 16 groups of 8 keys a lane, K's in lanes 0 to 15
            const float* const scales = lane < 16 ? a.kscale : a.vscale;
            const int group_at = (lane & 15) * 8;
            auto scale_page = [&](int t) -> int {
                const int pos = (un.tile_begin + t) * kTileKeys + group_at;
                return half == 0 && t < T && pos < un.part.n_keys ? pt[pos >> a.page_shift] : -1;
            };
            auto load_scales = [&](int t, long long pg) {          // groups past the part's end get 1 (K) and 0 (V)
                const uint32_t tile = tile0 + (uint32_t)t, at = tile % kScaleTiles;
                const int pos = (un.tile_begin + t) * kTileKeys + group_at;
                float* const dst = s_scale + at * 32u + lane;
                if (pos < un.part.n_keys) {
                    if (pg < 0 || pg >= a.num_pages) pg = 0;
                    cp_async4(smem_u32(dst), scales + ((pg * a.Hkv + un.kvh) << a.bpp_shift) + ((pos & (a.page_size - 1)) >> a.block_shift));
                    cp_async_arrive(&bars->scales[at]);
                } else {
                    *dst = lane < 16 ? 1.f : 0.f;
                    mbar_arrive(&bars->scales[at]);
                }
            };
            auto load = [&](int t, int page, bool is_v) -> bool {
                const uint32_t slot = ld % kStages, was = ld - kStages;      // (the load that had the slot)
                uint64_t* const full = &bars->codes_full[ld % kStageBars];
                const bool first_round = ld < (uint32_t)kStages;
                ++ld;
                if (!first_round && !wait(&bars->codes_empty[was % kStageBars], (was / kStageBars) & 1u)) return false;
                const int n_valid = min(pages_per_tile, total_pages - (un.tile_begin + t) * pages_per_tile);
                if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)((n_valid + 1 - half) >> 1) * page_bytes);
                __syncwarp();
                if (piece < n_valid) {
                    long long pg = page;
                    if (pg < 0 || pg >= a.num_pages) { war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE); pg = 0; }
                    tma_load_page(sStage + slot * kStageBytes + piece * page_bytes, is_v ? &v_map : &k_map, un.kvh, (int)pg, full);
                }
                return true;
            };
            int pg_cur = page_of(0), pg_nxt = page_of(1), sp_nxt = scale_page(1);
            if (half == 0) load_scales(0, scale_page(0));
            ok = load(0, pg_cur, false);                            // K0
            if (half == 1) {                                        // the unit's queries are wanted soon: into L2
                for (int r = lane; r < un.rows; r += 32) {
                    const int gr = un.row0 + r, j = gr / a.G;
                    const size_t slot_row = un.part.slot0 >= 0 ? (size_t)a.slot_map[un.part.slot0 + j] : (size_t)un.part.req * a.N + j;
                    const __nv_bfloat16* src = a.q + (slot_row * a.Hq + un.kvh * a.G + (gr - j * a.G)) * 128;
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(src));
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(src + 64));
                }
            }
            for (int t = 0; t < T && ok; ++t) {
                const int pg_nn = page_of(t + 2), sp_nn = scale_page(t + 2);         // page ids two tiles ahead, off the critical path
                if (t + 1 < T) ok = load(t + 1, pg_nxt, false);     // K(t+1)
                if (t + 1 < T && ok && half == 0) load_scales(t + 1, sp_nxt);
                if (ok) ok = load(t, pg_cur, true);                 // V(t)
                pg_cur = pg_nxt; pg_nxt = pg_nn; sp_nxt = sp_nn;
            }
            tile0 += (uint32_t)T;
        }
    } else if (warp >= kWarpWiden) {
        // ------------------------------------------------------------------ wideners: a quarter of the keys of every load each
        // A lane takes 16 codes of a row (TMA left 16-byte piece p of row r at p ^ (r & 7)) to two pieces of halves (2p and 2p + 1, modulo
        // 8, of the half of the slot that has their dims, swizzled alike).  Eight lanes have four pieces of rows r and r ^ 5: the rows
        // differ in bit 2, so that they read all banks, and in bit 0, so that they write all banks.
        const int w = warp - kWarpWiden, p = (lane & 3) | ((lane >> 1) & 4);
        uint32_t from_at[2], to_at[2];                              // for the first two and the other two pairs of eight rows
        int row8[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int b = 2 * x + (lane >> 4), r = (lane & 4) ? b ^ 5 : b;
            row8[x] = w * 32 + r;
            from_at[x] = (uint32_t)(row8[x] * 128 + ((p ^ r) << 4));
            to_at[x] = (uint32_t)((p >> 2) * 16384 + row8[x] * 128 + ((((p & 3) * 2) ^ r) << 4));
        }
        uint32_t ld = 0;
        bool ok = true;
        SharedUnit un;
        for (int k = 0; ok && unit_at(k, un); ++k) {
            const int T = un.tile_end - un.tile_begin, last = un.part.n_keys - un.tile_begin * kTileKeys;        // keys of the part from here
            for (int x = 0; x < 2 * T && ok; ++x, ++ld) {
                // K0 K1 V0 K2 V1 ... V(T-1)
                const bool is_v = x == 2 * T - 1 || (x > 0 && (x & 1) == 0);
                const int t = is_v ? (x == 2 * T - 1 ? T - 1 : x / 2 - 1) : (x + 1) / 2;
                const uint32_t slot = ld % kSlots, was = ld - kSlots;
                ok = wait(&bars->codes_full[ld % kStageBars], (ld / kStageBars) & 1u);
                if (ok && ld >= (uint32_t)kSlots) ok = wait(&bars->empty[was % kLoadBars], (was / kLoadBars) & 1u);
                if (!ok) break;
                const uint32_t src = sStage + (ld % kStages) * kStageBytes, dst = sRing + slot * kSlotBytes;
                const int live = is_v ? last - t * kTileKeys : kTileKeys;                   // (a weight of 0 times NaN would be NaN)
                auto widen = [&](auto all_c) {
#pragma unroll
                    for (int i0 = 0; i0 < 8; i0 += kWidenDeep) {
                        uint4 c[kWidenDeep];
#pragma unroll
                        for (int i = 0; i < kWidenDeep; ++i) {
                            const int x = (i0 + i) & 1, r0 = (i0 + i) / 2 * 8;
                            c[i] = ld_shared16(src + from_at[x] + (uint32_t)r0 * 128u);
                            if (!decltype(all_c)::value && row8[x] + r0 >= live) c[i] = make_uint4(0, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < kWidenDeep; ++i) {
                            const uint32_t to = dst + to_at[(i0 + i) & 1] + (uint32_t)((i0 + i) / 2) * 1024u;
                            uint32_t h[8];
                            widen16<kE5M2>(c[i], h);
                            st_shared16(to, h[0], h[1], h[2], h[3]);
                            st_shared16(to ^ 16u, h[4], h[5], h[6], h[7]);
                        }
                    }
                };
                if (live >= kTileKeys) widen(std::true_type()); else widen(std::false_type());
                fence_async_proxy();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&bars->codes_empty[ld % kStageBars]); mbar_arrive(&bars->full[ld % kLoadBars]); }
            }
        }
    } else {
        // ------------------------------------------------------------------ MMA issuers, a warp (one lane of it) per group
        const int g = warp - kWarpMma;
        uint32_t ld0 = 0, cg = 0, cg0 = 0, units_done = 0;              // tiles of this group, of group 0 so far
        constexpr uint32_t kHalves = ~((1u << 7) | (1u << 10));                      // A and B: half, not bf16
        constexpr uint32_t idesc_s = umma_idesc(128, 64, 0) & kHalves, idesc_o = umma_idesc(128, 128, 1) & kHalves;
        constexpr uint32_t hi_q = umma_desc_hi(1024);
        // K: K-major; V: MN-major.  8-row groups 1 KB apart, the halves of 64 dims 16 KB apart.
        constexpr uint32_t hi_kv = umma_desc_hi(1024);
        const uint32_t ring_lo = umma_desc_lo(sRing, 16), ring_lo_v = umma_desc_lo(sRing, 16384);
        constexpr uint32_t kHalfQ = 16384u >> 4, k_wide = 16384u >> 4;
        constexpr uint32_t kv_half = 8192u >> 4;                                     // keys 64..127 of a tile
        constexpr uint32_t v_step = 2048u >> 4;                                      // 16 keys of V
        const uint32_t d_s = tmem + (uint32_t)g * 128u, d_o = d_s + 256u;
        uint32_t q_lo = 0;
        auto mma_s = [&](uint32_t slot, int half) {
            const uint32_t k_lo = ring_lo + slot * (kSlotBytes >> 4) + (uint32_t)half * kv_half;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_bf16(d_s + (uint32_t)half * 64u, pack64(q_lo + (uint32_t)(ks >> 2) * kHalfQ + (uint32_t)(ks & 3) * 2u, hi_q),
                          pack64(k_lo + (uint32_t)(ks >> 2) * k_wide + (uint32_t)(ks & 3) * 2u, hi_kv), idesc_s, ks > 0);
            umma_commit(&bars->s_ready[g][half]);
        };
        bool ok = true;
        SharedUnit un;
        for (int k = 0; ok && unit_at(k, un); ++k) {
            const int T = un.tile_end - un.tile_begin;
            const bool pair = un.rows > kRowBlock;
            const int first = pair ? 0 : g, step = pair ? 1 : 2;
            q_lo = umma_desc_lo(sQ + (pair ? (uint32_t)g * 32768u : 0u), 16);
            auto release = [&](uint32_t load) {                     // once the products issued so far are through
                umma_commit(&bars->empty[load % kLoadBars]);
                if (!pair) umma_commit(&bars->empty[load % kLoadBars]);
            };
            ok = wait(&bars->q_ready, units_done & 1u);
            if (ok && first < T) {
                const uint32_t at_k = load_k(ld0, first);
                ok = landed(at_k);
                // a pair's second group starts when the first one has its first P, or soon: half a step apart the two neither compete for
                // the XU pipe nor do their products queue up behind each other (4 to 6 % of a tile)
                if (ok && pair && g == 1)
                    for (int tries = 0; tries < 64 && !mbar_test(&bars->p_ready[0][0], cg0 & 1u); ++tries) __nanosleep(20);
                __syncwarp();
                if (ok) {
                    tc_fence_after();
                    if (lane == 0) { mma_s(at_k % kSlots, 0); mma_s(at_k % kSlots, 1); release(at_k); }
                    __syncwarp();
                }
            }
            bool here = false;                                      // the tile's V has been seen
            for (int t = first; t < T && ok; t += step, ++cg) {
                const bool has_s = t + step < T;                    // the next S of a half goes out behind its P V(t)
                const uint32_t at_v = load_v(ld0, t, T), at_k = has_s ? load_k(ld0, t + step) : 0u, slot = at_v % kSlots, slot_k = at_k % kSlots;
                if (!here) ok = landed(at_v);
                here = false;
#pragma unroll 1
                for (int half = 0; half < 2 && ok; ++half) {
                    ok = wait(&bars->p_ready[g][half], cg & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (lane == 0) {
                        const uint32_t v_lo = ring_lo_v + slot * (kSlotBytes >> 4) + (uint32_t)half * kv_half, d_p = d_s + (uint32_t)half * 64u;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)              // 16 keys at a time
                            umma_bf16_ts(d_o, d_p + (uint32_t)ks * 8u, pack64(v_lo + (uint32_t)ks * v_step, hi_kv), idesc_o, ks > 0 || half > 0 || t > first);
                        if (!has_s) umma_commit(&bars->pv_done[g][half]);
                        if (half) release(at_v);
                    }
                    __syncwarp();
                    if (!has_s) continue;
                    if (half == 0) ok = landed(at_k);               // (a slot more for the loads than if both were waited for)
                    if (!ok) break;
                    if (lane == 0) {
                        mma_s(slot_k, half);
                        if (half) release(at_k);
                    }
                    __syncwarp();
                    // while the softmax warps have the second half: is the next tile's V there?
                    if (half == 0) here = landed_now(load_v(ld0, t + step, T));
                }
            }
            cg0 += pair ? T : (T + 1) >> 1;
            ld0 += 2u * T;
            ++units_done;
        }
    }
    } else {
        // ------------------------------------------------------------------ softmax groups, one thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int grp = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;                           // TMEM lane
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        const uint32_t tS = tmem + grp * 128u + lane_addr, tO = tmem + 256u + grp * 128u + lane_addr;
        uint32_t tile0 = 0, cgm = 0, units_done = 0, merges = 0;    // cgm: tiles this group has processed so far
        float* const s_lv0 = (float*)(smem + kOffLv) + grp * 64;
        uint32_t ends = 0, ends1 = 0;                               // units in which this group, group 1 has had tiles so far
        bool ok = true;
        SharedUnit un;
        for (int k = 0; ok && unit_at(k, un); ++k) {
            const int T = un.tile_end - un.tile_begin;
            const bool pair = un.rows > kRowBlock;
            const int first = pair ? 0 : grp, step_t = pair ? 1 : 2;
            const int r_u = (pair ? grp * kRowBlock : 0) + row;     // row of the unit
            const bool valid = r_u < un.rows;
            auto query = [&](int r, int& j) -> int {                // where row r of the unit has its query: (slot, head)
                const int gr = un.row0 + r;
                j = gr / a.G;
                const int slot = un.part.slot0 >= 0 ? a.slot_map[un.part.slot0 + j] : un.part.req * a.N + j;
                return slot * a.Hq + un.kvh * a.G + (gr - j * a.G);
            };
            int j = 0;
            const int qrow = valid ? query(r_u, j) : 0;
            const bool own = un.part.slot0 < 0;
            int q0 = 0, q1 = 0;
            if (own) {                                              // the tree, for its mask
                const int32_t* prow = a.parent + (size_t)un.part.req * a.N;
                q0 = lane < a.N ? prow[lane] : 0; q1 = lane + 32 < a.N ? prow[lane + 32] : 0;
            }
            const int pl = un.part.visible, L = un.part.n_keys;
            // the rows of Q that this warp brings in (half a warp a row): its own ones in a pair, sixteen of the block else
            const int rows_w = pair ? 32 : 16, row_w = pair ? grp * kRowBlock + quad * 32 : warp * 16;
            int unused, from = -1;
            if (lane < rows_w && row_w + lane < un.rows) from = query(row_w + lane, unused);
            // nobody may touch Q, O or the statistics before both groups are through with the unit before
            if (units_done > 0) {
                ok = wait(&bars->unit_done, (units_done - 1) & 1u);
                if (!ok) break;
            }
            // A row's largest magnitude fixes a power of two that puts it into [2^14, 2^15).
            float row_scale = 1.f;
#pragma unroll 4
            for (int k2 = 0; k2 < rows_w; k2 += 2) {
                const int rr = k2 + (lane >> 4), piece = lane & 15;
                const int src = __shfl_sync(0xffffffffu, from, rr);
                const uint4 x = src >= 0 ? reinterpret_cast<const uint4*>(a.q)[(size_t)src * 16 + piece] : make_uint4(0, 0, 0, 0);
                uint32_t top = max(max(mag2(x.x), mag2(x.y)), max(mag2(x.z), mag2(x.w)));          // bf16 magnitudes compare as integers
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const int e = (int)(top >> 7);                      // biased exponent of the largest
                const float f = __uint_as_float((uint32_t)(top == 0 ? 127 : min(254 + 14 - e, 254)) << 23);
                const float sc = top >= 0x7f80u ? CUDART_NAN_F : a.scale_log2 / f;                 // (NaN or infinity in the row: NaN)
                const uint32_t at = (uint32_t)(row_w + rr);         // (rows from 128 on are the second block, 32 KB behind the first)
                if (!pair && piece == 0) s_row_scale[at] = sc;
                const float s0 = __shfl_sync(0xffffffffu, sc, 0), s1 = __shfl_sync(0xffffffffu, sc, 16);
                if (lane == k2) row_scale = s0;
                if (lane == k2 + 1) row_scale = s1;
                st_shared16(sQ + (at >> 7) * 32768u + (uint32_t)(piece >> 3) * 16384u + (at & 127u) * 128u + (((uint32_t)piece & 7u) ^ (at & 7u)) * 16u,
                            halves2(x.x, f), halves2(x.y, f), halves2(x.z, f), halves2(x.w, f));
            }
            fence_async_proxy();
            warp_arrive(&bars->q_ready, lane);
            const bool warp_valid = __any_sync(0xffffffffu, valid);
            uint64_t anc = 0;
            if (own) {                                              // (the plan has looked at the tree)
                anc = warp_ancestor_mask(q0, q1, L - pl, j, lane);
                if (!valid) anc = 0;
            }
            float m_used = -CUDART_INF_F, l = 0.f;
            float v_ref = 1.f;                                      // power of two that V's scales are taken relative to
            // Half a tile.  kPlain: all of its keys are visible.
            auto step = [&](int t, int half, auto plain_c) -> bool {
                constexpr bool kPlain = decltype(plain_c)::value;
                const uint32_t tile = tile0 + (uint32_t)t, at_s = tile % kScaleTiles;
                const float* const sc = s_scale + at_s * 32u;
                float* const s_lv = s_lv0 + (cgm & 1u) * 32u;
                if (half == 0) {
                    if (!wait(&bars->scales[at_s], (tile / kScaleTiles) & 1u)) return false;
                    if (t == first && !pair) row_scale = s_row_scale[row];
                    const float sv = sc[16 + (lane & 15)];
                    if (t == first) v_ref = v_reference(sv);
                    const float rel = v_relative(sv, v_ref);
                    s_lv[lane] = lane < 16 ? v_log(rel) : rel * kWeightTop;        // (the group's four warps write the same)
                    __syncwarp();
                }
                uint32_t r[64];
                tmem_ld32(tS + half * 64, r);
                tmem_ld32(tS + half * 64 + 32, r + 32);
                tmem_wait_ld();
                if (!kPlain) {
                    // Which of its 64 keys this row sees, as a bit mask built once: the first d are prefix (all visible), key
                    // d + a is tree slot a (visible when a is the row's slot or an ancestor; the ancestor mask has no bit
                    // at or above num_nodes, so keys past the request's end are out; a shared part has no such bits).
                    const int d = pl - (un.tile_begin + t) * kTileKeys - half * 64;
                    const unsigned long long see = d >= 64 ? ~0ull : d > 0 ? ((1ull << d) - 1ull) | (anc << d) : d > -64 ? anc >> (-d) : 0ull;
                    const uint32_t w[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (!((w[e >> 5] >> (e & 31)) & 1u)) r[e] = 0xff800000u;     // -inf
                }
                float mx = -CUDART_INF_F;
#pragma unroll
                for (int g8 = 0; g8 < 8; ++g8) {                    // 8 keys with one scale: three-input max, then the scales
                    const uint32_t* x = r + g8 * 8;
                    const float m0 = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
                    const float m1 = max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5]));
                    mx = fmaxf(mx, fmaf(max3(m0, m1, fmaxf(__uint_as_float(x[6]), __uint_as_float(x[7]))), fmaxf(sc[half * 8 + g8] * row_scale, kTinyScale), s_lv[half * 8 + g8]));
                }
                // as in war_verify_attn_shared_sm100.cu (roots of factors: see half_step)
                const bool grows = mx > m_used + kRescaleThreshold || (m_used == -CUDART_INF_F && mx > -CUDART_INF_F);
                const float corr = grows ? exp2f(0.5f * (m_used - mx)) : 1.f;     // 0 when nothing was accumulated yet
                l = half_step(l, corr);
                m_used = grows ? mx : m_used;
                uint32_t pk[32];
                uint64_t sum[4] = {0, 0, 0, 0};
                const uint64_t neg_m = pair_of(m_used == -CUDART_INF_F ? 0.f : -m_used);
#pragma unroll
                for (int g8 = 0; g8 < 8; ++g8) {
                    const uint64_t ks2 = pair_of(fmaxf(sc[half * 8 + g8] * row_scale, kTinyScale)), vs2 = pair_of(s_lv[16 + half * 8 + g8]);
#pragma unroll
                    for (int e = g8 * 4; e < g8 * 4 + 4; ++e) weights2(r[2 * e], r[2 * e + 1], ks2, neg_m, vs2, sum[e & 3], pk[e]);
                }
                l += sum_of(sum[0], sum[1], sum[2], sum[3]);
                tmem_st32(tS + half * 64, pk);
                if (__any_sync(0xffffffffu, grows) && (t > first || half > 0)) {   // O of this group holds earlier keys of the unit
                    // it is stable once the products of the half before are through, which the S behind them says
                    if (half == 0 ? !wait(&bars->s_ready[grp][1], cgm & 1u)
                                  : t + step_t < T ? !wait(&bars->s_ready[grp][0], (cgm + 1) & 1u) : !wait(&bars->pv_done[grp][0], ends & 1u))
                        return false;
                    tc_fence_after();
#pragma unroll 1                                                                  // (rare: kept small)
                    for (int c = 0; c < 8; ++c) {
                        uint32_t o[16];
                        tmem_ld16(tO + c * 16, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(half_step(__uint_as_float(o[e]), corr));
                        tmem_st16(tO + c * 16, o);
                    }
                }
                tmem_wait_st();
                return true;
            };
            // Tiles of which every key is visible, then the others.  (In one loop the code of the rare tiles costs the common ones 290
            // cycles of a half tile.)
            int t = first;
            const int t_plain = pl / kTileKeys - un.tile_begin;           // local number of the first tile with a key that is not
            for (; t < min(T, t_plain) && ok; t += step_t, ++cgm) {
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    ok = wait(&bars->s_ready[grp][half], cgm & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (warp_valid) {
                        ok = step(t, half, std::true_type());
                        if (!ok) break;
                    }
                    tc_fence_before();
                    warp_arrive(&bars->p_ready[grp][half], lane);
                }
            }
            for (; t < T && ok; t += step_t, ++cgm) {
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    ok = wait(&bars->s_ready[grp][half], cgm & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (warp_valid) {
                        ok = step(t, half, std::false_type());
                        if (!ok) break;
                    }
                    tc_fence_before();
                    warp_arrive(&bars->p_ready[grp][half], lane);
                }
            }
            if (!ok) break;
            if (row_scale != row_scale) l = row_scale;
            const float w_o = normal_sum(m_used, l) * v_ref * (1.f / kWeightTop);           // what O is to be multiplied by
            const uint32_t theirs = pair ? (uint32_t)T : (uint32_t)(T + grp) >> 1;               // tiles of this unit that the other group has
            if (!pair && grp == 1) {
                stats[row] = make_float4(m_used, l, w_o, 0.f);
                warp_arrive(&bars->stats_ready, lane);
            } else {
                // epilogue: the last products, the other group's (max, sum, O) where it has the same rows, and the store
                ok = wait(&bars->pv_done[grp][1], ends & 1u);
                if (ok && !pair) {
                    ok = wait(&bars->stats_ready, merges & 1u);
                    if (ok && theirs > 0) ok = wait(&bars->pv_done[1][1], ends1 & 1u);
                }
                if (!ok) break;
                tc_fence_after();
                if (warp_valid) {
                    const bool use1 = !pair && theirs > 0;           // uniform: O of group 1 is stale when it had no tile
                    const float4 st = use1 ? stats[row] : make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
                    const float M = fmaxf(m_used, st.x);
                    const float e0 = m_used == -CUDART_INF_F ? 0.f : exp2f(m_used - M);
                    const float e1 = st.x == -CUDART_INF_F ? 0.f : exp2f(st.x - M);
                    float lsum = l * e0 + st.y * e1;
                    if (row_scale != row_scale) lsum = row_scale;
                    const float norm = un.part.whole ? (lsum == 0.f ? 0.f : 1.f / lsum) : 1.f;
                    const float f0 = e0 * w_o * norm, f1 = e1 * st.z * norm;
                    const int part_row = un.row0 + r_u;
                    float4* const part = reinterpret_cast<float4*>(a.part_o) + (size_t)un.part0 * 32 + part_row;
#pragma unroll 1                                                     // (once per unit: kept small)
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o0[32], o1[32];
                        tmem_ld32(tO + c * 32, o0);
                        if (use1) tmem_ld32(tO + 128u + c * 32, o1);
                        tmem_wait_ld();
                        float x[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            x[e] = __uint_as_float(o0[e]) * f0;
                            if (use1) x[e] = fmaf(__uint_as_float(o1[e]), f1, x[e]);
                        }
                        if (!valid) continue;
                        if (un.part.whole) {
                            uint4* dst = reinterpret_cast<uint4*>(a.out + (size_t)qrow * 128 + c * 32);
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                uint32_t w4[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const __nv_bfloat162 h = __floats2bfloat162_rn(x[v * 8 + 2 * e], x[v * 8 + 2 * e + 1]);
                                    w4[e] = *reinterpret_cast<const uint32_t*>(&h);
                                }
                                dst[v] = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                            }
                        } else {
#pragma unroll
                            for (int v = 0; v < 8; ++v) part[(size_t)(c * 8 + v) * un.part.rows] = make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]);
                        }
                    }
                    if (valid) {
                        if (un.part.whole) { if (a.lse) a.lse[qrow] = (M + log2f(lsum)) * kLn2; }
                        else *reinterpret_cast<float2*>(a.part_ml + ((size_t)un.part0 + part_row) * 2) = make_float2(M, lsum);
                    }
                }
                tc_fence_before();
            }
            warp_arrive(&bars->unit_done, lane);
            if (!pair) ++merges;
            if (first < T) ++ends;
            if (pair || T > 1) ++ends1;
            tile0 += (uint32_t)T;
            ++units_done;
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
        for (const auto kernel : {attn_shared_quant_kernel<false>, attn_shared_quant_kernel<true>})
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

}  // namespace

war_status_t war_attn_quant_launch_shared_wide(const void* q, const AttnQuantPools& pools, const int32_t* page_table, const int32_t* parent,
                                          const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                          int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int grid = war_attn_sm_count();
    if (grid <= 0) return WAR_ERR_CUDA;
    CUtensorMap k_map, v_map;
    if (!make_pool_map(&k_map, pools.k, p->num_pages, p->Hkv, p->page_size, pools.ks) ||
        !make_pool_map(&v_map, pools.v, p->num_pages, p->Hkv, p->page_size, pools.vs))
        return WAR_ERR_UNSUPPORTED;
    SharedQuantArgs a;
    a.q = (const __nv_bfloat16*)q; a.page_table = page_table; a.units = w.units; a.parts = w.parts; a.parent = parent; a.counters = w.counters; a.slot_map = w.slot_map;
    a.part_ml = w.part_ml; a.part_o = w.part_o; a.out = (__nv_bfloat16*)out; a.lse = lse; a.status_word = status_word;
    a.kscale = pools.kscale; a.vscale = pools.vscale;
    a.num_pages = p->num_pages; a.scale_log2 = p->scale * kLog2e;
    a.N = p->N; a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.page_size = p->page_size; a.max_pages = p->max_pages_per_req;
    a.page_shift = log2_of(p->page_size); a.block_shift = log2_of(pools.block); a.bpp_shift = a.page_shift - a.block_shift;
    return war_launch_behind(pools.kv == kKvE5M2 ? attn_shared_quant_kernel<true> : attn_shared_quant_kernel<false>, grid, kThreads, kSmemBytes, 1, s,
                             k_map, v_map, a);
}
