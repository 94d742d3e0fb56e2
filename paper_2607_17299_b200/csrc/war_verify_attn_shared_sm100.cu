// Tensor-core attention over shared prefixes for sm_100a, bf16 cache: TMA-staged pages -> tcgen05.mma -> online softmax -> tcgen05.mma,
// one persistent CTA per SM, units from war_verify_attn_shared.cu.
//
// What bounds it.  The prefix of a group is read once but multiplied with the rows of all members, so a shared part of more than 128
// rows is bound by the SM, not by memory.  Per 128 rows x 128 keys: S = Q K^T and P V take 512 cycles of the tensor pipe each, the 16384
// exponentials 1024 of the XU pipe, and shared memory gives the operands at 128 bytes a cycle.  The kernel of
// war_verify_attn takes 2050 cycles there: every tile waits for its S, the tensor pipe for its P (tensor and XU pipes half busy).  Here
//   * a tile is worked on in halves of 64 keys: while a group's softmax warps have one half, P V and the next S of the other are on the
//     tensor cores, so the warps find their next S ready;
//   * a unit has up to 256 rows: two groups of softmax warps with a block of 128 rows each on the same K and V tiles (half the copies
//     into shared memory, half the reads from L2).  With at most 128 rows (a request by itself, a small group), where memory is the bound,
//     the groups take the tiles in turn and their results are merged, as in war_verify_attn.
// Warp roles:  warps 8 and 11  producers (TMA copies of this GPU's own memory into a ring of 32 KB slots)
//              warps 9 and 10  MMA issuers, one lane each, for softmax group 0 and 1
//              warps 0-3, 4-7  softmax groups: one thread a row; P goes back into the first columns of its half of S
// Measured: a half tile of both groups 1735 cycles (tensor pipe 50 %, XU 47 %); 4 prompts of 16K to 32K tokens with 7 rollouts of 32 slots and 4
// requests alone, 32 + 8 heads: 525 us the call (each for itself 567); 32 prompts of 6K to 16K tokens with 8 rollouts of 8 slots: 710 to
// 725 us (1530), 60 % of the HBM bandwidth; floors 246 and 445.
// Layouts of tiles, loads in the order K0 K1 V0 K2 V1 ..., bounded waits: as in war_verify_attn_sm100.cu.
#include <mutex>
#include <type_traits>
#include "war_attn_sm100_parts.cuh"
#include "war_attn_shared.cuh"

namespace {

constexpr int kSlots = 5;
constexpr int kSlotBytes = 32768;
constexpr int kLoadBars = 8;
constexpr int kThreads = 384;
constexpr int kRegsSoftmax = 216, kRegsOther = 72;                  // register budgets after the hand-over below
constexpr int kWarpLoad0 = 8, kWarpMma = 9, kWarpLoad1 = 11;        // (group g's issuer is warp kWarpMma + g)
constexpr uint32_t kTmemCols = 512;
constexpr int kAhead = 2;                                           // units whose numbers a CTA holds
constexpr float kRescaleThreshold = 8.0f;                           // log2 units

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int kOffQ = 0;                                            // two blocks of 128 rows
constexpr int kOffRing = 65536;
constexpr int kOffBar = kOffRing + kSlots * kSlotBytes;
constexpr int kOffStats = kOffBar + 512;
constexpr int kSmemBytes = kOffStats + 1024 + 1024;
static_assert(kSmemBytes <= 232448, "shared memory");
static_assert(kThreads * 168 >= 256 * kRegsSoftmax + 128 * kRegsOther, "the hand-over draws on the registers of the launch");

struct Bars {
    uint64_t full[kLoadBars];                                       // two arrivals, one of each producer
    uint64_t empty[kLoadBars];                                      // two arrivals, one of each issuer or both of one
    uint64_t s_ready[2][2], p_ready[2][2];                          // [group][half of a tile]
    uint64_t pv_done[2][2];                                         // of a group's last tile in a unit (else the next S says it)
    uint64_t q_ready, stats_ready, unit_done;
    uint64_t next_full[kAhead], next_free[kAhead];                  // numbers of the CTA's units, in the order they are run
    int next[kAhead];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// Load n of the CTA (see load_k) goes into ring slot n % 5.  Its barriers are number n % 8: with more barriers than loads in flight a
// parity tells a load's phase from any other that can be asked for.

// Two elements of a softmax row: P = exp2(x * scale - m) as packed bf16, added to a pair of sums in 32 bits.  Written as one
// block of packed 32-bit instructions: with the intrinsics the same instructions take 13 % longer (two groups, 64 columns: 1318 cycles
// against 1162; the exponentials alone are 1024).
__device__ __forceinline__ void weights2(uint32_t x0, uint32_t x1, uint64_t scale2, uint64_t neg_m2, uint64_t& sum2, uint32_t& packed) {
    asm("{\n.reg .b64 x, y;\n.reg .f32 a, b;\n"
        "mov.b64 x, {%2, %3};\n"
        "fma.rn.f32x2 x, x, %4, %5;\n"
        "mov.b64 {a, b}, x;\n"
        "ex2.approx.ftz.f32 a, a;\n"
        "ex2.approx.ftz.f32 b, b;\n"
        "mov.b64 y, {a, b};\n"
        "add.rn.f32x2 %1, %1, y;\n"
        "cvt.rn.bf16x2.f32 %0, b, a;\n}\n"
        : "=r"(packed), "+l"(sum2) : "r"(x0), "r"(x1), "l"(scale2), "l"(neg_m2));
}

struct KernelArgs {
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
    long long num_pages;
    float scale_log2;
    int N, Hq, Hkv, G, page_size, max_pages;
};

template <bool kTokenMajor>
__global__ void __launch_bounds__(kThreads, 1)
attn_shared_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const KernelArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars* bars = (Bars*)(smem + kOffBar);
    float2* stats = (float2*)(smem + kOffStats);                    // group 1's (max, sum) per row, where the groups share rows
    const uint32_t sQ = smem_u32(smem + kOffQ), sRing = smem_u32(smem + kOffRing);
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
    const uint32_t page_bytes = (uint32_t)a.page_size * 256u;

    if (tid == 0) {
        for (int i = 0; i < kLoadBars; ++i) { mbar_init(&bars->full[i], 2); mbar_init(&bars->empty[i], 2); }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bars->s_ready[0][i], 1); mbar_init(&bars->p_ready[0][i], 4); mbar_init(&bars->pv_done[0][i], 1);
        }
        mbar_init(&bars->q_ready, 8);
        mbar_init(&bars->stats_ready, 4);
        mbar_init(&bars->unit_done, 8);
        for (int i = 0; i < kAhead; ++i) { mbar_init(&bars->next_full[i], 1); mbar_init(&bars->next_free[i], 11); }
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
        // would not do here: with five slots the one could get two rounds ahead of the other, and parities would mislead it.)
        const int half = warp == kWarpLoad1;
        const int piece = 2 * lane + half;                          // this lane's page of a tile
        uint32_t ld = 0;
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
            auto load = [&](int t, int page, bool is_v) -> bool {
                const uint32_t slot = ld % kSlots, was = ld - kSlots;        // (the load that had the slot)
                uint64_t* const full = &bars->full[ld % kLoadBars];
                const bool first_round = ld < (uint32_t)kSlots;
                ++ld;
                if (!first_round && !wait(&bars->empty[was % kLoadBars], (was / kLoadBars) & 1u)) return false;
                const int n_valid = min(pages_per_tile, total_pages - (un.tile_begin + t) * pages_per_tile);
                if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)((n_valid + 1 - half) >> 1) * page_bytes);
                __syncwarp();
                if (piece < n_valid) {
                    long long pg = page;
                    if (pg < 0 || pg >= a.num_pages) { war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE); pg = 0; }
                    const CUtensorMap* map = is_v ? &v_map : &k_map;
                    if (!kTokenMajor) tma_load_block(sRing + slot * kSlotBytes + piece * page_bytes, map, (int)(pg * a.Hkv + un.kvh), full);
                    else {
                        const uint32_t dst = sRing + slot * kSlotBytes + piece * (page_bytes >> 1);
                        tma_load_half_page(dst, map, 0, un.kvh, (int)pg, full);
                        tma_load_half_page(dst + 16384u, map, 64, un.kvh, (int)pg, full);
                    }
                }
                return true;
            };
            int pg_cur = page_of(0), pg_nxt = page_of(1);
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
                const int pg_nn = page_of(t + 2);                   // page ids two tiles ahead, off the critical path
                if (t + 1 < T) ok = load(t + 1, pg_nxt, false);     // K(t+1)
                if (ok) ok = load(t, pg_cur, true);                 // V(t)
                pg_cur = pg_nxt; pg_nxt = pg_nn;
            }
        }
    } else {
        // ------------------------------------------------------------------ MMA issuers, a warp (one lane of it) per group
        const int g = warp - kWarpMma;
        uint32_t ld0 = 0, cg = 0, cg0 = 0, units_done = 0;              // tiles of this group, of group 0 so far
        constexpr uint32_t idesc_s = umma_idesc(128, 64, 0), idesc_o = umma_idesc(128, 128, 1);
        constexpr uint32_t hi_q = umma_desc_hi(1024);
        // K: K-major; V: MN-major.  Head-major tiles: 8-row groups 2 KB apart, the 64-wide halves 1 KB apart.
        // Token-major tiles: 8-row groups 1 KB apart, the halves 16 KB apart.
        const uint32_t hi_kv = kTokenMajor ? umma_desc_hi(1024) : umma_desc_hi(2048);
        const uint32_t ring_lo = umma_desc_lo(sRing, 16), ring_lo_v = umma_desc_lo(sRing, kTokenMajor ? 16384 : 1024);
        constexpr uint32_t kHalfQ = 16384u >> 4;
        constexpr uint32_t k_wide = (kTokenMajor ? 16384u : 1024u) >> 4;             // second 64 dims of K
        constexpr uint32_t kv_half = (kTokenMajor ? 8192u : 16384u) >> 4;            // keys 64..127 of a tile
        constexpr uint32_t v_step = (kTokenMajor ? 2048u : 4096u) >> 4;              // 16 keys of V
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
            bool here = false;                                      // the tile's loads have been seen
            for (int t = first; t < T && ok; t += step, ++cg) {
                const bool has_s = t + step < T;                    // the next S of a half goes out behind its P V(t)
                const uint32_t at_v = load_v(ld0, t, T), at_k = has_s ? load_k(ld0, t + step) : 0u, slot = at_v % kSlots, slot_k = at_k % kSlots;
                if (!here) ok = landed(at_v) && (!has_s || landed(at_k));
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
                        if (has_s) {
                            mma_s(slot_k, half);
                            if (half) release(at_k);
                        }
                    }
                    __syncwarp();
                    // while the softmax warps have the second half: are the next tile's loads there?
                    if (half == 0 && has_s) here = landed_now(load_v(ld0, t + step, T)) && (t + 2 * step >= T || landed_now(load_k(ld0, t + 2 * step)));
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
        uint32_t ld0 = 0, cgm = 0, units_done = 0, merges = 0;      // cgm: tiles this group has processed so far
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
#pragma unroll 4
            for (int k2 = 0; k2 < rows_w; k2 += 2) {
                const int rr = k2 + (lane >> 4), piece = lane & 15;
                const int src = __shfl_sync(0xffffffffu, from, rr);
                const uint4 x = src >= 0 ? reinterpret_cast<const uint4*>(a.q)[(size_t)src * 16 + piece] : make_uint4(0, 0, 0, 0);
                const uint32_t at = (uint32_t)(row_w + rr);         // (rows from 128 on are the second block, 32 KB behind the first)
                st_shared16(sQ + (at >> 7) * 32768u + (uint32_t)(piece >> 3) * 16384u + (at & 127u) * 128u + (((uint32_t)piece & 7u) ^ (at & 7u)) * 16u, x.x, x.y, x.z, x.w);
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
            // Half a tile.  kPlain: all of its keys are visible.
            auto step = [&](int t, int half, auto plain_c) -> bool {
                constexpr bool kPlain = decltype(plain_c)::value;
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
                float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int e = 0; e < 64; e += 8)
#pragma unroll
                    for (int v = 0; v < 4; ++v) mx4[v] = max3(mx4[v], __uint_as_float(r[e + 2 * v]), __uint_as_float(r[e + 2 * v + 1]));
                const float mx = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]) * a.scale_log2;        // scale > 0
                // The reference grows rarely.  Up to the store of P every half is one run of instructions without a branch; what O
                // needs comes behind it.  (In front of the weights it costs every half 280 cycles.)
                const bool grows = mx > m_used + kRescaleThreshold || (m_used == -CUDART_INF_F && mx > -CUDART_INF_F);
                const float corr = grows ? exp2f(m_used - mx) : 1.f;              // 0 when nothing was accumulated yet
                l *= corr;
                m_used = grows ? mx : m_used;
                uint32_t pk[32];
                uint64_t sum[4] = {0, 0, 0, 0};
                const uint64_t scale2 = pair_of(a.scale_log2), neg_m = pair_of(m_used == -CUDART_INF_F ? 0.f : -m_used);
#pragma unroll
                for (int e = 0; e < 32; ++e) weights2(r[2 * e], r[2 * e + 1], scale2, neg_m, sum[e & 3], pk[e]);
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
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
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
                const int key0 = (un.tile_begin + t) * kTileKeys;
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    ok = wait(&bars->s_ready[grp][half], cgm & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (warp_valid) {
                        ok = step(t, half, std::false_type());
                        if (!ok) break;
                    }
                    // the unit's last tile may hold rows past the part's last key: zero their V (P is exactly 0 there, but 0 x NaN
                    // garbage would still poison the product)
                    if (half == 0 && key0 + kTileKeys > L) {
                        const uint32_t at_v = load_v(ld0, t, T), slot = at_v % kSlots;
                        ok = landed(at_v);
                        if (!ok) break;
                        if (row >= L - key0) {
                            const uint32_t base = sRing + slot * kSlotBytes +
                                                  (kTokenMajor ? (uint32_t)row * 128u : (uint32_t)(row >> 3) * 2048u + (uint32_t)(row & 7) * 128u);
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int c = 0; c < 8; ++c) st_shared16(base + h * (kTokenMajor ? 16384u : 1024u) + c * 16u, 0, 0, 0, 0);
                        }
                        fence_async_proxy();
                    }
                    tc_fence_before();
                    warp_arrive(&bars->p_ready[grp][half], lane);
                }
            }
            if (!ok) break;
            const uint32_t theirs = pair ? (uint32_t)T : (uint32_t)(T + grp) >> 1;               // tiles of this unit that the other group has
            if (!pair && grp == 1) {
                stats[row] = make_float2(m_used, l);
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
                    const float2 st = use1 ? stats[row] : make_float2(-CUDART_INF_F, 0.f);
                    const float M = fmaxf(m_used, st.x);
                    const float w0 = m_used == -CUDART_INF_F ? 0.f : exp2f(m_used - M);
                    const float w1 = st.x == -CUDART_INF_F ? 0.f : exp2f(st.x - M);
                    const float lsum = l * w0 + st.y * w1;
                    const float norm = un.part.whole ? (lsum > 0.f ? 1.f / lsum : 0.f) : 1.f;
                    const float f0 = w0 * norm, f1 = w1 * norm;
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
            ld0 += 2u * T;
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
        for (const auto kernel : {attn_shared_kernel<false>, attn_shared_kernel<true>})
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

}  // namespace

war_status_t war_attn_shared_launch(const void* q, const void* k, const void* v, const int32_t* page_table, const int32_t* parent,
                                    const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                    int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int grid = war_attn_sm_count();
    if (grid <= 0) return WAR_ERR_CUDA;
    const int token_major = war_attn_pool_layout(p->k_strides, p) == 1;
    CUtensorMap k_map, v_map;
    if (!make_pool_map(&k_map, k, p->num_pages, p->Hkv, p->page_size, token_major) ||
        !make_pool_map(&v_map, v, p->num_pages, p->Hkv, p->page_size, token_major))
        return WAR_ERR_UNSUPPORTED;
    KernelArgs a;
    a.q = (const __nv_bfloat16*)q; a.page_table = page_table; a.units = w.units; a.parts = w.parts; a.parent = parent; a.counters = w.counters; a.slot_map = w.slot_map;
    a.part_ml = w.part_ml; a.part_o = w.part_o; a.out = (__nv_bfloat16*)out; a.lse = lse; a.status_word = status_word;
    a.num_pages = p->num_pages; a.scale_log2 = p->scale * kLog2e;
    a.N = p->N; a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.page_size = p->page_size; a.max_pages = p->max_pages_per_req;
    return war_launch_behind(token_major ? attn_shared_kernel<true> : attn_shared_kernel<false>, grid, kThreads, kSmemBytes, 1, s, k_map, v_map, a);
}
