// Attention over requests that share a prefix: argument checks, the planning kernel and the merge of the parts.
//
// With the keys of a row split into any parts, part c giving m_c = max x, l_c = sum exp2(x - m_c), O_c = sum exp2(x - m_c) v, the whole is
//     m = max m_c,   l = sum l_c exp2(m_c - m),   out = sum O_c exp2(m_c - m) / l,   lse = (m + log2 l) ln 2.
// So the prefix of a group is one part whose rows are those of all members, read once, and what each member has for itself is
// another.  Their units come from here; the kernels are war_verify_attn_shared_sm100.cu (bf16 cache), war_verify_attn_quant_many.cu and
// war_verify_attn_shared_quant_sm100.cu (8-bit cache).
#include <cuda_bf16.h>
#include <math_constants.h>
#include <mutex>
#include "war_common.cuh"
#include "war_attn_shared.cuh"
#include "war_attn_quant.cuh"
#include "war_quant.cuh"

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPlanThreads = 1024;

// Exclusive scan of x over the block, and the sum.  Contains block barriers.
__device__ __forceinline__ int block_scan(int x, int* warp_sums, int n_warps, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const int y = lane < n_warps ? warp_sums[lane] : 0;
        int yi = y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int z = __shfl_up_sync(0xffffffffu, yi, o); if (lane >= o) yi += z; }
        warp_sums[lane] = yi - y;
        if (lane == 31) warp_sums[32] = yi;
    }
    __syncthreads();
    const int before = warp_sums[warp];
    *total = warp_sums[32];
    __syncthreads();
    return before + incl - x;
}

struct PlanArrays {                       // dynamic shared memory of the planning kernel, E = B + B / 2 parts
    int *tiles, *rows, *units;            // [E]; units: cost of a part's longest unit
    int *members, *group_rows, *first;    // [B] by leader: running members, their rows, the lowest of them
    int *first_unit;                      // [E] units before each position; where members and group_rows were
    int *slots;                           // [B] by leader: first entry in slot_map
    int *prefix, *shared;                 // [B] prefix_len, shared_len
    uint16_t *order, *nc;                 // [E] part at each position; chunks of a part
    uint16_t *leader, *group;             // [B]; number of the group by leader
    uint16_t *lead;                       // [B / 2] leader by number of the group
    uint8_t *n;                           // [B] validated slot count
};
__host__ __device__ inline size_t plan_arrays(PlanArrays* a, uint8_t* base, int B) {
    const int E = B + B / 2 + 4;
    size_t at = 0;
    auto take = [&](size_t bytes) { uint8_t* p = base + at; at += (bytes + 15) & ~(size_t)15; return p; };
    a->tiles = (int*)take(4 * E); a->rows = (int*)take(4 * E); a->units = (int*)take(4 * E);
    a->members = a->first_unit = (int*)take(4 * (2 * B > E ? 2 * B : E)); a->group_rows = a->members + B;
    a->first = (int*)take(4 * B); a->slots = (int*)take(4 * B);
    a->prefix = (int*)take(4 * B); a->shared = (int*)take(4 * B);
    a->order = (uint16_t*)take(2 * E); a->nc = (uint16_t*)take(2 * E); a->leader = (uint16_t*)take(2 * B); a->group = (uint16_t*)take(2 * B);
    a->lead = (uint16_t*)take(2 * (B / 2 + 1)); a->n = (uint8_t*)take(B);
    return at;
}

constexpr int kNobody = 0xffff;
constexpr int kMaxChunks = 0x7fff;
constexpr int kMinChunkCost = 4;          // tiles of one row block

// One block.  Trees and groups are checked, parts are laid out and cut into chunks.  The time of a part's tile counts 1, or 2 where two
// row blocks of 128 rows work on it together.  A chunk costs C = max(4, sqrt(36 * all / CTAs), all / kTargetUnits): smaller ones pay for
// more units (queries, first S, partial results written and merged: 12 to 18 such tiles each), larger ones for a longer tail.  (Nine shapes:
// 6 in place of 36 is 2 to 25 % slower, 100 from 3 % faster to 29 % slower; a search over 32 chunk costs by an estimate of the time was no
// better; shared and own parts in turn instead of by length: 818 us against 728 with 256 requests.)  With little work C is what makes a unit
// for every CTA, if that is less.  Units are sorted, the longest first; the CTAs draw them one by one.  Cold: 13 us for 32 requests, 23 for 256.
// A part's place is found by comparing it with all others, and a member's rows by a walk over the requests before it, so the time grows with the square
// of the requests (trees of 8 slots): 75 us for 1024 in groups of eight (91 in one group), 223 for 2048, 760 for 4096 (1270 in pairs, 970 in one group).
__global__ void __launch_bounds__(kPlanThreads)                    // (a quarter of the threads for small batches: barriers are cheaper)
attn_shared_plan_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ num_nodes, const int32_t* __restrict__ parent,
                        const int32_t* __restrict__ leader, const int32_t* __restrict__ shared_len, int B, int N, int Hkv, int G,
                        int page_size, int max_pages, int n_ctas, int block, SharedWorkspace w, int* status_word) {
    extern __shared__ __align__(16) uint8_t plan_smem[];
    war_wait_before();
    __shared__ int s_warp[33];
    __shared__ long long s_sum[32];
    PlanArrays a;
    plan_arrays(&a, plan_smem, B);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_threads = blockDim.x, n_warps = n_threads >> 5;
    auto row_blocks_of = [block](int rows) -> int { return (rows + block - 1) / block; };
    auto tile_cost = [](int rows) -> int { return rows > kRowBlock ? 2 : 1; };

    for (int i = tid; i < B; i += n_threads) {
        const int l = leader[i];
        a.leader[i] = l >= 0 && l < B ? (uint16_t)l : (uint16_t)kNobody;
        a.shared[i] = shared_len[i];
        a.members[i] = 0; a.group_rows[i] = 0; a.first[i] = B;
    }
    // ---- per request, one warp: is the tree one?  (lane l holds slots l and l + 32).  Four requests are asked for at a time: a warp
    // waits once for memory, not four times.  What a slot sees is worked out by the warps that use it (200 trees' ancestors take
    // one SM 16 thousand cycles). ----
    const int j0 = lane, j1 = lane + 32;
    for (int i0 = warp; i0 < B; i0 += 4 * n_warps) {
        int q0[4], q1[4], nn[4], pf[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + n_warps * k;
            const int32_t* prow = parent + (size_t)i * N;
            q0[k] = i < B && j0 < N ? prow[j0] : 0; q1[k] = i < B && j1 < N ? prow[j1] : 0;
            nn[k] = i < B ? num_nodes[i] : 0; pf[k] = i < B ? prefix_len[i] : 0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + n_warps * k;
            int n = nn[k];
            const bool bad_l = (j0 > 0 && j0 < n && (q0[k] < 0 || q0[k] >= j0)) || (j1 < n && (q1[k] < 0 || q1[k] >= j1));
            const bool bad = __any_sync(0xffffffffu, bad_l) || n < 0 || n > N || pf[k] < 0;
            if (lane == 0 && i < B) {
                if (bad) { war_set_device_status(status_word, WAR_ERR_BAD_TREE); n = 0; }
                if (n > 0 && (long long)pf[k] + n > (long long)max_pages * page_size) { war_set_device_status(status_word, WAR_ERR_BAD_PAGE); n = 0; }
                a.n[i] = (uint8_t)n; a.prefix[i] = pf[k];
            }
        }
    }
    __syncthreads();

    // ---- groups: members behind their leader, then the leader itself (its shared_len does not count when it is alone) ----
    auto shares = [&](int l) -> int { return a.shared[l] / page_size * page_size; };
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = tid; i < B; i += n_threads) {
            if (a.n[i] == 0) continue;
            const int l = a.leader[i];
            if ((l == i) != (pass == 1)) continue;
            bool ok = l != kNobody && a.leader[l] == l;
            if (ok && (pass == 0 || a.members[i] > 0)) ok = a.shared[l] >= 0 && shares(l) <= a.prefix[i];
            if (!ok) { war_set_device_status(status_word, WAR_ERR_INVALID_ARG); a.n[i] = 0; continue; }
            atomicAdd(&a.members[l], 1);
            atomicAdd(&a.group_rows[l], G * a.n[i]);
            atomicMin(&a.first[l], i);
        }
        __syncthreads();
    }
    // ---- number of every group that shares something, its place in slot_map, its part ----
    int groups = 0, slots = 0;
    for (int i0 = 0; i0 < B; i0 += n_threads) {
        const int i = i0 + tid;
        const bool active = i < B && a.members[i] >= 2 && shares(i) > 0;
        int both;                                                            // groups << 20 | slots (at most 2^18 in all)
        const int before = block_scan(active ? (1 << 20) + a.group_rows[i] / G : 0, s_warp, n_warps, &both);
        const int g = groups + (before >> 20);
        if (i < B) a.group[i] = active ? (uint16_t)g : (uint16_t)kNobody;
        if (active) {
            a.slots[i] = slots + (before & 0xfffff);
            a.tiles[B + g] = (shares(i) + kTileKeys - 1) / kTileKeys;
            a.rows[B + g] = a.group_rows[i];
            a.lead[g] = (uint16_t)i;
        }
        groups += both >> 20; slots += both & 0xfffff;
    }
    __syncthreads();
    const int E = B + groups;
    for (int i = tid; i < B; i += n_threads) {
        const int n = a.n[i];
        int sh = 0;
        SharedReq rq;
        rq.n = n; rq.group = -1; rq.row0 = 0; rq.pad = 0;
        if (n > 0 && a.group[a.leader[i]] != kNobody) {
            const int l = a.leader[i];
            sh = shares(l);
            int before = 0;                                                  // slots of the members before this one
#pragma unroll 4
            for (int q = a.first[l]; q < i; ++q) before += a.leader[q] == l ? (int)a.n[q] : 0;
            rq.group = a.group[l]; rq.row0 = before * G;
            for (int j = 0; j < n; ++j) w.slot_map[a.slots[l] + before + j] = i * N + j;
        }
        w.reqs[i] = rq;
        a.tiles[i] = n > 0 ? (a.prefix[i] - sh + n + kTileKeys - 1) / kTileKeys : 0;
        a.rows[i] = G * n;
    }
    __syncthreads();

    // ---- cost of a chunk ----
    long long mine = 0;
    int blocks = 0;
    for (int e = tid; e < E; e += n_threads) {
        const int rbs = row_blocks_of(a.rows[e]);
        mine += (long long)a.tiles[e] * rbs * tile_cost(min(a.rows[e], block));
        blocks += a.tiles[e] > 0 ? rbs : 0;
    }
    blocks = __reduce_add_sync(0xffffffffu, blocks);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) { s_sum[warp] = mine; s_warp[warp] = blocks; }
    __syncthreads();
    long long all = lane < n_warps ? s_sum[lane] : 0;
    blocks = __reduce_add_sync(0xffffffffu, lane < n_warps ? s_warp[lane] : 0) * Hkv;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    all *= Hkv;
    const long long least = (all + kTargetUnits - 1) / kTargetUnits;
    long long want = (long long)sqrtf(36.f * (float)all / (float)n_ctas);
    if (blocks < n_ctas) want = min(want, (all + n_ctas - blocks - 1) / (n_ctas - blocks));
    const int chunk = (int)max(max((long long)kMinChunkCost, least), want);
    // chunks of a part and the cost of the longest of them, for the order
    for (int e = tid; e < E; e += n_threads) {
        const int t = a.tiles[e], cost = tile_cost(min(a.rows[e], block)), nc = min((t * cost + chunk - 1) / chunk, min(t, kMaxChunks));
        a.nc[e] = (uint16_t)nc;
        a.units[e] = nc > 0 ? (t + nc - 1) / nc * cost : 0;
    }
    __syncthreads();

    // ---- longest first: a part's place is the number of parts in front of it, a warp each ----
    for (int e = warp; e < E; e += n_warps) {
        const int c = a.units[e];
        int before = 0;
        for (int q = lane; q < E; q += 32) before += a.units[q] > c || (a.units[q] == c && q < e);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) a.order[before] = (uint16_t)e;
    }
    __syncthreads();
    // ---- units and rows of partial results before every part; the parts ----
    int units = 0, rows_before = 0;
    for (int p0 = 0; p0 < E; p0 += n_threads) {
        const int pos = p0 + tid;
        int u = 0, r = 0, e = 0;
        if (pos < E) { e = a.order[pos]; u = a.nc[e] * Hkv * row_blocks_of(a.rows[e]); r = a.nc[e] * Hkv * a.rows[e]; }
        int u_all, r_all;
        const int u0 = units + block_scan(u, s_warp, n_warps, &u_all), r0 = rows_before + block_scan(r, s_warp, n_warps, &r_all);
        units += u_all; rows_before += r_all;
        if (pos >= E) continue;
        a.first_unit[pos] = u0;
        const int t = a.tiles[e], nc = a.nc[e];
        SharedPart x;
        x.part0 = r0; x.n_chunks = nc; x.rows = a.rows[e];
        x.each = nc > 0 ? t / nc : 0; x.more = t - x.each * nc;
        if (e < B) {
            const int l = a.leader[e], sh = a.n[e] > 0 && a.group[l] != kNobody ? shares(l) : 0;
            x.req = e; x.page0 = sh / page_size;
            x.visible = a.prefix[e] - sh; x.n_keys = x.visible + a.n[e];
            x.slot0 = -1; x.whole = nc == 1 && sh == 0;
        } else {
            const int l = a.lead[e - B];
            x.req = a.first[l]; x.page0 = 0;
            x.visible = x.n_keys = shares(l);
            x.slot0 = a.slots[l]; x.whole = 0;
        }
        x.pad = 0;
        w.parts[e] = x;
    }
    if (tid == 0) { w.counters[0] = 0; w.counters[1] = units; }
    __syncthreads();
    // ---- unit table: (chunk, kv head, row block), a thread each ----
    for (int u = tid; u < units; u += n_threads) {
        int lo = 0, hi = E - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.first_unit[mid] <= u) lo = mid; else hi = mid - 1;
        }
        const unsigned e = a.order[lo], rbs = (unsigned)row_blocks_of(a.rows[e]), local = (unsigned)(u - a.first_unit[lo]);
        const unsigned c = local / (Hkv * rbs), rem = local - c * (Hkv * rbs), h = rem / rbs;
        w.units[u] = make_uint2(e | (c << 16), h | ((rem - h * rbs) << 16));
    }
}

// A warp merges eight rows of one (request, kv head), half of the columns, four lanes a row: the chunks of the group's part, then those of
// the request's own, in this order (results do not depend on timing), each folded in as it comes.  The lanes of a row take every fourth
// piece of four columns.  Bound by HBM and L2: 80 MB of parts in 24 us, cold.
constexpr int kMergeWarps = 8;
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_shared_merge_kernel(SharedWorkspace w, int B, int N, int Hq, int Hkv, int G, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    war_wait_before();
    const int i = blockIdx.x / Hkv, kvh = blockIdx.x - i * Hkv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = (blockIdx.y * (kMergeWarps / 2) + (warp >> 1)) * 8 + (lane & 7), c0 = (warp & 1) * 16 + (lane >> 3);
    const SharedReq rq = w.reqs[i];
    const SharedPart own = w.parts[i];
    if (r - (lane & 7) >= G * rq.n || (rq.group < 0 && own.n_chunks <= 1)) return;
    const bool live = r < G * rq.n;
    int g_chunks = 0, g_part0 = 0, g_rows = 0;
    if (rq.group >= 0) { const SharedPart& g = w.parts[B + rq.group]; g_chunks = g.n_chunks; g_part0 = g.part0; g_rows = g.rows; }
    const int rr = live ? r : 0;
    float M = -CUDART_INF_F, l = 0.f;
    float4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fold = [&](int n, int part0, int rows, int row) {
        const float2* ml = reinterpret_cast<const float2*>(w.part_ml) + part0 + (size_t)kvh * rows + row;
        const float4* o = reinterpret_cast<const float4*>(w.part_o) + ((size_t)part0 + (size_t)kvh * rows) * 32 + (size_t)c0 * rows + row;
        const size_t step = (size_t)Hkv * rows;
#pragma unroll 4
        for (int c = 0; c < n; ++c, ml += step, o += step * 32) {
            const float2 y = __ldcs(ml);
            float4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __ldcs(o + (size_t)(4 * k) * rows);
            const float top = fmaxf(M, y.x);
            const float keep = M == -CUDART_INF_F ? 0.f : exp2f(M - top), sc = y.x == -CUDART_INF_F ? 0.f : exp2f(y.x - top);
            M = top;
            l = fmaf(l, keep, y.y * sc);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc[k].x = fmaf(acc[k].x, keep, x[k].x * sc); acc[k].y = fmaf(acc[k].y, keep, x[k].y * sc);
                acc[k].z = fmaf(acc[k].z, keep, x[k].z * sc); acc[k].w = fmaf(acc[k].w, keep, x[k].w * sc);
            }
        }
    };
    fold(g_chunks, g_part0, g_rows, rq.row0 + rr);
    fold(own.n_chunks, own.part0, own.rows, rr);
    if (!live) return;
    const float inv = 1.f / l;
    const int j = r / G, g = r - j * G;
    const size_t at = ((size_t)i * N + j) * Hq + kvh * G + g;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h0 = __floats2bfloat162_rn(acc[k].x * inv, acc[k].y * inv), h1 = __floats2bfloat162_rn(acc[k].z * inv, acc[k].w * inv);
        uint2 packed;
        packed.x = *reinterpret_cast<const uint32_t*>(&h0);
        packed.y = *reinterpret_cast<const uint32_t*>(&h1);
        *reinterpret_cast<uint2*>(out + at * 128 + (c0 + 4 * k) * 4) = packed;
    }
    if (lse && c0 == 0) lse[at] = (M + log2f(l)) * kLn2;
}

constexpr int kMaxDevices = 64;
std::once_flag g_dev_once[kMaxDevices];
war_status_t g_dev_status[kMaxDevices];

war_status_t device_setup(int dev) {
    std::call_once(g_dev_once[dev], [dev]() {
        PlanArrays a;
        g_dev_status[dev] = cudaFuncSetAttribute(attn_shared_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)plan_arrays(&a, nullptr, kMaxPlanB)) == cudaSuccess ? WAR_OK : WAR_ERR_CUDA;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    return g_dev_status[dev];
}

// What both caches have in common; the layouts of the pools are looked at by the callers.
war_status_t check_shape(const war_attn_params_t* p) {
    if (p->B < 0 || p->N < 1 || p->N > 64 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->max_pages_per_req < 0 ||
        p->num_pages < 0 || p->kernel != 0 || !(p->scale > 0.f))
        return WAR_ERR_INVALID_ARG;
    if (p->D != 128 || (p->page_size != 8 && p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128))
        return WAR_ERR_UNSUPPORTED;
    // (a unit's record has 16 bits for the kv head; rows of partial results are counted in 32)
    if ((p->Hq / p->Hkv) * p->N > 512 || p->B > kMaxPlanB || p->Hkv > 65535 || (long long)p->B * p->N * p->Hq >= (1ll << 29)) return WAR_ERR_UNSUPPORTED;
    if ((long long)p->max_pages_per_req * p->page_size >= (1ll << 30)) return WAR_ERR_UNSUPPORTED;    // contexts below 2^30 tokens
    return WAR_OK;
}
war_status_t check_bf16(const war_attn_params_t* p) {
    if (!p) return WAR_ERR_INVALID_ARG;
    const war_status_t st = check_shape(p);
    if (st != WAR_OK) return st;
    const int layout = war_attn_pool_layout(p->k_strides, p);
    return layout < 0 || war_attn_pool_layout(p->v_strides, p) != layout ? WAR_ERR_UNSUPPORTED : WAR_OK;
}

war_status_t check_quant(const war_attn_quant_params_t* q) {
    if (!q) return WAR_ERR_INVALID_ARG;
    const war_attn_params_t* p = &q->attn;
    const war_status_t st = check_shape(p);
    if (st != WAR_OK) return st;
    if (q->kv_type != kKvE4M3 && q->kv_type != kKvE5M2) return WAR_ERR_INVALID_ARG;
    return war_quant_block_ok(p->page_size, q->scale_block) && war_rows_aligned(p->k_strides, 1) && war_rows_aligned(p->v_strides, 1)
               ? WAR_OK : WAR_ERR_UNSUPPORTED;
}

war_status_t launch_plan(const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* parent, const int32_t* leader,
                         const int32_t* shared_len, const war_attn_params_t* p, int block, const SharedWorkspace& w, int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int n_sm = war_attn_sm_count();
    if (n_sm <= 0) return WAR_ERR_CUDA;
    PlanArrays a;
    return war_launch_behind(attn_shared_plan_kernel, 1, p->B <= 128 ? kPlanThreads / 4 : kPlanThreads, plan_arrays(&a, nullptr, p->B), 1, s, prefix_len,
                             num_nodes, parent, leader, shared_len, p->B, p->N, p->Hkv, p->Hq / p->Hkv, p->page_size, p->max_pages_per_req, n_sm,
                             block, w, status_word);
}
war_status_t launch_merge(const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse, cudaStream_t s) {
    const int G = p->Hq / p->Hkv;
    return war_launch_behind(attn_shared_merge_kernel, dim3(p->B * p->Hkv, (G * p->N + kMergeWarps * 4 - 1) / (kMergeWarps * 4)), kMergeWarps * 32, 0, 1,
                             s, w, p->B, p->N, p->Hq, p->Hkv, G, (__nv_bfloat16*)out, lse);
}

}  // namespace

extern "C" size_t war_verify_attn_shared_workspace_bytes(const war_attn_params_t* p) {
    return check_bf16(p) == WAR_OK ? war_attn_shared_layout(p, nullptr).bytes : 0;
}

extern "C" war_status_t war_verify_attn_shared(const void* d_q, const void* d_kpool, const void* d_vpool, const int32_t* d_page_table,
                                               const int32_t* d_prefix_len, const int32_t* d_num_nodes, const int32_t* d_parent,
                                               const int32_t* d_leader, const int32_t* d_shared_len, const war_attn_params_t* p,
                                               void* d_workspace, void* d_out, float* d_lse, war_stream_t stream) {
    war_status_t st = check_bf16(p);
    if (st != WAR_OK) return st;
    if (p->B == 0) return WAR_OK;
    if (!d_q || !d_kpool || !d_vpool || !d_page_table || !d_prefix_len || !d_num_nodes || !d_parent || !d_leader || !d_shared_len ||
        !d_workspace || !d_out || p->num_pages == 0)
        return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_q | (uintptr_t)d_out) & 15) || (((uintptr_t)d_kpool | (uintptr_t)d_vpool) & 127))
        return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    const SharedWorkspace w = war_attn_shared_layout(p, d_workspace);
    st = launch_plan(d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len, p, kSharedBlock, w, status_word, stream);
    if (st != WAR_OK) return st;
    st = war_attn_shared_launch(d_q, d_kpool, d_vpool, d_page_table, d_parent, p, w, d_out, d_lse, status_word, stream);
    return st == WAR_OK ? launch_merge(p, w, d_out, d_lse, stream) : st;
}

extern "C" size_t war_verify_attn_shared_quant_workspace_bytes(const war_attn_quant_params_t* qp) {
    return check_quant(qp) == WAR_OK ? war_attn_shared_layout(&qp->attn, nullptr).bytes : 0;
}

extern "C" war_status_t war_verify_attn_shared_quant(const void* d_q, const void* d_kpool, const void* d_vpool, const float* d_kscale,
                                                     const float* d_vscale, const int32_t* d_page_table, const int32_t* d_prefix_len,
                                                     const int32_t* d_num_nodes, const int32_t* d_parent, const int32_t* d_leader,
                                                     const int32_t* d_shared_len, const war_attn_quant_params_t* qp, void* d_workspace,
                                                     void* d_out, float* d_lse, war_stream_t stream) {
    war_status_t st = check_quant(qp);
    if (st != WAR_OK) return st;
    const war_attn_params_t* p = &qp->attn;
    if (p->B == 0) return WAR_OK;
    if (!d_q || !d_kpool || !d_vpool || !d_kscale || !d_vscale || !d_page_table || !d_prefix_len || !d_num_nodes || !d_parent ||
        !d_leader || !d_shared_len || !d_workspace || !d_out || p->num_pages == 0)
        return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_q | (uintptr_t)d_out | (uintptr_t)d_kpool | (uintptr_t)d_vpool) & 15))
        return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    AttnQuantPools pools;
    pools.k = (const uint8_t*)d_kpool; pools.v = (const uint8_t*)d_vpool; pools.kscale = d_kscale; pools.vscale = d_vscale;
    for (int i = 0; i < 3; ++i) { pools.ks[i] = p->k_strides[i]; pools.vs[i] = p->v_strides[i]; }
    pools.kv = qp->kv_type; pools.block = qp->scale_block;
    const SharedWorkspace w = war_attn_shared_layout(p, d_workspace);
    const bool wide = p->Hq / p->Hkv * p->N > kQuantWideRows;
    st = launch_plan(d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len, p, wide ? kSharedBlock : kSharedQuantBlock, w, status_word, stream);
    if (st != WAR_OK) return st;
    st = (wide ? war_attn_quant_launch_shared_wide : war_attn_quant_launch_shared)(d_q, pools, d_page_table, d_parent, p, w, d_out, d_lse, status_word, stream);
    return st == WAR_OK ? launch_merge(p, w, d_out, d_lse, stream) : st;
}
