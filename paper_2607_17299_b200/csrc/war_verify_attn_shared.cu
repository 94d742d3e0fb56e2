// Attention over requests that share a prefix: argument checks, the planning kernel and the merge of the parts.
//
// With the keys of a row split into any parts, part c giving m_c = max x, l_c = sum exp2(x - m_c), O_c = sum exp2(x - m_c) v, the whole is
//     m = max m_c,   l = sum l_c exp2(m_c - m),   out = sum O_c exp2(m_c - m) / l,   lse = (m + log2 l) ln 2.
// So the prefix of a group is one part whose rows are those of all members, read once, and what each member has for itself is
// another.  The attention kernels are those of war_verify_attn and war_verify_attn_quant; only their units come from here.
#include <cuda_bf16.h>
#include <math_constants.h>
#include <mutex>
#include "war_common.cuh"
#include "war_attn_shared.cuh"
#include "war_attn_fused_plan.cuh"
#include "war_attn_quant.cuh"
#include "war_quant.cuh"

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPlanThreads = 1024;
constexpr int kSearchMaxB = 64;           // up to this many requests the chunk length is searched

__device__ __forceinline__ uint64_t shfl64(uint64_t v, int src) {
    const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)v, src);
    const uint32_t hi = __shfl_sync(0xffffffffu, (uint32_t)(v >> 32), src);
    return ((uint64_t)hi << 32) | lo;
}

// Exclusive scan of x over the block, and the sum.  Contains block barriers.
__device__ __forceinline__ int block_scan(int x, int* warp_sums, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const int y = warp_sums[lane];
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

// Exclusive scan of n numbers in shared memory, in place; returns the sum.
__device__ __forceinline__ int scan_array(int* a, int n, int* warp_sums) {
    const int per = (n + kPlanThreads - 1) / kPlanThreads, b0 = min(n, (int)threadIdx.x * per), b1 = min(n, b0 + per);
    int sum = 0, total;
    for (int q = b0; q < b1; ++q) sum += a[q];
    int run = block_scan(sum, warp_sums, &total);
    for (int q = b0; q < b1; ++q) { const int x = a[q]; a[q] = run; run += x; }
    __syncthreads();
    return total;
}

struct PlanArrays {                       // dynamic shared memory of the planning kernel, E = B + B / 2 parts
    int *tiles, *rows, *units, *part;     // [E]; units and part by position, then their exclusive scans
    int *members, *group_rows, *first;    // [B] by leader: running members, their rows, the lowest of them
    int *slots;                           // [B] by leader: first entry in slot_map
    int *shared;                          // [B] by request: keys that it shares with its group (0: none)
    uint16_t *order;                      // [E] part at each position
    uint16_t *leader, *group;             // [B]; number of the group by leader
    uint16_t *lead;                       // [B / 2] leader by number of the group
    uint8_t *n;                           // [B] validated slot count
};
__host__ __device__ inline size_t plan_arrays(PlanArrays* a, uint8_t* base, int B) {
    const int E = B + B / 2 + 4;
    size_t at = 0;
    auto take = [&](size_t bytes) { uint8_t* p = base + at; at += (bytes + 15) & ~(size_t)15; return p; };
    a->tiles = (int*)take(4 * E); a->rows = (int*)take(4 * E); a->units = (int*)take(4 * E); a->part = (int*)take(4 * E);
    a->members = (int*)take(4 * B); a->group_rows = (int*)take(4 * B); a->first = (int*)take(4 * B); a->slots = (int*)take(4 * B);
    a->shared = (int*)take(4 * B);
    a->order = (uint16_t*)take(2 * E); a->leader = (uint16_t*)take(2 * B); a->group = (uint16_t*)take(2 * B);
    a->lead = (uint16_t*)take(2 * (B / 2 + 1)); a->n = (uint8_t*)take(B);
    return at;
}

__device__ __forceinline__ int row_blocks_of(int rows) { return (rows + kRowBlock - 1) / kRowBlock; }

// One block.  Trees and groups are checked, parts are laid out, cut into chunks and dealt as in attn_plan_kernel (longest part
// first; up to 64 requests the chunk length is searched).
__global__ void __launch_bounds__(kPlanThreads)
attn_shared_plan_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ num_nodes, const int32_t* __restrict__ parent,
                        const int32_t* __restrict__ leader, const int32_t* __restrict__ shared_len, int B, int N, int Hkv, int G,
                        int page_size, int max_pages, int n_ctas, SharedWorkspace w, int* status_word) {
    extern __shared__ __align__(16) uint8_t plan_smem[];
    __shared__ int s_warp[33], s_keys[64], s_tmax;
    __shared__ long long s_sum[32];
    PlanArrays a;
    plan_arrays(&a, plan_smem, B);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s_tmax = 0;

    // ---- per request, one warp: the tree (lane l holds slots l and l + 32; pointer jumping: after round r a slot's mask covers its
    // 2^r nearest ancestors-or-self) ----
    for (int i = warp; i < B; i += 32) {
        const int j0 = lane, j1 = lane + 32;
        const int32_t* prow = parent + (size_t)i * N;
        int p0 = j0 < N ? prow[j0] : 0, p1 = j1 < N ? prow[j1] : 0, n = num_nodes[i];
        const int pl = prefix_len[i];
        const bool bad_l = (j0 > 0 && j0 < n && (p0 < 0 || p0 >= j0)) || (j1 < n && (p1 < 0 || p1 >= j1));
        bool bad = n < 0 || n > N || pl < 0;
        bad = bad || __any_sync(0xffffffffu, bad_l);
        if (bad) { if (lane == 0) war_set_device_status(status_word, WAR_ERR_BAD_TREE); n = 0; }
        if (n > 0 && (long long)pl + n > (long long)max_pages * page_size) {
            if (lane == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
            n = 0;
        }
        if (n > 0) {
            if (j0 == 0 || j0 >= n) p0 = 0;
            if (j1 >= n) p1 = 0;
            uint64_t a0 = 1ull << j0, a1 = 1ull << j1;
#pragma unroll 1
            for (int r = 1; r < n; r <<= 1) {
                const uint64_t b00 = shfl64(a0, p0 & 31), b01 = shfl64(a1, p0 & 31), b10 = shfl64(a0, p1 & 31), b11 = shfl64(a1, p1 & 31);
                const int q00 = __shfl_sync(0xffffffffu, p0, p0 & 31), q01 = __shfl_sync(0xffffffffu, p1, p0 & 31);
                const int q10 = __shfl_sync(0xffffffffu, p0, p1 & 31), q11 = __shfl_sync(0xffffffffu, p1, p1 & 31);
                a0 |= p0 >= 32 ? b01 : b00;
                a1 |= p1 >= 32 ? b11 : b10;
                p0 = p0 >= 32 ? q01 : q00;
                p1 = p1 >= 32 ? q11 : q10;
            }
            if (j0 < n) w.anc[(size_t)i * N + j0] = a0;
            if (j1 < n) w.anc[(size_t)i * N + j1] = a1;
        }
        if (lane == 0) a.n[i] = (uint8_t)n;
    }
    for (int i = tid; i < B; i += kPlanThreads) { a.members[i] = 0; a.group_rows[i] = 0; a.first[i] = B; }
    __syncthreads();

    // ---- groups: members behind their leader, then the leader itself (its shared_len does not count when it is alone) ----
    auto shares = [&](int l) -> int { return shared_len[l] / page_size * page_size; };
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = tid; i < B; i += kPlanThreads) {
            if (a.n[i] == 0) continue;
            const int l = leader[i];
            if ((l == i) != (pass == 1)) continue;
            bool ok = l >= 0 && l < B && leader[l] == l;
            if (ok && (pass == 0 || a.members[i] > 0)) ok = shared_len[l] >= 0 && shares(l) <= prefix_len[i];
            if (!ok) { war_set_device_status(status_word, WAR_ERR_INVALID_ARG); a.n[i] = 0; continue; }
            a.leader[i] = (uint16_t)l;
            atomicAdd(&a.members[l], 1);
            atomicAdd(&a.group_rows[l], G * a.n[i]);
            atomicMin(&a.first[l], i);
        }
        __syncthreads();
    }
    // ---- number of every group that shares something, its place in slot_map, its part ----
    int groups = 0, slots = 0;
    for (int i0 = 0; i0 < B; i0 += kPlanThreads) {
        const int i = i0 + tid;
        const bool active = i < B && a.members[i] >= 2 && shares(i) > 0;
        int more, more_slots;
        const int g = groups + block_scan(active ? 1 : 0, s_warp, &more);
        const int at = slots + block_scan(active ? a.group_rows[i] / G : 0, s_warp, &more_slots);
        if (i < B) a.group[i] = active ? (uint16_t)g : (uint16_t)0xffff;
        if (active) {
            a.slots[i] = at;
            a.tiles[B + g] = (shares(i) + kTileKeys - 1) / kTileKeys;
            a.rows[B + g] = a.group_rows[i];
            a.lead[g] = (uint16_t)i;
        }
        groups += more; slots += more_slots;
    }
    __syncthreads();
    const int E = B + groups;
    for (int i = tid; i < B; i += kPlanThreads) {
        const int n = a.n[i];
        SharedReq rq;
        rq.n = n; rq.group = -1; rq.row0 = 0; rq.pad = 0;
        int sh = 0;
        if (n > 0 && a.group[a.leader[i]] != 0xffff) {
            const int l = a.leader[i];
            sh = shares(l);
            int before = 0;                                                  // slots of the members before this one
            for (int q = a.first[l]; q < i; ++q) if (a.n[q] > 0 && a.leader[q] == l) before += a.n[q];
            rq.group = a.group[l]; rq.row0 = before * G;
            for (int j = 0; j < n; ++j) w.slot_map[a.slots[l] + before + j] = i * N + j;
        }
        w.reqs[i] = rq;
        a.shared[i] = sh;
        a.tiles[i] = n > 0 ? (prefix_len[i] - sh + n + kTileKeys - 1) / kTileKeys : 0;
        a.rows[i] = G * n;
    }
    __syncthreads();

    // ---- chunk length ----
    long long mine = 0;
    int t_mine = 0;
    for (int e = tid; e < E; e += kPlanThreads) { mine += (long long)a.tiles[e] * row_blocks_of(a.rows[e]); t_mine = max(t_mine, a.tiles[e]); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    t_mine = __reduce_max_sync(0xffffffffu, t_mine);
    if (lane == 0) { s_sum[warp] = mine; atomicMax(&s_tmax, t_mine); }
    __syncthreads();
    long long tot = 0;
    for (int k = 0; k < kPlanThreads / 32; ++k) tot += s_sum[k];
    tot *= Hkv;
    int chunk = (int)max((long long)kMinChunkTiles, (tot + kTargetUnits - 1) / kTargetUnits);
    const int t_max = s_tmax;
    if (B <= kSearchMaxB) {
        int* const weight = a.units;                                         // (idle until the order is known)
        for (int e = tid; e < E + 4; e += kPlanThreads) {
            weight[e] = e < E && a.tiles[e] > 0 ? Hkv * row_blocks_of(a.rows[e]) : 0;
            if (e >= E) a.tiles[e] = 0;
        }
        __syncthreads();
        chunk = fused_plan::chunk_search<kFusedThreads>(a.tiles, weight, E, max(fused_plan::chunk_floor(t_max), chunk), t_max, n_ctas, s_keys);
        __syncthreads();
    }
    auto chunks_of = [&](int t) -> int { return (t + chunk - 1) / chunk; };

    // ---- longest first; units and rows of partial results by position ----
    for (int e = tid; e < E; e += kPlanThreads) {
        const int t = a.tiles[e];
        int pos = 0;
        for (int q = 0; q < E; ++q) pos += (a.tiles[q] > t) || (a.tiles[q] == t && q < e);
        const int nc = chunks_of(t);
        a.order[pos] = (uint16_t)e;
        a.units[pos] = nc * Hkv * row_blocks_of(a.rows[e]);
        a.part[pos] = nc * Hkv * a.rows[e];
    }
    __syncthreads();
    const int total = scan_array(a.units, E, s_warp);
    scan_array(a.part, E, s_warp);
    if (tid == 0) { w.counters[1] = total; w.counters[3] = 0; }
    for (int pos = tid; pos < E; pos += kPlanThreads) {
        const int e = a.order[pos];
        SharedPart x;
        x.part0 = a.part[pos]; x.n_chunks = chunks_of(a.tiles[e]); x.rows = a.rows[e]; x.n_tiles = a.tiles[e];
        w.parts[e] = x;
    }
    // ---- unit table, one thread per unit: (chunk, kv head, row block) ----
    for (int u = tid; u < total; u += kPlanThreads) {
        int lo = 0, hi = E - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.units[mid] <= u) lo = mid; else hi = mid - 1;
        }
        const int e = a.order[lo], t = a.tiles[e], rows = a.rows[e], nc = chunks_of(t), rbs = row_blocks_of(rows);
        const int local = u - a.units[lo], c = local / (Hkv * rbs), rem = local % (Hkv * rbs);
        SharedUnit x;
        x.kvh = rem / rbs; x.rb = rem % rbs;
        x.tile_begin = (int)((long long)t * c / nc); x.tile_end = (int)((long long)t * (c + 1) / nc);
        x.rows = rows;
        x.part0 = a.part[lo] + (c * Hkv + x.kvh) * rows + x.rb * kRowBlock;
        if (e < B) {
            x.req = e; x.page0 = a.shared[e] / page_size;
            x.visible = prefix_len[e] - a.shared[e]; x.n_keys = x.visible + a.n[e];
            x.slot0 = -1; x.whole = nc == 1 && a.shared[e] == 0;
        } else {
            const int l = a.lead[e - B];
            x.req = a.first[l]; x.page0 = 0;
            x.visible = x.n_keys = shares(l);
            x.slot0 = a.slots[l]; x.whole = 0;
        }
        w.units[u] = x;
    }
}

// One warp per output row: the chunks of the group's part, then those of the request's own, in this order (results do not depend
// on timing).  Lanes first reduce the chunks' maxima, then stream their rows, float4 a lane.
constexpr int kMergeWarps = 4;
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_shared_merge_kernel(SharedWorkspace w, int B, int N, int Hq, int Hkv, int G, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    const int i = blockIdx.x / Hkv, kvh = blockIdx.x % Hkv;
    const SharedReq rq = w.reqs[i];
    const SharedPart own = w.parts[i];
    const int lane = threadIdx.x & 31, r = blockIdx.y * kMergeWarps + (threadIdx.x >> 5);
    if (r >= G * rq.n || (rq.group < 0 && own.n_chunks <= 1)) return;
    SharedPart grp{0, 0, 0, 0};
    if (rq.group >= 0) grp = w.parts[B + rq.group];
    const int n_chunks = grp.n_chunks + own.n_chunks;
    auto at = [&](int c) -> size_t {
        if (c < grp.n_chunks) return (size_t)grp.part0 + (size_t)(c * Hkv + kvh) * grp.rows + rq.row0 + r;
        return (size_t)own.part0 + (size_t)((c - grp.n_chunks) * Hkv + kvh) * own.rows + r;
    };
    float M = -CUDART_INF_F;
    for (int c = lane; c < n_chunks; c += 32) M = fmaxf(M, w.part_ml[at(c) * 2]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    float l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < n_chunks; ++c) {
        const size_t base = at(c);
        const float2 ml = *reinterpret_cast<const float2*>(w.part_ml + base * 2);
        const float4 o = *reinterpret_cast<const float4*>(w.part_o + base * 128 + lane * 4);
        const float sc = ml.x == -CUDART_INF_F ? 0.f : exp2f(ml.x - M);
        l = fmaf(ml.y, sc, l);
        acc.x = fmaf(o.x, sc, acc.x); acc.y = fmaf(o.y, sc, acc.y); acc.z = fmaf(o.z, sc, acc.z); acc.w = fmaf(o.w, sc, acc.w);
    }
    const float inv = 1.f / l;
    const int j = r / G, g = r % G;
    const size_t row = ((size_t)i * N + j) * Hq + kvh * G + g;
    const __nv_bfloat162 h0 = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), h1 = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
    uint2 packed;
    packed.x = *reinterpret_cast<const uint32_t*>(&h0);
    packed.y = *reinterpret_cast<const uint32_t*>(&h1);
    *reinterpret_cast<uint2*>(out + row * 128 + lane * 4) = packed;
    if (lse && lane == 0) lse[row] = (M + log2f(l)) * kLn2;
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
    if ((p->Hq / p->Hkv) * p->N > 512 || p->B > kMaxPlanB || (long long)p->B * p->N * p->Hq >= (1ll << 29)) return WAR_ERR_UNSUPPORTED;
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
                         const int32_t* shared_len, const war_attn_params_t* p, const SharedWorkspace& w, int* status_word, cudaStream_t s) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    const war_status_t st = device_setup(dev);
    if (st != WAR_OK) return st;
    const int n_sm = war_attn_sm_count();
    if (n_sm <= 0) return WAR_ERR_CUDA;
    PlanArrays a;
    attn_shared_plan_kernel<<<1, kPlanThreads, plan_arrays(&a, nullptr, p->B), s>>>(prefix_len, num_nodes, parent, leader, shared_len, p->B, p->N,
                                                                              p->Hkv, p->Hq / p->Hkv, p->page_size, p->max_pages_per_req,
                                                                              n_sm, w, status_word);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
}
war_status_t launch_merge(const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse, cudaStream_t s) {
    const int G = p->Hq / p->Hkv;
    attn_shared_merge_kernel<<<dim3(p->B * p->Hkv, (G * p->N + kMergeWarps - 1) / kMergeWarps), kMergeWarps * 32, 0, s>>>(
        w, p->B, p->N, p->Hq, p->Hkv, G, (__nv_bfloat16*)out, lse);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
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
    st = launch_plan(d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len, p, w, status_word, stream);
    if (st != WAR_OK) return st;
    st = war_attn_launch_sm100_shared(d_q, d_kpool, d_vpool, d_page_table, p, w, d_out, d_lse, status_word, stream);
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
    st = launch_plan(d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len, p, w, status_word, stream);
    if (st != WAR_OK) return st;
    st = war_attn_quant_launch_shared(d_q, pools, d_page_table, p, w, d_out, d_lse, status_word, stream);
    return st == WAR_OK ? launch_merge(p, w, d_out, d_lse, stream) : st;
}
