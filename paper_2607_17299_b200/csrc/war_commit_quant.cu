// Commit for the 8-bit cache: the accepted slots' rows move behind the root, as in war_commit, and because a row's codes
// mean something only under its block's scale, a row that comes from a block with another scale is re-encoded.
//
// A block that receives rows gets the largest scale among the blocks its live rows come from (its own, if rows stay in
// it), so nothing saturates; with the powers of two the store chooses, re-encoding for a larger scale is exact down to the
// type's smallest normal number.
//
// A step moves a few kilobytes a request, so what counts is the length of the chain page table -> scale -> row -> write
// and the number of launches (8 requests of up to 16 slots 7.0 us, 256 of up to 32 slots 11.3 us, 6 MB, the kernel alone; one
// launch, where war_commit makes two).  One cluster of thread blocks per request: its warps take one (head, K or V) each, lanes
// hold the scales of the blocks that can be involved (at most ten in a row), sixteen rows are in flight at a time; after a
// cluster barrier (everybody has read prefix_len) the first block advances the context.
#include <cooperative_groups.h>
#include "war_common.cuh"
#include "war_quant.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kMaxSlots = 64;
constexpr int kMaxTail = 32;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct CommitArgs {
    const int32_t *ids, *accept_len, *accept_path, *bonus, *page_table;
    uint8_t *kpool, *vpool;
    float *kscale, *vscale;
    int32_t *prefix_len, *tail, *tail_len;
    int* status_word;
    long long ks[3], vs[3];                   // pool strides (page, head, token) in elements
    long long num_pages;
    int N, P, Hkv, page_size, max_pages, block, block_shift, blocks_per_page;     // block: a power of two
};

__global__ void __launch_bounds__(kThreads)
war_commit_quant_kernel(const CommitArgs a, const int kv) {
    cg::cluster_group cluster = cg::this_cluster();
    const int part = (int)cluster.block_rank(), parts = (int)cluster.num_blocks();
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int k = a.accept_len[b], pl = a.prefix_len[b], tl = a.tail_len[b], bn = a.bonus[b];
    const int32_t* path = a.accept_path + (size_t)b * a.N;
    // Every warp checks the request for itself: accept_len in [0, N), slots strictly increasing inside [1, N), all rows
    // inside the page table.  Lane l holds path entries l and l + 32.
    const int s0 = lane < a.N ? path[lane] : 0, s1 = lane + 32 < a.N ? path[lane + 32] : 0;
    bool wrong = k < 0 || k >= a.N || pl < 0 || tl > a.P;
    {
        int before0 = __shfl_up_sync(0xffffffffu, s0, 1), before1 = __shfl_up_sync(0xffffffffu, s1, 1);
        const int mid = __shfl_sync(0xffffffffu, s0, 31);
        if (lane == 0) { before0 = 0; before1 = mid; }
        wrong = wrong || (lane < k && (s0 <= before0 || s0 >= a.N)) || (lane + 32 < k && (s1 <= before1 || s1 >= a.N));
    }
    wrong = __any_sync(0xffffffffu, wrong);
    auto slot_of = [&](int d) -> int {                                    // path[d], d uniform or per lane; all lanes call it
        const int x = __shfl_sync(0xffffffffu, s0, d & 31), y = __shfl_sync(0xffffffffu, s1, d & 31);
        return d >= 32 ? y : x;
    };
    const int last = !wrong && k > 0 ? slot_of(k - 1) : 0;
    if (!wrong && k > 0 && ((long long)pl + last) / a.page_size >= a.max_pages) wrong = true;
    const bool running = tl >= 0;

    if (running && !wrong && k > 0) {
        const int32_t* pt = a.page_table + (size_t)b * a.max_pages;
        const int fb = (pl + 1) >> a.block_shift;                                // first block that can receive a row
        const int n_blocks = ((pl + last) >> a.block_shift) - fb + 1;              // blocks that hold sources or destinations: at most 10
        // lane l: page and place of block fb + l
        long long page = -1;
        if (lane < n_blocks) page = pt[(int)((long long)(fb + lane) * a.block / a.page_size)];
        const bool page_ok = page >= 0 && page < a.num_pages;
        if (lane < n_blocks && !page_ok && part == 0 && warp == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
        const int row_in_page = lane < n_blocks ? (int)((long long)(fb + lane) * a.block % a.page_size) : 0;
        const int t_last = ((pl + k) >> a.block_shift) - fb;              // last block that receives a row
        // lane l: source and destination block of the path's slots l and l + 32
        const int from0 = lane < k ? ((pl + s0) >> a.block_shift) - fb : 0, to0 = lane < k ? ((pl + 1 + lane) >> a.block_shift) - fb : -1;
        const int from1 = lane + 32 < k ? ((pl + s1) >> a.block_shift) - fb : 0, to1 = lane + 32 < k ? ((pl + 33 + lane) >> a.block_shift) - fb : -1;
        for (int task = part * kWarps + warp; task < 2 * a.Hkv; task += parts * kWarps) {
            const int which = task & 1, h = task >> 1;
            const long long* st = which ? a.vs : a.ks;
            uint8_t* pool = which ? a.vpool : a.kpool;
            float* scale_p = (which ? a.vscale : a.kscale) + ((page_ok ? page : 0) * a.Hkv + h) * a.blocks_per_page + (row_in_page >> a.block_shift);
            const float scale = page_ok && lane < n_blocks ? *scale_p : 0.f;
            const long long base = page_ok ? page * st[0] + h * st[1] + (long long)row_in_page * st[2] : -1;
            // new scale of every receiving block: the largest among the blocks its live rows come from
            float s_new = lane == 0 && ((pl + 1) & (a.block - 1)) != 0 ? scale : 0.f;        // rows up to the root stay where they are
            const float a0 = __shfl_sync(0xffffffffu, scale, from0), a1 = __shfl_sync(0xffffffffu, scale, from1);    // (0 for a block whose page is bad)
            for (int t = 0; t <= t_last; ++t) {
                // (scales are not negative: ordered as whole numbers)
                const uint32_t m = max(to0 == t && a0 > 0.f ? __float_as_uint(a0) : 0u, to1 == t && a1 > 0.f ? __float_as_uint(a1) : 0u);
                const float top = __uint_as_float(__reduce_max_sync(0xffffffffu, m));
                if (lane == t) s_new = fmaxf(s_new, top);
            }
            if (!(s_new > 0.f)) s_new = scale;
            // rows that stay in a block whose scale has grown: those up to the root, and accepted slots already in place
            for (int t = 0; t <= t_last; ++t) {
                const float so = __shfl_sync(0xffffffffu, scale, t), sn = __shfl_sync(0xffffffffu, s_new, t);
                const long long at = __shfl_sync(0xffffffffu, base, t);
                if (at < 0 || sn == so) continue;
                const float ratio = so / sn;
                const int pos0 = (fb + t) * a.block;
                const int end = min(a.block, pl + k + 1 - pos0);
                for (int r0 = 0; r0 < end; r0 += 4) {
                    const int r = r0 + (lane >> 3), d = pos0 + r - pl - 1;
                    const int slot = slot_of(min(max(d, 0), kMaxSlots - 1));
                    if (r < end && (d < 0 || slot == d + 1)) {
                        uint4* p = reinterpret_cast<uint4*>(pool + at + r * st[2]) + (lane & 7);
                        const uint4 x = *p;
                        const uint2 lo = quant::recode8(make_uint2(x.x, x.y), ratio, kv), hi = quant::recode8(make_uint2(x.z, x.w), ratio, kv);
                        *p = make_uint4(lo.x, lo.y, hi.x, hi.y);
                    }
                }
            }
            // Rows that move, 16 at a time: a destination lies before the source of every later move, so reading a group
            // before writing it is enough.
            for (int d0 = 0; d0 < k; d0 += 16) {
                uint4 x[4];
                float ratio[4];
                long long to_at[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int d = d0 + 4 * u + (lane >> 3), dc = min(d, k - 1);
                    const int slot = slot_of(dc);
                    const int src = pl + slot, dst = pl + 1 + dc;
                    const int from = (src >> a.block_shift) - fb, to = (dst >> a.block_shift) - fb;
                    const long long from_at = __shfl_sync(0xffffffffu, base, from);
                    const float so = __shfl_sync(0xffffffffu, scale, from), sn = __shfl_sync(0xffffffffu, s_new, to);
                    to_at[u] = __shfl_sync(0xffffffffu, base, to);
                    ratio[u] = so == sn ? 1.f : so / sn;
                    if (d >= k || slot == dc + 1 || from_at < 0) to_at[u] = -1;
                    if (to_at[u] >= 0) {
                        to_at[u] += (long long)(dst - (fb + to) * a.block) * st[2];
                        x[u] = *(reinterpret_cast<const uint4*>(pool + from_at + (long long)(src - (fb + from) * a.block) * st[2]) + (lane & 7));
                    }
                }
                __syncwarp();
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (to_at[u] < 0) continue;
                    if (ratio[u] != 1.f) {
                        const uint2 lo = quant::recode8(make_uint2(x[u].x, x[u].y), ratio[u], kv), hi = quant::recode8(make_uint2(x[u].z, x[u].w), ratio[u], kv);
                        x[u] = make_uint4(lo.x, lo.y, hi.x, hi.y);
                    }
                    *(reinterpret_cast<uint4*>(pool + to_at[u]) + (lane & 7)) = x[u];
                }
                __syncwarp();
            }
            if (lane <= t_last && base >= 0 && s_new != scale) *scale_p = s_new;
        }
    }
    cluster.sync();                                                       // everybody has read prefix_len
    if (part != 0 || warp != 0 || !running) return;
    if (wrong) {
        if (lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_TREE);
        return;
    }
    // context' = old window ++ accepted ids ++ bonus (if any); the new window is its last min(P, length) tokens
    const int added = k + (bn >= 0 ? 1 : 0), total = tl + added, new_len = min(total, a.P);
    const int idx = total - new_len + (lane - (a.P - new_len));           // index into context'
    const int slot = slot_of(min(max(idx - tl, 0), kMaxSlots - 1));
    int v = 0;
    if (lane < a.P && lane >= a.P - new_len) {
        if (idx < tl) v = a.tail[(size_t)b * a.P + (a.P - tl + idx)];
        else v = idx - tl < k ? a.ids[(size_t)b * a.N + slot] : bn;
    }
    __syncwarp();                                                         // every read of the old window is done
    if (lane < a.P) a.tail[(size_t)b * a.P + lane] = v;
    if (lane == 0) {
        a.tail_len[b] = new_len;
        a.prefix_len[b] = pl + added;
    }
}

}  // namespace

extern "C" war_status_t war_commit_quant(const int32_t* d_ids, const int32_t* d_accept_len, const int32_t* d_accept_path,
                                         const int32_t* d_bonus, void* d_kpool, void* d_vpool, float* d_kscale, float* d_vscale,
                                         const int32_t* d_page_table, const war_commit_quant_params_t* q, int32_t* d_prefix_len,
                                         int32_t* d_tail, int32_t* d_tail_len, war_stream_t stream) {
    if (!q) return WAR_ERR_INVALID_ARG;
    const war_commit_params_t* p = &q->commit;
    if (p->B < 0 || p->N < 1 || p->N > kMaxSlots || p->P < 1 || p->P > kMaxTail || p->Hkv < 1 || p->page_size < 1 ||
        p->max_pages_per_req < 1 || p->num_pages < 1 || (q->kv_type != kKvE4M3 && q->kv_type != kKvE5M2))
        return WAR_ERR_INVALID_ARG;
    if (p->D != 128 || !war_quant_block_ok(p->page_size, q->scale_block)) return WAR_ERR_UNSUPPORTED;
    if ((long long)p->max_pages_per_req * p->page_size >= (1ll << 30) || p->B > 65535 || p->Hkv > (1 << 20)) return WAR_ERR_UNSUPPORTED;
    if (!war_rows_aligned(p->k_strides, 1) || !war_rows_aligned(p->v_strides, 1)) return WAR_ERR_UNSUPPORTED;
    if (p->B == 0) return WAR_OK;
    if (!d_ids || !d_accept_len || !d_accept_path || !d_bonus || !d_kpool || !d_vpool || !d_kscale || !d_vscale || !d_page_table ||
        !d_prefix_len || !d_tail || !d_tail_len)
        return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_kpool | (uintptr_t)d_vpool) & 15) return WAR_ERR_UNSUPPORTED;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    CommitArgs a;
    a.ids = d_ids; a.accept_len = d_accept_len; a.accept_path = d_accept_path; a.bonus = d_bonus; a.page_table = d_page_table;
    a.kpool = (uint8_t*)d_kpool; a.vpool = (uint8_t*)d_vpool; a.kscale = d_kscale; a.vscale = d_vscale;
    a.prefix_len = d_prefix_len; a.tail = d_tail; a.tail_len = d_tail_len; a.status_word = status_word;
    for (int i = 0; i < 3; ++i) { a.ks[i] = p->k_strides[i]; a.vs[i] = p->v_strides[i]; }
    a.num_pages = p->num_pages; a.N = p->N; a.P = p->P; a.Hkv = p->Hkv; a.page_size = p->page_size; a.max_pages = p->max_pages_per_req;
    a.block_shift = 0;
    while (1 << a.block_shift < q->scale_block) ++a.block_shift;
    a.block = q->scale_block; a.blocks_per_page = p->page_size / q->scale_block;
    int parts = (2 * p->Hkv + kWarps - 1) / kWarps;                       // a warp per (head, K or V), at most eight blocks
    if (parts > 8) parts = 8;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parts, p->B);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, war_commit_quant_kernel, a, q->kv_type) != cudaSuccess) { (void)cudaGetLastError(); return WAR_ERR_CUDA; }
    return WAR_OK;
}
