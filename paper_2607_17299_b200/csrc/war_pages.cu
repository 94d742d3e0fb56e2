// The books of a paged cache: which pages requests hold, who shares them, which are free; and the copies that follow from it.
//
// refs[page] counts the table entries that hold a page, bit page % 32 of free[page / 32] is set iff it is 0.  Whatever changes the
// books gives the same result in any order of the atomics: counts are sums, bits follow from counts, and pages are given out by
// number (the k-th page wanted is the k-th lowest free one), not by who comes first.
//
// All of this is a few kilobytes to a few megabytes of integers per call, so a call costs its launch and the chain of dependent reads.
// One launch each, then.  Fork and compaction need all blocks to have read before one writes; they run as one cluster of
// eight blocks, whose hardware barrier takes the place of further launches (a barrier: about 0.5 us; a launch in a graph: 1.5 to 2).
// Measured, a launch by itself, cold: 1024 requests with 0.5 million pages: free 8.6 us, grow 9.6; 256 requests resampled: fork 38;
// 128 requests in 3.5 GB of 64 KB pages: compaction 19, the copy of its moves 254 (6.3 TB/s, the rate of a plain copy); groups among
// 512 requests of up to 73 000 tokens 15.
#include <cooperative_groups.h>
#include <mutex>
#include "war_common.cuh"
#include "war_quant.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kMaxB = 4096;
constexpr int kThreads = 1024;
constexpr int kCluster = 8;
constexpr int kMaxTail = 32;
constexpr int kRound = 4 * kThreads;      // words of the free map that a block looks at together

// ------------------------------------------------------------------------------------------------
// block-wide sums
// ------------------------------------------------------------------------------------------------
struct ScanScratch { int warp[33]; };

// Exclusive scan of x over the block, and the sum.  Block barriers inside.
__device__ __forceinline__ int block_scan(int x, ScanScratch& s, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
    if (lane == 31) s.warp[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const int y = s.warp[lane];
        int yi = y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int z = __shfl_up_sync(0xffffffffu, yi, o); if (lane >= o) yi += z; }
        s.warp[lane] = yi - y;
        if (lane == 31) s.warp[32] = yi;
    }
    __syncthreads();
    const int before = s.warp[warp];
    *total = s.warp[32];
    __syncthreads();
    return before + incl - x;
}

// The same for two numbers at once.
__device__ __forceinline__ int2 block_scan2(int2 x, int2* s_warp, int2* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl.x, o), z = __shfl_up_sync(0xffffffffu, incl.y, o);
        if (lane >= o) { incl.x += y; incl.y += z; }
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    const int2 w = s_warp[lane];                                  // every warp adds the warps' sums up for itself: one barrier less
    int2 wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, wi.x, o), z = __shfl_up_sync(0xffffffffu, wi.y, o);
        if (lane >= o) { wi.x += y; wi.y += z; }
    }
    const int2 before = make_int2(__shfl_sync(0xffffffffu, wi.x - w.x, warp), __shfl_sync(0xffffffffu, wi.y - w.y, warp));
    *total = make_int2(__shfl_sync(0xffffffffu, wi.x, 31), __shfl_sync(0xffffffffu, wi.y, 31));
    __syncthreads();
    return make_int2(before.x + incl.x - x.x, before.y + incl.y - x.y);
}

// the position of the k-th (from 0) set bit of a word that has it
__device__ __forceinline__ int nth_bit(uint32_t word, int k) {
    int at = 0;
#pragma unroll
    for (int width = 16; width > 0; width >>= 1) {
        const int low = __popc((word >> at) & ((1u << width) - 1u));
        if (k >= low) { k -= low; at += width; }
    }
    return at;
}

// largest i in [0, n) with a[i] <= x (a ascending, a[0] <= x)
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// A round of the free map in shared memory: words, and how many free pages lie before each.
struct FreeRound { uint32_t word[kRound]; int before[kRound + 1]; };

// Loads words [first, first + kRound) (pages behind the pool's last one as taken); `before` counts from `base` on.  Returns the free pages.
__device__ __forceinline__ int load_round(FreeRound& r, const uint32_t* free_map, long long first, long long num_pages, int base, ScanScratch& s) {
    const int w0 = (int)threadIdx.x * 4;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {                                // (coalesced, then turned: a thread's four words are neighbours)
        const int at = (int)threadIdx.x + k * kThreads;
        const long long left = num_pages - (first + at) * 32;
        r.word[at] = left <= 0 ? 0u : free_map[first + at] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) { w[k] = r.word[w0 + k]; count += __popc(w[k]); }
    int total, run = base + block_scan(count, s, &total);
#pragma unroll
    for (int k = 0; k < 4; ++k) { r.before[w0 + k] = run; run += __popc(w[k]); }
    if (threadIdx.x == kThreads - 1) r.before[kRound] = run;
    __syncthreads();
    return total;
}
// The k-th free page (counted over all rounds) of the round that holds it.
__device__ __forceinline__ int nth_free(const FreeRound& r, long long first, int k) {
    const int at = last_at_most(r.before, kRound, k);            // (the last of equals: a word that holds pages)
    return (int)((first + at) * 32 + nth_bit(r.word[at], k - r.before[at]));
}

// ------------------------------------------------------------------------------------------------
// free
// ------------------------------------------------------------------------------------------------
// A block per request.  Pages of a group come back with their last holder, whichever block that is.  A thread asks for four entries at
// once and then for the four counts (one after the other they cost two trips to L2 each).
constexpr int kFreeThreads = 256, kFreeDeep = 4;
__global__ void __launch_bounds__(kFreeThreads)
pages_free_kernel(war_pages_t p, const int32_t* __restrict__ done, int32_t* tail_len, int* status_word) {
    war_wait_before();
    const int b = blockIdx.x;
    if (done[b] == 0) return;
    const int held = p.d_held[b];
    int32_t* row = p.d_page_table + (size_t)b * p.max_pages_per_req;
    if (held < 0 || held > p.max_pages_per_req) {
        if (threadIdx.x == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
        return;
    }
    for (int j0 = threadIdx.x; j0 < held; j0 += kFreeThreads * kFreeDeep) {
        int page[kFreeDeep], had[kFreeDeep];
#pragma unroll
        for (int k = 0; k < kFreeDeep; ++k) page[k] = j0 + k * kFreeThreads < held ? row[j0 + k * kFreeThreads] : -2;
#pragma unroll
        for (int k = 0; k < kFreeDeep; ++k) had[k] = page[k] >= 0 && page[k] < p.num_pages ? atomicSub(&p.d_refs[page[k]], 1) : 2;
#pragma unroll
        for (int k = 0; k < kFreeDeep; ++k) {
            if (page[k] == -2 && j0 + k * kFreeThreads >= held) continue;
            row[j0 + k * kFreeThreads] = -1;
            if (page[k] < 0 || page[k] >= p.num_pages) { war_set_device_status(status_word, WAR_ERR_BAD_PAGE); continue; }
            if (had[k] == 1) atomicOr(&p.d_free[page[k] >> 5], 1u << (page[k] & 31));
            if (had[k] <= 0) { atomicAdd(&p.d_refs[page[k]], 1); war_set_device_status(status_word, WAR_ERR_BAD_PAGE); }
        }
    }
    __syncthreads();                                              // (every thread has read held)
    if (threadIdx.x == 0) {
        p.d_held[b] = 0;
        if (tail_len) tail_len[b] = -1;
    }
}

// ------------------------------------------------------------------------------------------------
// grow
// ------------------------------------------------------------------------------------------------
struct GrowShared {
    ScanScratch scan;
    FreeRound round;
    int upto[kMaxB + 1];                   // pages wanted by the requests before
    int held[kMaxB];
};

__global__ void __launch_bounds__(kThreads, 1)
pages_grow_kernel(war_pages_t p, int N, const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ tail_len, int32_t* granted,
                  int* status_word) {
    extern __shared__ __align__(16) uint8_t pages_smem[];
    war_wait_before();
    GrowShared& s = *reinterpret_cast<GrowShared*>(pages_smem);
    const int tid = threadIdx.x, B = p.B;
    const long long n_words = (p.num_pages + 31) / 32;
    // ---- what every request wants ----
    int wanted = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + tid;
        int need = 0, have = 0;
        if (b < B) {
            have = p.d_held[b];
            const long long pl = prefix_len[b];
            const bool runs = !tail_len || tail_len[b] >= 0;
            const long long want = (pl + N + p.page_size - 1) / p.page_size;
            bool ok = runs;
            if (runs && (pl < 0 || have < 0 || have > p.max_pages_per_req || want > p.max_pages_per_req)) {
                war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
                ok = false;
            }
            need = ok ? max(0, (int)want - have) : 0;
            s.held[b] = ok ? have : -1;                           // (-1: not to be served)
        }
        int total;
        const int before = wanted + block_scan(need, s.scan, &total);
        if (b < B) s.upto[b] = before;
        wanted += total;
    }
    if (tid == 0) s.upto[B] = wanted;
    __syncthreads();
    // ---- are there so many?  (rounds of the map until there are) ----
    int found = 0, rounds = 0;
    if (wanted > 0)
        for (long long first = 0; first < n_words && found < wanted; first += kRound, ++rounds) found += load_round(s.round, p.d_free, first, p.num_pages, found, s.scan);
    // a request is served iff all pages wanted up to and with it are there
    int served = wanted;
    if (found < wanted) served = s.upto[last_at_most(s.upto, B + 1, found)];
    // ---- the k-th of them goes to the request that wants it ----
    int base = 0;
    for (int r = 0; r < rounds && base < served; ++r) {
        const long long first = (long long)r * kRound;
        int here = s.round.before[kRound] - s.round.before[0];
        if (rounds > 1) {
            __syncthreads();
            here = load_round(s.round, p.d_free, first, p.num_pages, base, s.scan);
        }
        for (int k = base + tid; k < min(base + here, served); k += kThreads) {
            const int page = nth_free(s.round, first, k);
            const int b = last_at_most(s.upto, B, k);
            p.d_page_table[(size_t)b * p.max_pages_per_req + s.held[b] + (k - s.upto[b])] = page;
            p.d_refs[page] = 1;
            atomicAnd(&p.d_free[page >> 5], ~(1u << (page & 31)));
        }
        base += here;
    }
    for (int b = tid; b < B; b += kThreads) {
        const int need = s.upto[b + 1] - s.upto[b];
        const bool ok = s.held[b] >= 0 && (need == 0 || s.upto[b + 1] <= served);
        granted[b] = ok;
        if (ok && need > 0) p.d_held[b] = s.held[b] + need;
    }
}

// ------------------------------------------------------------------------------------------------
// fork
// ------------------------------------------------------------------------------------------------
// What changes is decided by every block for itself from the books as they are; after the cluster's barrier the blocks write, a tile of
// columns each at a time: a table's column is changed by one block alone, which holds all of its old entries in shared memory, so
// requests that swap places need no second table.
// An entry counts before the call, so a count that is found at 0 or below (or falls below) belongs to books that say less than the tables
// hold.  Asking for the counts of the pages that gain holders, too, costs 256 resampled requests 31.0 -> 34.5 us.
constexpr int kDeep = 4, kForkDeep = 8;   // entries that a thread asks for at once
constexpr int kForkTile = 16384;          // entries of a tile
constexpr int kNoPage = 0x7fffffff;       // a source's partly filled page that lies outside the pool: its copies get none
struct ForkShared {
    ScanScratch scan;
    FreeRound round;
    int16_t src[kMaxB];                    // source, -1: the request stays as it is
    int first[kMaxB];                      // lowest request that takes this one, kMaxB: none
    int takers[kMaxB];
    int full[kMaxB];                       // full pages of this request
    int held[kMaxB];
    int last[kMaxB];                       // a request that is replaced: its partly filled page; -1: none
    int fresh[kMaxB];                      // pages wanted by the requests before
    int entries[kForkTile];
    int columns;
    int uncounted;                         // (the first block's) an entry was met that refs does not count
};

__global__ void __launch_bounds__(kThreads, 1)
pages_fork_kernel(war_pages_t p, const int32_t* __restrict__ d_src, int P, int32_t* prefix_len, int32_t* tail, int32_t* tail_len,
                  int32_t* copies, int32_t* n_copies, int32_t* ok_word, int* status_word) {
    extern __shared__ __align__(16) uint8_t pages_smem[];
    war_wait_before();
    ForkShared& s = *reinterpret_cast<ForkShared*>(pages_smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, B = p.B, rank = (int)cluster.block_rank(), width = p.max_pages_per_req, page_size = p.page_size;
    const long long n_words = (p.num_pages + 31) / 32;
    // ---- who becomes whom ----
    for (int b = tid; b < B; b += kThreads) { s.first[b] = kMaxB; s.takers[b] = 0; }
    if (tid == 0) s.columns = s.uncounted = 0;
    __syncthreads();
    for (int b = tid; b < B; b += kThreads) {
        int src = d_src[b];
        const int held = p.d_held[b];
        s.held[b] = held;
        s.full[b] = prefix_len[b] / page_size;                    // (looked at for sources only, which are checked)
        if (src == b || src < 0) src = -1;
        else {
            bool ok = src < B && held >= 0 && held <= width;
            if (ok && tail_len[src] < 0) ok = false;
            if (ok) {
                const int pl = prefix_len[src], src_held = p.d_held[src];
                ok = pl >= 0 && src_held >= 0 && src_held <= width && (pl + (long long)page_size - 1) / page_size <= src_held;
            }
            if (!ok) { if (rank == 0) war_set_device_status(status_word, WAR_ERR_INVALID_ARG); src = -1; }
        }
        s.src[b] = (int16_t)src;
        if (src >= 0) { atomicMin(&s.first[src], b); atomicAdd(&s.takers[src], 1); }
    }
    __syncthreads();
    // ---- partly filled pages: the first that takes a request which is itself replaced gets its page, the others a fresh one ----
    int wanted = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + tid;
        int fresh = 0;
        if (b < B) {
            const int src = s.src[b];
            int last = -1;
            if (src >= 0 && prefix_len[src] % page_size != 0) {
                last = p.d_page_table[(size_t)src * width + s.full[src]];
                const bool bad = last < 0 || last >= p.num_pages;
                if (bad) { if (rank == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE); last = kNoPage; }
                fresh = !bad && !(s.src[src] >= 0 && s.first[src] == b && p.d_refs[last] == 1);
            }
            s.last[b] = last;
            if (src >= 0) atomicMax(&s.columns, max(s.held[b], s.full[src] + (last >= 0)));
        }
        int total;
        const int before = wanted + block_scan(fresh, s.scan, &total);
        if (b < B) s.fresh[b] = fresh ? before : -1;
        wanted += total;
    }
    // ---- the fresh pages; all or nothing ----
    int found = 0;
    bool enough = true;
    __syncthreads();
    if (wanted > 0) {
        // (fresh[b] holds the page's number in the order of the free ones until its round comes, then ~page)
        for (long long first = 0; first < n_words && found < wanted; first += kRound) {
            const int here = load_round(s.round, p.d_free, first, p.num_pages, found, s.scan);
            for (int b = tid; b < B; b += kThreads) {
                const int k = s.fresh[b];
                if (k >= found && k < found + here) s.fresh[b] = ~nth_free(s.round, first, k) - 1;           // (below -1)
            }
            found += here;
            __syncthreads();
        }
        enough = found >= wanted;
    }
    const int columns = s.columns;
    int* const uncounted = cluster.map_shared_rank(&s.uncounted, 0);
    if (rank == 0 && tid == 0) { *ok_word = enough; *n_copies = enough ? wanted : 0; }
    // ---- everything has been read but the rows themselves and the tails; every block takes its columns ----
    // Tiles of 2^lg columns (and one more, the tail windows): the width that leaves the least to the busiest block, a tile's barriers and
    // trips to memory counted as 16 columns.
    int lg = 0, least = 0x7fffffff;
    for (int w = 0; w <= 6 && ((long long)B << w) <= kForkTile; ++w) {
        const int busiest = ((((columns + (1 << w) - 1) >> w) + kCluster - 1) / kCluster) * ((1 << w) + 16);
        if (busiest <= least) { least = busiest; lg = w; }
    }
    const int tile_cols = 1 << lg, tiles = ((columns + tile_cols - 1) >> lg) + 1;
    int pl_new[kMaxB / kThreads], tl_new[kMaxB / kThreads];
#pragma unroll
    for (int k = 0; k < kMaxB / kThreads; ++k) {
        const int b = tid + k * kThreads;
        pl_new[k] = tl_new[k] = 0;
        if (b < B && s.src[b] >= 0) { pl_new[k] = prefix_len[s.src[b]]; tl_new[k] = tail_len[s.src[b]]; }
    }
    // ---- list of copies: fresh pages in the order of the requests ----
    int listed = 0;
    if (rank == 0 && enough) {
        for (int b0 = 0; b0 < B; b0 += kThreads) {
            const int b = b0 + tid;
            const bool fresh = b < B && s.fresh[b] < -1;
            int total;
            const int at = listed + block_scan(fresh ? 1 : 0, s.scan, &total);
            if (fresh) {
                copies[3 * at] = s.last[b]; copies[3 * at + 1] = ~(s.fresh[b] + 1); copies[3 * at + 2] = prefix_len[s.src[b]] % page_size;
            }
            listed += total;
        }
    }
    cluster.sync();
    if (!enough) return;
    if (rank == 0) {
#pragma unroll
        for (int k = 0; k < kMaxB / kThreads; ++k) {
            const int b = tid + k * kThreads;
            if (b >= B || s.src[b] < 0) continue;
            prefix_len[b] = pl_new[k];
            tail_len[b] = tl_new[k];
            p.d_held[b] = s.full[s.src[b]] + (s.last[b] >= 0);
        }
    }
    for (int t = rank; t < tiles; t += kCluster) {
        const bool is_tail = t == tiles - 1;
        const int c0 = is_tail ? 0 : t * tile_cols;
        const int cols = is_tail ? P : min(tile_cols, columns - c0);
        int32_t* const table = is_tail ? tail : p.d_page_table + c0;
        const int stride = is_tail ? P : width;
        const int batch = is_tail ? kForkTile / kMaxTail : B;     // (tails of many requests do not fit at once; see below)
        if (is_tail && B > batch) {
            // too many for one tile: column by column
            for (int c = 0; c < P; ++c) {
                __syncthreads();
                for (int b = tid; b < B; b += kThreads) s.entries[b] = tail[(size_t)b * P + c];
                __syncthreads();
                for (int b = tid; b < B; b += kThreads) if (s.src[b] >= 0) tail[(size_t)b * P + c] = s.entries[s.src[b]];
            }
            continue;
        }
        __syncthreads();
        const int wide = is_tail ? 5 : lg, entries = B << wide;   // (a tail window has at most 32 tokens)
        for (int x0 = tid; x0 < entries; x0 += kThreads * kForkDeep) {
            int v[kForkDeep];
#pragma unroll
            for (int k = 0; k < kForkDeep; ++k) {
                const int x = x0 + k * kThreads, b = x >> wide, c = x & ((1 << wide) - 1);
                v[k] = x < entries && c < cols && (s.src[b] >= 0 || s.takers[b] > 0) ? table[(size_t)b * stride + c] : 0;
            }
#pragma unroll
            for (int k = 0; k < kForkDeep; ++k) if (x0 + k * kThreads < entries) s.entries[x0 + k * kThreads] = v[k];
        }
        __syncthreads();
        for (int x0 = tid; x0 < entries; x0 += kThreads * kForkDeep) {
            int had[kForkDeep], page[kForkDeep];
            uint32_t taken = 0;                                   // entries that gain holders
#pragma unroll
            for (int k = 0; k < kForkDeep; ++k) {
                const int x = x0 + k * kThreads;
                had[k] = 2;
                page[k] = 0;
                const int b = x >> wide, c = x & ((1 << wide) - 1);
                if (x >= entries || c >= cols) continue;
                const int src = s.src[b];
                if (is_tail) {
                    if (src >= 0) tail[(size_t)b * P + c] = s.entries[(src << wide) + c];
                    continue;
                }
                const int col = c0 + c;
                // what this entry's page gains and loses: a holder for every request that takes it as a full page, this row if it is
                // replaced, unless its partly filled page is handed on
                int delta = (col < s.full[b] ? s.takers[b] : 0) - (src >= 0 && col < s.held[b] ? 1 : 0);
                if (delta < 0 && col == s.full[b] && s.first[b] < kMaxB && s.last[s.first[b]] >= 0 && s.fresh[s.first[b]] == -1) delta = 0;
                if (delta != 0) {
                    page[k] = s.entries[x];
                    if (page[k] < 0 || page[k] >= p.num_pages) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
                    else had[k] = atomicAdd(&p.d_refs[page[k]], delta);
                    if (delta > 0) taken |= 1u << k;
                }
                if (src < 0) continue;
                int now = -1;
                if (col < s.full[src]) {
                    now = s.entries[(src << wide) + c];           // (one outside the pool stays what it is)
                    if (now < 0 || now >= p.num_pages) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
                } else if (col == s.full[src] && s.last[b] >= 0) now = s.fresh[b] < -1 ? ~(s.fresh[b] + 1) : s.last[b] == kNoPage ? -1 : s.last[b];
                else if (col >= s.held[b]) continue;              // (nothing stood there)
                p.d_page_table[(size_t)b * width + col] = now;
            }
#pragma unroll
            for (int k = 0; k < kForkDeep; ++k) {
                if (had[k] == 1 && !(taken >> k & 1u)) atomicOr(&p.d_free[page[k] >> 5], 1u << (page[k] & 31));
                if (had[k] <= 0) *uncounted = 1;                  // more entries than refs counts: their pages' counts began too low
            }
        }
    }
    // ---- the fresh pages come last: earlier, their counts would hide that an entry of the books as they were is not counted ----
    cluster.sync();
    if (rank != 0) return;
    if (s.uncounted) {
        // Sums are the same in any order, what was seen on the way is not: counts below 0 become 0, and the bits follow from the counts.
        if (tid == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
        for (long long w = tid; w < n_words; w += kThreads) {
            uint32_t word = 0;
            for (int k = 0; k < 32 && w * 32 + k < p.num_pages; ++k) {
                const int refs = __ldcg(&p.d_refs[w * 32 + k]);
                if (refs < 0) p.d_refs[w * 32 + k] = 0;
                if (refs <= 0) word |= 1u << k;
            }
            p.d_free[w] = word;
        }
        __syncthreads();
    }
    for (int b = tid; b < B; b += kThreads) {
        if (s.fresh[b] >= -1) continue;
        const int page = ~(s.fresh[b] + 1);
        atomicAdd(&p.d_refs[page], 1);
        atomicAnd(&p.d_free[page >> 5], ~(1u << (page & 31)));
    }
}

// ------------------------------------------------------------------------------------------------
// compact
// ------------------------------------------------------------------------------------------------
// The i-th highest used page goes to the i-th lowest free page while it lies above it.  With U pages in use that moves exactly the
// used pages at or above U, so the two lists are the free pages below U, upwards, and the used ones from U on, downwards.
// The map as it was is kept: a table's entry that it has as free is not counted in refs, whichever side of U its page is on, and place[] holds for it
// what the workspace held.  (A word for 32 pages, mostly out of L1: 18.8 us where 17.6 without the look, 3.5 GB pool;
// to look the page up in its list instead costs two dependent reads an entry, 24.6.)
struct CompactShared {
    int2 warp[32];
    int used;                              // of this block's words
    int free_below, used_above;            // of this block's words, below / from U on
};

__global__ void __launch_bounds__(kThreads, 1)
pages_compact_kernel(war_pages_t p, int32_t* ws, int max_copies, int32_t* copies, int32_t* n_copies, int32_t* top, int* status_word) {
    __shared__ CompactShared s;
    war_wait_before();
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, rank = (int)cluster.block_rank();
    const int n_words = (int)((p.num_pages + 31) / 32);
    int32_t* const place = ws;                                    // [num_pages] where a used page from U on goes
    int32_t* const to = ws + p.num_pages;                         // free pages below U; as many as used ones from U on, at most half of all
    int32_t* const from = to + p.num_pages / 2;                   // used pages from U on
    uint32_t* const was = (uint32_t*)(ws + 2 * p.num_pages);      // the map before the moves
    const int per = (n_words + kCluster - 1) / kCluster, w0 = min(n_words, rank * per), w1 = min(n_words, w0 + per);
    auto valid = [&](int w) -> uint32_t {                         // pages of a word that exist
        const long long left = p.num_pages - (long long)w * 32;
        return left >= 32 ? 0xffffffffu : (1u << left) - 1u;
    };
    // ---- pages in use ----
    const bool once = w1 - w0 <= kThreads;                        // a word a thread: it is read and summed up once
    const uint32_t mine = w0 + tid < w1 ? p.d_free[w0 + tid] : 0u;
    int used = w0 + tid < w1 ? __popc(~mine & valid(w0 + tid)) : 0;
    if (w0 + tid < w1) was[w0 + tid] = mine;
    for (int w = w0 + tid + kThreads; w < w1; w += kThreads) { const uint32_t f = p.d_free[w]; was[w] = f; used += __popc(~f & valid(w)); }
    int2 total;
    block_scan2(make_int2(used, 0), s.warp, &total);
    if (tid == 0) s.used = total.x;
    cluster.sync();
    int U = 0;
    for (int r = 0; r < kCluster; ++r) U += *cluster.map_shared_rank(&s.used, r);
    // ---- this block's part of both lists ----
    auto below = [&](int w) -> uint32_t {                         // pages of a word below U
        const int left = U - w * 32;
        return left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
    };
    auto free_of = [&](int w, uint32_t f) -> uint32_t { return w < w1 ? f & below(w) : 0u; };
    auto used_of = [&](int w, uint32_t f) -> uint32_t { return w < w1 ? ~f & valid(w) & ~below(w) : 0u; };
    int2 own = make_int2(__popc(free_of(w0 + tid, mine)), __popc(used_of(w0 + tid, mine)));
    for (int w = w0 + tid + kThreads; w < w1; w += kThreads) { const uint32_t f = p.d_free[w]; own.x += __popc(free_of(w, f)); own.y += __popc(used_of(w, f)); }
    const int2 before = block_scan2(own, s.warp, &total);
    if (tid == 0) { s.free_below = total.x; s.used_above = total.y; }
    cluster.sync();
    int lo_at = 0, hi_at = total.y, moves = 0;                    // free ones before this block's, used ones from its own on
    for (int r = 0; r < kCluster; ++r) {
        const int x = *cluster.map_shared_rank(&s.free_below, r), y = *cluster.map_shared_rank(&s.used_above, r);
        if (r < rank) lo_at += x;
        if (r > rank) hi_at += y;
        moves += x;
    }
    for (int first = w0; first < w1; first += kThreads) {         // words in order: free ones from the front, used ones from the back
        const int w = first + tid;
        const uint32_t f = first == w0 ? mine : w < w1 ? p.d_free[w] : 0u;
        uint32_t a = free_of(w, f), c = used_of(w, f);
        int2 round, at2 = before;
        if (!once) at2 = block_scan2(make_int2(__popc(a), __popc(c)), s.warp, &round);
        int at = lo_at + at2.x, back = hi_at - at2.y;
        if (!once) { lo_at += round.x; hi_at -= round.y; }
        while (a) { to[at++] = w * 32 + __ffs(a) - 1; a &= a - 1; }
        while (c) { from[--back] = w * 32 + __ffs(c) - 1; c &= c - 1; }
    }
    cluster.sync();
    // ---- the moves ----
    const int done = min(moves, max_copies);
    for (int i0 = rank * kThreads + tid; i0 < moves; i0 += kCluster * kThreads * kDeep) {
        int a[kDeep], c[kDeep], refs[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int i = i0 + k * kCluster * kThreads;
            a[k] = i < moves ? from[i] : 0; c[k] = i < done ? to[i] : a[k];
        }
#pragma unroll
        for (int k = 0; k < kDeep; ++k) refs[k] = i0 + k * kCluster * kThreads < done ? p.d_refs[a[k]] : 0;
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int i = i0 + k * kCluster * kThreads;
            if (i >= moves) break;
            place[a[k]] = c[k];
            if (i >= done) continue;
            p.d_refs[c[k]] = refs[k];
            p.d_refs[a[k]] = 0;
            atomicAnd(&p.d_free[c[k] >> 5], ~(1u << (c[k] & 31)));
            atomicOr(&p.d_free[a[k] >> 5], 1u << (a[k] & 31));
            copies[3 * i] = a[k]; copies[3 * i + 1] = c[k]; copies[3 * i + 2] = p.page_size;
        }
    }
    if (rank == 0 && tid == 0) {
        *n_copies = done;
        *top = done < moves ? from[done] + 1 : U;
    }
    cluster.sync();
    // ---- the tables follow, a warp a row ----
    for (int b = (rank * kThreads + tid) >> 5; b < p.B; b += kCluster * kThreads / 32) {
        const int held = p.d_held[b], lane = tid & 31;
        int32_t* row = p.d_page_table + (size_t)b * p.max_pages_per_req;
        if (held < 0 || held > p.max_pages_per_req) { if (lane == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE); continue; }
        for (int j0 = lane; j0 < held; j0 += 32 * 2 * kDeep) {
            int page[2 * kDeep], now[2 * kDeep];
            bool bad[2 * kDeep];
#pragma unroll
            for (int k = 0; k < 2 * kDeep; ++k) page[k] = j0 + k * 32 < held ? row[j0 + k * 32] : 0;
#pragma unroll
            for (int k = 0; k < 2 * kDeep; ++k) {
                bad[k] = page[k] < 0 || page[k] >= p.num_pages;
                now[k] = !bad[k] && page[k] >= U ? place[page[k]] : page[k];
                bad[k] = bad[k] || (was[page[k] >> 5] >> (page[k] & 31) & 1u);
            }
#pragma unroll
            for (int k = 0; k < 2 * kDeep; ++k) {
                if (j0 + k * 32 >= held) continue;
                if (bad[k]) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
                else if (page[k] >= U) row[j0 + k * 32] = now[k];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// groups
// ------------------------------------------------------------------------------------------------
// A block per request: it leaves if a lower request has the same page in that column, else it is the leader and compares its row with
// all of its members', a column a thread, until the columns in which all agree end.  Blocks have nothing to tell each other.
constexpr int kGroupThreads = 512, kGroupDeep = 2, kGroupRows = 4;
__global__ void __launch_bounds__(kGroupThreads)
prefix_groups_kernel(const int32_t* __restrict__ table, const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ tail_len,
                     int B, int page_size, int width, int column, int32_t* leader, int32_t* shared_len) {
    __shared__ uint16_t s_member[kMaxB];
    __shared__ int s_members, s_full, s_same;
    war_wait_before();
    const int tid = threadIdx.x, me = blockIdx.x;
    auto full_of = [&](int b) -> int {                            // full pages of a running request's prefix
        const int pl = prefix_len[b], run = tail_len ? tail_len[b] : 0;
        return run >= 0 && pl > 0 ? min(pl / page_size, width) : 0;
    };
    const int my_full = full_of(me), my_key = table[(size_t)me * width + min(column, width - 1)];
    if (tid == 0) { s_members = 0; s_full = my_full; }
    bool lower = false;
    __syncthreads();
    if (my_full > column && my_key >= 0) {                        // (uniform: all threads have read the same)
        for (int q0 = 0; q0 < B; q0 += kGroupThreads * kGroupDeep) {
            int key[kGroupDeep], full[kGroupDeep];
#pragma unroll
            for (int k = 0; k < kGroupDeep; ++k) {
                const int q = q0 + k * kGroupThreads + tid;
                full[k] = q < B ? full_of(q) : 0;
                key[k] = q < B ? table[(size_t)q * width + column] : -1;
            }
#pragma unroll
            for (int k = 0; k < kGroupDeep; ++k) {
                const int q = q0 + k * kGroupThreads + tid;
                if (full[k] <= column || key[k] != my_key || q == me) continue;
                if (q < me) lower = true;
                else { s_member[atomicAdd(&s_members, 1)] = (uint16_t)q; atomicMin(&s_full, full[k]); }
            }
            if (__syncthreads_or(lower)) return;                  // (the leader's block answers for this request)
        }
    }
    const int members = s_members, n = s_full;
    const int32_t* mine = table + (size_t)me * width;
    int same = 0;
    if (members > 0) {
        for (same = 0; same < n;) {
            if (tid == 0) s_same = n;
            __syncthreads();
            int first = n;
            int x[kGroupDeep];
#pragma unroll
            for (int k = 0; k < kGroupDeep; ++k) { const int c = same + k * kGroupThreads + tid; x[k] = c < n ? mine[c] : 0; }
            for (int m = 0; m < members; m += kGroupRows) {       // (the rows of a few members at once)
                int y[kGroupRows][kGroupDeep];
#pragma unroll
                for (int r = 0; r < kGroupRows; ++r) {
                    const int32_t* row = table + (size_t)s_member[min(m + r, members - 1)] * width;
#pragma unroll
                    for (int k = 0; k < kGroupDeep; ++k) { const int c = same + k * kGroupThreads + tid; y[r][k] = c < n ? row[c] : x[k]; }
                }
#pragma unroll
                for (int r = 0; r < kGroupRows; ++r)
#pragma unroll
                    for (int k = kGroupDeep - 1; k >= 0; --k) if (y[r][k] != x[k]) first = min(first, same + k * kGroupThreads + tid);
            }
            if (first < n) atomicMin(&s_same, first);
            __syncthreads();
            const int end = s_same, next = min(n, same + kGroupThreads * kGroupDeep);
            __syncthreads();
            same = min(end, next);
            if (end < next) break;
        }
    }
    const bool group = members > 0 && same > column;
    if (tid == 0) { leader[me] = me; shared_len[me] = group ? same * page_size : 0; }
    for (int m = tid; m < members; m += kGroupThreads) {
        const int q = s_member[m];
        leader[q] = group ? me : q;
        shared_len[q] = group ? same * page_size : 0;
    }
}

// ------------------------------------------------------------------------------------------------
// copy
// ------------------------------------------------------------------------------------------------
struct CopyArgs {
    uint8_t *k, *v;
    float *kscale, *vscale;
    long long ks[3], vs[3];                // strides (page, head, token) in bytes
    const int32_t *copies, *n_copies;
    long long num_pages;
    int max_copies, Hkv, page_size, block;
};

// A warp per (copy, K or V, head): rows of 256 or 128 bytes, 512 bytes a warp's instruction, up to eight of them in flight.
constexpr int kCopyWarps = 8;
template <int kLanesPerRow>                // 16-byte pieces of a row: 16 (bf16) or 8
__global__ void __launch_bounds__(kCopyWarps * 32)
pages_copy_kernel(const CopyArgs a, int* status_word) {
    constexpr int kRows = 32 / kLanesPerRow, kDeep = 8;
    war_wait_before();
    const int lane = threadIdx.x & 31, r0 = lane / kLanesPerRow, piece = lane % kLanesPerRow;
    const int n = min(max(*a.n_copies, 0), a.max_copies);
    const long long tasks = (long long)n * 2 * a.Hkv, step = (long long)gridDim.x * kCopyWarps;
    for (long long t = (long long)blockIdx.x * kCopyWarps + (threadIdx.x >> 5); t < tasks; t += step) {
        const int c = (int)(t / (2 * a.Hkv)), rest = (int)(t - (long long)c * 2 * a.Hkv), which = rest / a.Hkv, h = rest - which * a.Hkv;
        const int32_t* const line = a.copies + 3 * (long long)c;
        const long long from = line[0], to = line[1];
        const int rows = min(max(line[2], 0), a.page_size);
        if (from < 0 || from >= a.num_pages || to < 0 || to >= a.num_pages) {
            if (lane == 0) war_set_device_status(status_word, WAR_ERR_BAD_PAGE);
            continue;
        }
        uint8_t* const pool = which ? a.v : a.k;
        const long long s_page = which ? a.vs[0] : a.ks[0], s_head = which ? a.vs[1] : a.ks[1], s_row = which ? a.vs[2] : a.ks[2];
        const uint8_t* src = pool + from * s_page + h * s_head + piece * 16;
        uint8_t* dst = pool + to * s_page + h * s_head + piece * 16;
        for (int r = r0; r < rows; r += kRows * kDeep) {
            uint4 x[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k)
                if (r + k * kRows < rows) x[k] = __ldcs(reinterpret_cast<const uint4*>(src + (r + k * kRows) * s_row));
#pragma unroll
            for (int k = 0; k < kDeep; ++k)
                if (r + k * kRows < rows) *reinterpret_cast<uint4*>(dst + (r + k * kRows) * s_row) = x[k];
        }
        if (a.block > 0) {                                        // scales of the blocks that hold these rows
            float* const sc = which ? a.vscale : a.kscale;
            const int bpp = a.page_size / a.block;
            if (lane < (rows + a.block - 1) / a.block) sc[(to * a.Hkv + h) * bpp + lane] = sc[(from * a.Hkv + h) * bpp + lane];
        }
    }
}

// ------------------------------------------------------------------------------------------------
constexpr int kMaxDevices = 64;
std::once_flag g_dev_once[kMaxDevices];
int g_sm_count[kMaxDevices];
war_status_t g_dev_status[kMaxDevices];

war_status_t device_setup(int* sm_count) {
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    std::call_once(g_dev_once[dev], [dev]() {
        g_dev_status[dev] = WAR_ERR_CUDA;
        if (cudaDeviceGetAttribute(&g_sm_count[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return;
        if (cudaFuncSetAttribute(pages_grow_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(GrowShared)) != cudaSuccess) return;
        if (cudaFuncSetAttribute(pages_fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ForkShared)) != cudaSuccess) return;
        g_dev_status[dev] = WAR_OK;
    });
    if (g_dev_status[dev] != WAR_OK) (void)cudaGetLastError();
    *sm_count = g_sm_count[dev];
    return g_dev_status[dev];
}
static_assert(sizeof(ForkShared) <= 232448 && sizeof(GrowShared) <= 232448, "shared memory");

war_status_t check_pages(const war_pages_t* p) {
    if (!p || p->B < 0 || p->page_size < 1 || p->max_pages_per_req < 1 || p->num_pages < 1) return WAR_ERR_INVALID_ARG;
    if (p->B > kMaxB || p->num_pages > (1ll << 30) || (long long)p->B * p->max_pages_per_req >= (1ll << 31)) return WAR_ERR_UNSUPPORTED;   // (entries are counted in 32 bits)
    if (p->B > 0 && (!p->d_refs || !p->d_free || !p->d_page_table || !p->d_held)) return WAR_ERR_INVALID_ARG;
    return WAR_OK;
}

}  // namespace

extern "C" war_status_t war_pages_free(const war_pages_t* p, const int32_t* d_done, int32_t* d_tail_len, war_stream_t stream) {
    const war_status_t st = check_pages(p);
    if (st != WAR_OK) return st;
    if (p->B == 0) return WAR_OK;
    if (!d_done) return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    return war_launch_behind(pages_free_kernel, p->B, kFreeThreads, 0, 1, stream, *p, d_done, d_tail_len, status_word);
}

extern "C" war_status_t war_pages_grow(const war_pages_t* p, int32_t N, const int32_t* d_prefix_len, const int32_t* d_tail_len,
                                       int32_t* d_granted, war_stream_t stream) {
    war_status_t st = check_pages(p);
    if (st != WAR_OK) return st;
    if (N < 0 || (long long)N + p->page_size >= (1ll << 30)) return WAR_ERR_INVALID_ARG;
    if (p->B == 0) return WAR_OK;
    if (!d_prefix_len || !d_granted) return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    int sms;
    st = device_setup(&sms);
    if (st != WAR_OK) return st;
    return war_launch_behind(pages_grow_kernel, 1, kThreads, sizeof(GrowShared), 1, stream, *p, N, d_prefix_len, d_tail_len, d_granted, status_word);
}

extern "C" war_status_t war_pages_fork(const war_pages_t* p, const int32_t* d_src, int32_t P, int32_t* d_prefix_len, int32_t* d_tail,
                                       int32_t* d_tail_len, int32_t* d_copies, int32_t* d_n_copies, int32_t* d_ok, war_stream_t stream) {
    war_status_t st = check_pages(p);
    if (st != WAR_OK) return st;
    if (P < 1 || P > kMaxTail || !d_n_copies || !d_ok) return WAR_ERR_INVALID_ARG;
    if (p->B > 0 && (!d_src || !d_prefix_len || !d_tail || !d_tail_len || !d_copies)) return WAR_ERR_INVALID_ARG;   // (without requests both words are written all the same)
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    int sms;
    st = device_setup(&sms);
    if (st != WAR_OK) return st;
    return war_launch_behind(pages_fork_kernel, kCluster, kThreads, sizeof(ForkShared), kCluster, stream, *p, d_src, P, d_prefix_len, d_tail, d_tail_len, d_copies, d_n_copies,
                          d_ok, status_word);
}

extern "C" size_t war_pages_compact_workspace_bytes(int64_t num_pages) {
    return num_pages < 1 || num_pages > (1ll << 30) ? 0 : (size_t)num_pages * 3 * sizeof(int32_t);
}

extern "C" war_status_t war_pages_compact(const war_pages_t* p, void* d_workspace, int32_t max_copies, int32_t* d_copies,
                                          int32_t* d_n_copies, int32_t* d_top, war_stream_t stream) {
    war_status_t st = check_pages(p);
    if (st != WAR_OK) return st;
    if (max_copies < 0 || !p->d_refs || !p->d_free) return WAR_ERR_INVALID_ARG;
    if (!d_workspace || ((uintptr_t)d_workspace & 3) || (!d_copies && max_copies > 0) || !d_n_copies || !d_top) return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    int sms;
    st = device_setup(&sms);
    if (st != WAR_OK) return st;
    return war_launch_behind(pages_compact_kernel, kCluster, kThreads, 0, kCluster, stream, *p, (int32_t*)d_workspace, max_copies, d_copies, d_n_copies, d_top, status_word);
}

extern "C" war_status_t war_prefix_groups(const int32_t* d_page_table, const int32_t* d_prefix_len, const int32_t* d_tail_len, int32_t B,
                                          int32_t page_size, int32_t max_pages_per_req, int32_t min_shared, int32_t* d_leader,
                                          int32_t* d_shared_len, war_stream_t stream) {
    if (B < 0 || page_size < 1 || max_pages_per_req < 1 || min_shared < 1) return WAR_ERR_INVALID_ARG;
    if (B > kMaxB) return WAR_ERR_UNSUPPORTED;
    if (B == 0) return WAR_OK;
    if (!d_page_table || !d_prefix_len || !d_leader || !d_shared_len) return WAR_ERR_INVALID_ARG;
    const int column = (min_shared - 1) / page_size;
    return war_launch_behind(prefix_groups_kernel, B, kGroupThreads, 0, 1, stream, d_page_table, d_prefix_len, d_tail_len, B, page_size,
                             max_pages_per_req, column, d_leader, d_shared_len);
}

extern "C" war_status_t war_pages_copy(const int32_t* d_copies, const int32_t* d_n_copies, int32_t max_copies, void* d_kpool, void* d_vpool,
                                       float* d_kscale, float* d_vscale, const war_pages_copy_params_t* q, war_stream_t stream) {
    if (!q || max_copies < 0 || q->Hkv < 1 || q->Hkv > 65535 || q->page_size < 1 || q->num_pages < 1) return WAR_ERR_INVALID_ARG;
    if (q->kv_type != kKvBf16 && q->kv_type != kKvE4M3 && q->kv_type != kKvE5M2) return WAR_ERR_INVALID_ARG;
    if (q->D != 128 || q->num_pages > (1ll << 30)) return WAR_ERR_UNSUPPORTED;
    const bool quant = q->kv_type != kKvBf16;
    if (quant && !war_quant_block_ok(q->page_size, q->scale_block)) return WAR_ERR_UNSUPPORTED;
    if (quant && q->page_size / q->scale_block > 32) return WAR_ERR_UNSUPPORTED;
    const int size = quant ? 1 : 2;
    if (!war_rows_aligned(q->kpool_strides, size) || !war_rows_aligned(q->vpool_strides, size)) return WAR_ERR_UNSUPPORTED;
    if (max_copies == 0) return WAR_OK;
    if (!d_copies || !d_n_copies || !d_kpool || !d_vpool || (quant && (!d_kscale || !d_vscale))) return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_kpool | (uintptr_t)d_vpool) & 15) return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    int sms;
    const war_status_t st = device_setup(&sms);
    if (st != WAR_OK) return st;
    CopyArgs a;
    a.k = (uint8_t*)d_kpool; a.v = (uint8_t*)d_vpool; a.kscale = d_kscale; a.vscale = d_vscale;
    for (int i = 0; i < 3; ++i) { a.ks[i] = q->kpool_strides[i] * size; a.vs[i] = q->vpool_strides[i] * size; }
    a.copies = d_copies; a.n_copies = d_n_copies; a.num_pages = q->num_pages; a.max_copies = max_copies;
    a.Hkv = q->Hkv; a.page_size = q->page_size; a.block = quant ? q->scale_block : 0;
    const long long blocks = ((long long)max_copies * 2 * q->Hkv + kCopyWarps - 1) / kCopyWarps;
    const int grid = (int)(blocks < sms * 8ll ? blocks : sms * 8ll);
    return war_launch_behind(quant ? pages_copy_kernel<8> : pages_copy_kernel<16>, grid, kCopyWarps * 32, 0, 1, stream, a, status_word);
}
