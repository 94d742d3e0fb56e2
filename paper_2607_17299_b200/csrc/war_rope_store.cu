// Rotary positions for a draft tree's queries and keys, and the write of its K and V rows into the paged cache.
//
//   (y, z) = (a * c - b * s, b * c + a * s)   for the pairs (a, b) of the first rot_dim elements of every head,
//   c = factor * cos(t), s = factor * sin(t), t = (prefix_len + depth of the slot) * inv_freq[pair]
//
// The angle of a far position does not fit 32 bits (2^20 radians leave a step of 2^-4 of one), so it is reduced in 64
// bits, in turns, and its sine and cosine are taken there too and rounded once (with the 32-bit functions half as many keys
// again fell on the wrong side of a code's border); everything else is 32-bit arithmetic with one rounding at the end.
//
// Nothing here computes much: each value is read once and written once, and what matters is that every SM has rows to
// move.  A thread block works for one request: it fills a table of (c, s) for the depths of the request's tree (shared
// by slots, heads and both roles), and its warps then take tasks,
//   rows    one slot, up to kHeadsPerTask heads: eight lanes a row, two groups of eight elements (16 bytes) a lane, chosen so
//           that an element and its partner are the same lane's; the lane's (c, s) stay in registers over the heads
//   blocks  (8-bit pools) one head's K or V rows of one scale block: largest magnitude first, then the scale, the
//           re-encoding of older rows if the scale has grown, and the new rows (turned again from the kept input)
// and the request's tasks are dealt over several thread blocks when there are few requests.
//
// Measured: 128 requests of 64 slots, 64 + 8 heads, bf16 pool (336 MB): 59 us, 5.7 TB/s (sixteen lanes a row with the partner
// fetched by shuffle took 93).  256 requests of 8 slots, 32 + 8 heads, e4m3 pool (46 MB): 17 to 18.5 us (37 before); no unit is at
// its limit there (issue slots 54 %, DRAM 13 %, 28 % of the warps resident): a warp's four to six tasks follow each other, each a chain
// of dependent instructions, and scale blocks pass their values twice.  One slot of 8 requests: 4.6 us, the chain of dependent reads.
#include <cuda_bf16.h>
#include <math.h>
#include "war_common.cuh"
#include "war_attn_plan.cuh"
#include "war_quant.cuh"

namespace {

constexpr int kMaxSlots = 64;
constexpr int kThreads = 384;
constexpr int kWarps = kThreads / 32;
constexpr int kHeadsPerTask = 8;
constexpr int kResident = 2;                  // thread blocks that an SM holds at a time
// How a lane's elements are laid out: kSplit (a pair is half the rotation apart), kAdjacent (a pair is two neighbours), both
// where the rotation covers whole lanes; kOdd takes every other rot_dim, through shared memory.
constexpr int kSplit = 0, kAdjacent = 1, kOdd = 2;
constexpr int kScratchRow = 136;              // floats from row to row: four rows' neighbours in different banks

struct StoreArgs {
    const __nv_bfloat16 *q, *k, *v;
    const float* inv_freq;
    const int32_t *page_table, *prefix_len, *num_nodes, *parent;
    uint8_t *kpool, *vpool;
    float *kscale, *vscale;
    __nv_bfloat16* q_out;
    int* status_word;
    long long qs[3], ks[3], vs[3];            // input strides (request, slot, head) in elements
    long long kp[3], vp[3];                   // pool strides (page, head, token) in elements
    long long num_pages;
    float factor;
    int N, Hq, Hkv, page_size, max_pages, half, interleaved, block, blocks_per_page;
    int chunks;                               // row tasks of a slot
    uint32_t hkv_magic, chunks_magic;         // for quotient()
    int page_shift, block_shift;              // logarithms of page_size (-1: no power of two) and block (8-bit pools)
};

// n / d for 0 <= n < 2^32 / d by a product with floor(2^32 / d) + 1 (a division by a run-time number is some 25 instructions, and
// a task has six); magic 0: a division.
__host__ __device__ __forceinline__ uint32_t magic_of(int d) { return d > 1 && d <= 4096 ? (uint32_t)((1ull << 32) / d + 1) : 0u; }
__device__ __forceinline__ int quotient(int n, int d, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)n, magic) : n / d; }

struct Raw { uint4 a, b; };                   // a lane's two groups of a row
struct Row { float a[8], b[8]; };
struct Turn { float c[8], s[8]; };            // of the lane's eight pairs

__device__ __forceinline__ void widen(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ Row widen(const Raw& r) {
    Row x;
    widen(r.a, x.a); widen(r.b, x.b);
    return x;
}
__device__ __forceinline__ uint4 narrow(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What a lane knows about its place in a row.
struct Place {
    int s, a, b;                              // lane of the row (0 to 7); first elements of its groups
    int half, interleaved;
    bool turns;                               // its elements rotate (kSplit, kAdjacent)
    float* scratch;                           // kScratchRow floats of this row's eight lanes (kOdd)
};
template <int kMode>
__device__ __forceinline__ Place place(int lane, int half, int interleaved, float* scratch) {
    Place p;
    p.s = lane & 7; p.half = half; p.interleaved = interleaved; p.scratch = scratch;
    const int g = half >> 3;                                              // lanes that rotate
    p.turns = p.s < g;
    const bool split = kMode == kSplit && p.turns;
    // kSplit: group s and the one half the rotation later; lanes past the rotation share the groups behind it: 2 * s and 2 * s + 1
    // kOdd: the lanes' groups side by side, in both halves of the head
    p.a = split || kMode == kOdd ? 8 * p.s : 16 * p.s;
    p.b = split ? 8 * p.s + half : kMode == kOdd ? 64 + 8 * p.s : 16 * p.s + 8;
    return p;
}

// Where pair i of a slot stands in its row of the table: so that eight lanes read 16 bytes each side by side.
template <int kMode>
__device__ __forceinline__ int table_at(int i, int half) {
    return kMode == kOdd ? i : ((i & 7) >> 1) * (half >> 3) * 2 + (i >> 3) * 2 + (i & 1);
}
template <int kMode>
__device__ __forceinline__ Turn load_turn(const float2* table, const Place& p) {
    Turn t;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float4 v = make_float4(1.f, 0.f, 1.f, 0.f);
        if (kMode != kOdd && p.turns) v = reinterpret_cast<const float4*>(table)[k * (p.half >> 3) + p.s];
        t.c[2 * k] = v.x; t.s[2 * k] = v.y; t.c[2 * k + 1] = v.z; t.s[2 * k + 1] = v.w;
    }
    return t;
}

// separate roundings of the two products: the value does not depend on which of them a fused operation would keep
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
    const float u = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)), v = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
    x = u; y = v;
}
// Rotates the rows of a warp, four of them.  All 32 lanes call it together.
template <int kMode>
__device__ __forceinline__ void rotate(Row& r, const Turn& t, const float2* table, const Place& p) {
    if constexpr (kMode == kSplit) {
        if (p.turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) turn_pair(r.a[i], r.b[i], t.c[i], t.s[i]);
        }
    } else if constexpr (kMode == kAdjacent) {
        if (p.turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                turn_pair(r.a[2 * i], r.a[2 * i + 1], t.c[i], t.s[i]);
                turn_pair(r.b[2 * i], r.b[2 * i + 1], t.c[i + 4], t.s[i + 4]);
            }
        }
    } else {
        __syncwarp();
        float4* const a4 = reinterpret_cast<float4*>(p.scratch + p.a);
        float4* const b4 = reinterpret_cast<float4*>(p.scratch + p.b);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a4[i] = make_float4(r.a[4 * i], r.a[4 * i + 1], r.a[4 * i + 2], r.a[4 * i + 3]);
            b4[i] = make_float4(r.b[4 * i], r.b[4 * i + 1], r.b[4 * i + 2], r.b[4 * i + 3]);
        }
        __syncwarp();
#pragma unroll 2
        for (int k = p.s; k < p.half; k += 8) {
            const float2 cs = table[k];
            float* x = p.scratch + (p.interleaved ? 2 * k : k);
            turn_pair(x[0], x[p.interleaved ? 1 : p.half], cs.x, cs.y);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 x = a4[i], y = b4[i];
            r.a[4 * i] = x.x; r.a[4 * i + 1] = x.y; r.a[4 * i + 2] = x.z; r.a[4 * i + 3] = x.w;
            r.b[4 * i] = y.x; r.b[4 * i + 1] = y.y; r.b[4 * i + 2] = y.z; r.b[4 * i + 3] = y.w;
        }
    }
}

template <int kv, int kMode>
__global__ void __launch_bounds__(kThreads, 2)
war_rope_store_kernel(const StoreArgs a, const int parts) {
    extern __shared__ __align__(16) float2 s_table[];                     // [depth, up to N of them][half]
    __shared__ int s_depth[kMaxSlots], s_levels;
    __shared__ __align__(16) float s_scratch[kMode == kOdd ? kWarps : 1][4][kScratchRow];
    const int b = blockIdx.x, part = blockIdx.y;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, side = lane >> 3;
    const int n = a.num_nodes[b], pl = a.prefix_len[b];
    bool bad = n < 0 || n > a.N || pl < 0;
    if (!bad && warp == 0) {
        // depth by pointer jumping: lane l holds slots l and l + 32; after round r the pointer is the 2^r-th ancestor
        const int32_t* prow = a.parent + (size_t)b * a.N;
        int p0 = lane > 0 && lane < n ? prow[lane] : 0, p1 = lane + 32 < n ? prow[lane + 32] : 0;
        const bool wrong = (lane > 0 && lane < n && (p0 < 0 || p0 >= lane)) || (lane + 32 < n && (p1 < 0 || p1 >= lane + 32));
        if (__any_sync(0xffffffffu, wrong)) {
            if (lane == 0) s_depth[0] = -1;
        } else {
            int d0 = lane > 0 && lane < n, d1 = lane + 32 < n;
            for (int r = 0; r < 6; ++r) {
                const int e00 = __shfl_sync(0xffffffffu, d0, p0 & 31), e01 = __shfl_sync(0xffffffffu, d1, p0 & 31);
                const int e10 = __shfl_sync(0xffffffffu, d0, p1 & 31), e11 = __shfl_sync(0xffffffffu, d1, p1 & 31);
                const int q00 = __shfl_sync(0xffffffffu, p0, p0 & 31), q01 = __shfl_sync(0xffffffffu, p1, p0 & 31);
                const int q10 = __shfl_sync(0xffffffffu, p0, p1 & 31), q11 = __shfl_sync(0xffffffffu, p1, p1 & 31);
                d0 += p0 >= 32 ? e01 : e00; d1 += p1 >= 32 ? e11 : e10;
                p0 = p0 >= 32 ? q01 : q00; p1 = p1 >= 32 ? q11 : q10;
            }
            s_depth[lane] = d0; s_depth[lane + 32] = d1;
            const int deepest = __reduce_max_sync(0xffffffffu, max(d0, d1));
            if (lane == 0) s_levels = deepest + 1;
        }
    }
    __syncthreads();
    bad = bad || s_depth[0] < 0;
    if (bad) {
        if (tid == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_TREE);
        return;
    }
    if (n == 0) return;
    if ((long long)pl + n > (long long)a.max_pages * a.page_size) {
        if (tid == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
        return;
    }
    const int32_t* pt = a.page_table + (size_t)b * a.max_pages;
    const int first_block = kv == kKvBf16 ? 0 : pl >> a.block_shift;
    const int blocks = kv == kKvBf16 ? 0 : ((pl + n - 1) >> a.block_shift) - first_block + 1;
    const int block_tasks = 2 * a.Hkv * blocks;
    const int heads = a.Hq + (kv == kKvBf16 ? 2 * a.Hkv : 0);             // heads the row tasks cover: q, then k and v of a bf16 pool
    const int chunks = a.chunks;
    auto page_index = [&](int pos) -> int { return a.page_shift >= 0 ? pos >> a.page_shift : pos / a.page_size; };
    const int tasks = block_tasks + n * chunks;
    const Place at = place<kMode>(lane, a.half, a.interleaved, s_scratch[kMode == kOdd ? warp : 0][side]);

    constexpr int kKept = 2;                                              // rows of a lane that are in registers at a time
    static_assert(kHeadsPerTask == 4 * kKept, "a row task is one load");
    Raw in[kKept];
    auto fetch = [&](int u, const __nv_bfloat16* src, bool valid) {
        in[u].a = in[u].b = make_uint4(0, 0, 0, 0);
        if (valid) {
            in[u].a = *reinterpret_cast<const uint4*>(src + at.a);
            in[u].b = *reinterpret_cast<const uint4*>(src + at.b);
        }
    };
    auto fetch_heads = [&](int j, int h0) {
#pragma unroll
        for (int u = 0; u < kKept; ++u) {
            const int h = h0 + 4 * u + side;
            fetch(u, h < a.Hq ? a.q + b * a.qs[0] + j * a.qs[1] + h * a.qs[2]
                     : h < a.Hq + a.Hkv ? a.k + b * a.ks[0] + j * a.ks[1] + (h - a.Hq) * a.ks[2]
                                        : a.v + b * a.vs[0] + j * a.vs[1] + (h - a.Hq - a.Hkv) * a.vs[2], h < heads);
        }
    };
    auto fetch_rows = [&](int which, int h, int j, int j1) {
        const long long* ss = which ? a.vs : a.ks;
        const __nv_bfloat16* src = (which ? a.v : a.k) + b * ss[0] + h * ss[2];
#pragma unroll
        for (int u = 0; u < kKept; ++u) fetch(u, src + (j + 4 * u + side) * ss[1], j + 4 * u + side < j1);
    };
    auto fetch_task = [&](int task) {
        if (task >= block_tasks) {
            const int r = task - block_tasks, j = quotient(r, chunks, a.chunks_magic);
            fetch_heads(j, (r - j * chunks) * kHeadsPerTask);
        } else {
            const int t = quotient(task >> 1, a.Hkv, a.hkv_magic), pos0 = (first_block + t) << a.block_shift;
            fetch_rows(task & 1, (task >> 1) - t * a.Hkv, max(0, pos0 - pl), min(n, pos0 + a.block - pl));
        }
    };
    // the first task's values arrive while the table is filled
    int task = part * kWarps + warp;
    if (task < tasks) fetch_task(task);
    for (int x = tid; x < s_levels * a.half; x += kThreads) {
        const int j = x / a.half, i = x - j * a.half;
        const double turns = (double)(pl + j) * ((double)a.inv_freq[i] * 0.15915494309189533577);
        double s, c;
        sincospi(2.0 * (turns - rint(turns)), &s, &c);
        s_table[j * a.half + table_at<kMode>(i, a.half)] = make_float2((float)(c * (double)a.factor), (float)(s * (double)a.factor));
    }
    __syncthreads();


    for (bool first = true; task < tasks; task += parts * kWarps, first = false) {
        if (!first) fetch_task(task);
        if (task >= block_tasks) {
            const int r = task - block_tasks, j = quotient(r, chunks, a.chunks_magic), h0 = (r - j * chunks) * kHeadsPerTask;
            const float2* table = s_table + s_depth[j] * a.half;
            const Turn turn = load_turn<kMode>(table, at);
            const int h1 = min(h0 + kHeadsPerTask, heads);
#pragma unroll
            for (int u = 0; u < kKept; ++u) {
                if (h0 + 4 * u >= h1) break;                              // (uniform: the warp's rows rotate together)
                const int h = h0 + 4 * u + side;
                Row row = widen(in[u]);
                rotate<kMode>(row, turn, table, at);
                if (h >= h1) continue;
                if (h < a.Hq + a.Hkv) { in[u].a = narrow(row.a); in[u].b = narrow(row.b); }    // v is copied as it is
                __nv_bfloat16* dst;
                if (h < a.Hq) {
                    dst = a.q_out + (((size_t)b * a.N + j) * a.Hq + h) * 128;
                } else {
                    const int pos = pl + j;
                    const int pi = page_index(pos);
                    const long long page = pt[pi];
                    if (page < 0 || page >= a.num_pages) {
                        if (at.s == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
                        continue;
                    }
                    const bool is_k = h < a.Hq + a.Hkv;
                    const long long* st = is_k ? a.kp : a.vp;
                    const int kh = h - a.Hq - (is_k ? 0 : a.Hkv);
                    dst = reinterpret_cast<__nv_bfloat16*>(is_k ? a.kpool : a.vpool) + page * st[0] + kh * st[1] + (long long)(pos - pi * a.page_size) * st[2];
                }
                *reinterpret_cast<uint4*>(dst + at.a) = in[u].a;
                *reinterpret_cast<uint4*>(dst + at.b) = in[u].b;
            }
            continue;
        }
        if constexpr (kv != kKvBf16) {
            // ---- one scale block of one head's K or V
            const int t = quotient(task >> 1, a.Hkv, a.hkv_magic), which = task & 1, h = (task >> 1) - t * a.Hkv;
            const int pos0 = (first_block + t) << a.block_shift;
            const int j0 = max(0, pos0 - pl), j1 = min(n, pos0 + a.block - pl);
            const int pi = page_index(pos0);
            const long long page = pt[pi];
            if (page < 0 || page >= a.num_pages) {
                if (lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
                continue;
            }
            const long long* ps = which ? a.vp : a.kp;
            const int row0 = pos0 - pi * a.page_size;
            uint8_t* dst = (which ? a.vpool : a.kpool) + page * ps[0] + h * ps[1] + (long long)row0 * ps[2];
            float* scale = (which ? a.vscale : a.kscale) + (page * a.Hkv + h) * a.blocks_per_page + (row0 >> a.block_shift);
            const int old = min(max(pl - pos0, 0), a.block);              // rows of earlier tokens in the block
            const float s_old = old > 0 ? *scale : 0.f;
            auto turned = [&](const Raw& raw, int j) -> Row {
                Row r = widen(raw);
                if (!which) {
                    const float2* table = s_table + s_depth[min(j + side, j1 - 1)] * a.half;
                    rotate<kMode>(r, load_turn<kMode>(table, at), table, at);
                }
                return r;
            };
            float top = 0.f;
            for (int j = j0; j < j1; j += 4 * kKept) {
                if (j > j0) fetch_rows(which, h, j, j1);
#pragma unroll
                for (int u = 0; u < kKept; ++u) {
                    if (j + 4 * u >= j1) break;                           // (uniform)
                    const Row r = turned(in[u], j + 4 * u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(r.a[i]), fabsf(r.b[i])));
                }
            }
            top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));    // (not negative, no NaN: ordered as integers)
            float s_new = fmaxf(s_old, quant::pow2_scale(top, kv));
            if (!(s_new > 0.f)) s_new = 1.f;
            if (s_new != s_old && old > 0) {
                const float ratio = s_old / s_new;
                for (int r = side; r < old; r += 4) {
                    uint4* p = reinterpret_cast<uint4*>(dst + r * ps[2]) + at.s;
                    const uint4 c = *p;
                    const uint2 lo = quant::recode8(make_uint2(c.x, c.y), ratio, kv), hi = quant::recode8(make_uint2(c.z, c.w), ratio, kv);
                    *p = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
            // dividing by a power of two is multiplying by its reciprocal; a scale that was there may be another number
            const bool pow2 = (__float_as_uint(s_new) & 0x7fffffu) == 0 && s_new >= kSmallestScale;
            const float inv = 1.f / s_new;
            auto codes = [&](float* x) -> uint2 {
                if (pow2) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= inv;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = __fdiv_rn(x[i], s_new);
                }
                return make_uint2(quant::encode2(x[0], x[1], kv) | (quant::encode2(x[2], x[3], kv) << 16),
                                  quant::encode2(x[4], x[5], kv) | (quant::encode2(x[6], x[7], kv) << 16));
            };
            for (int j = j0; j < j1; j += 4 * kKept) {
                if (j1 - j0 > 4 * kKept) fetch_rows(which, h, j, j1);     // (else they are there)
#pragma unroll
                for (int u = 0; u < kKept; ++u) {
                    const int x = j + 4 * u + side;
                    if (j + 4 * u >= j1) break;
                    Row r = turned(in[u], j + 4 * u);
                    if (x >= j1) continue;
                    uint8_t* to = dst + (long long)(pl + x - pos0) * ps[2];
                    *reinterpret_cast<uint2*>(to + at.a) = codes(r.a);
                    *reinterpret_cast<uint2*>(to + at.b) = codes(r.b);
                }
            }
            if (lane == 0 && s_new != s_old) *scale = s_new;
        }
    }
}

template <int kv, int kMode>
war_status_t launch(const StoreArgs& a, dim3 grid, size_t table, cudaStream_t s) {
    if (kMode == kOdd && table > 8 * 1024)                                // next to its scratch: past the 48 KB that need no request
        WAR_CUDA_TRY(cudaFuncSetAttribute(war_rope_store_kernel<kv, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024));
    war_rope_store_kernel<kv, kMode><<<grid, kThreads, table, s>>>(a, (int)grid.y);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
}
template <int kv>
war_status_t launch(const StoreArgs& a, int mode, dim3 grid, size_t table, cudaStream_t s) {
    return mode == kSplit ? launch<kv, kSplit>(a, grid, table, s) : mode == kAdjacent ? launch<kv, kAdjacent>(a, grid, table, s) : launch<kv, kOdd>(a, grid, table, s);
}

}  // namespace

extern "C" war_status_t war_rope_store(const void* d_q, const void* d_k, const void* d_v, const float* d_inv_freq,
                                       const int32_t* d_page_table, const int32_t* d_prefix_len, const int32_t* d_num_nodes,
                                       const int32_t* d_parent, const war_rope_store_params_t* p, void* d_kpool, void* d_vpool,
                                       float* d_kscale, float* d_vscale, void* d_q_out, war_stream_t stream) {
    if (!p) return WAR_ERR_INVALID_ARG;
    if (p->B < 0 || p->N < 1 || p->N > kMaxSlots || p->Hq < 0 || p->Hkv < 1 || p->page_size < 1 || p->max_pages_per_req < 1 ||
        p->num_pages < 1 || p->rot_dim < 0 || p->rot_dim > 128 || (p->rot_dim & 1) || p->kv_type < 0 || p->kv_type > 2 ||
        (p->interleaved != 0 && p->interleaved != 1) || !(fabsf(p->factor) <= 3.0e38f))
        return WAR_ERR_INVALID_ARG;
    if (p->D != 128) return WAR_ERR_UNSUPPORTED;
    if ((long long)p->max_pages_per_req * p->page_size >= (1ll << 30) || p->Hq > (1 << 20) || p->Hkv > (1 << 20)) return WAR_ERR_UNSUPPORTED;
    const int element = p->kv_type == kKvBf16 ? 2 : 1;
    if (p->kv_type != kKvBf16 && !war_quant_block_ok(p->page_size, p->scale_block)) return WAR_ERR_UNSUPPORTED;
    if (!war_rows_aligned(p->q_strides, 2) || !war_rows_aligned(p->k_strides, 2) || !war_rows_aligned(p->v_strides, 2) ||
        !war_rows_aligned(p->kpool_strides, element) || !war_rows_aligned(p->vpool_strides, element))
        return WAR_ERR_UNSUPPORTED;
    if (p->B == 0) return WAR_OK;
    if (!d_k || !d_v || !d_page_table || !d_prefix_len || !d_num_nodes || !d_parent || !d_kpool || !d_vpool ||
        (p->Hq > 0 && (!d_q || !d_q_out)) || (p->rot_dim > 0 && !d_inv_freq) || (p->kv_type != kKvBf16 && (!d_kscale || !d_vscale)))
        return WAR_ERR_INVALID_ARG;
    if (((uintptr_t)d_q | (uintptr_t)d_k | (uintptr_t)d_v | (uintptr_t)d_kpool | (uintptr_t)d_vpool | (uintptr_t)d_q_out) & 15)
        return WAR_ERR_UNSUPPORTED;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    StoreArgs a;
    a.q = (const __nv_bfloat16*)d_q; a.k = (const __nv_bfloat16*)d_k; a.v = (const __nv_bfloat16*)d_v;
    a.inv_freq = d_inv_freq; a.page_table = d_page_table; a.prefix_len = d_prefix_len; a.num_nodes = d_num_nodes; a.parent = d_parent;
    a.kpool = (uint8_t*)d_kpool; a.vpool = (uint8_t*)d_vpool; a.kscale = d_kscale; a.vscale = d_vscale;
    a.q_out = (__nv_bfloat16*)d_q_out; a.status_word = status_word;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = p->q_strides[i]; a.ks[i] = p->k_strides[i]; a.vs[i] = p->v_strides[i];
        a.kp[i] = p->kpool_strides[i]; a.vp[i] = p->vpool_strides[i];
    }
    a.num_pages = p->num_pages; a.factor = p->factor;
    a.N = p->N; a.Hq = p->Hq; a.Hkv = p->Hkv; a.page_size = p->page_size; a.max_pages = p->max_pages_per_req;
    a.half = p->rot_dim / 2; a.interleaved = p->interleaved;
    a.block = p->kv_type == kKvBf16 ? p->page_size : p->scale_block;
    a.blocks_per_page = p->page_size / a.block;
    a.page_shift = -1; a.block_shift = 0;
    for (int k = 0; k < 30; ++k) if (p->page_size == 1 << k) a.page_shift = k;
    while (p->kv_type != kKvBf16 && 1 << a.block_shift < a.block) ++a.block_shift;
    // how many thread blocks share a request: enough to fill the GPU, no more than there are tasks
    const long long heads = p->Hq + (p->kv_type == kKvBf16 ? 2ll * p->Hkv : 0);
    a.chunks = (int)((heads + kHeadsPerTask - 1) / kHeadsPerTask);
    a.hkv_magic = magic_of(p->Hkv); a.chunks_magic = magic_of(a.chunks);
    const long long tasks = (p->kv_type == kKvBf16 ? 0 : 2ll * p->Hkv * ((p->N + a.block - 2) / a.block + 1)) +
                            (long long)p->N * ((heads + kHeadsPerTask - 1) / kHeadsPerTask);
    const int n_sm = war_attn_sm_count();
    if (n_sm <= 0) return WAR_ERR_CUDA;
    long long parts = n_sm * kResident / p->B;
    if (parts > (tasks + kWarps - 1) / kWarps) parts = (tasks + kWarps - 1) / kWarps;
    if (parts < 1) parts = 1;
    const int mode = p->rot_dim % 16 != 0 ? kOdd : p->interleaved ? kAdjacent : kSplit;
    const size_t table = sizeof(float2) * (size_t)p->N * (size_t)(a.half > 0 ? a.half : 1);
    const dim3 grid(p->B, (unsigned)parts);
    return p->kv_type == kKvBf16 ? launch<kKvBf16>(a, mode, grid, table, stream)
         : p->kv_type == kKvE4M3 ? launch<kKvE4M3>(a, mode, grid, table, stream) : launch<kKvE5M2>(a, mode, grid, table, stream);
}

// Frequencies of the rotation, worked out on the host in 64 bits and rounded once.
extern "C" war_status_t war_rope_frequencies(const war_rope_freq_params_t* p, float* h_inv_freq, float* h_factor) {
    if (!p || (!h_inv_freq && p->rot_dim > 0)) return WAR_ERR_INVALID_ARG;
    const int n = p->rot_dim / 2;
    if (p->rot_dim < 0 || p->rot_dim > 128 || (p->rot_dim & 1) || p->kind < 0 || p->kind > 4 || !(p->base > 1.0) || !(p->base < 1e300))
        return WAR_ERR_INVALID_ARG;
    if (p->kind != WAR_ROPE_PLAIN && (!(p->scale >= 1.0) || !(p->scale < 1e9))) return WAR_ERR_INVALID_ARG;
    const bool by_length = p->kind == WAR_ROPE_RAMP || p->kind == WAR_ROPE_BANDS;
    if (by_length && (!(p->original_length > 0.0) || !(p->slow > 0.0) || !(p->fast > p->slow) || !(p->fast < 1e9) || !(p->original_length < 1e12)))
        return WAR_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    double base = p->base;
    if (p->kind == WAR_ROPE_BASE && p->rot_dim > 2) base *= pow(p->scale, (double)p->rot_dim / (double)(p->rot_dim - 2));
    // ramp: the pair index at which a wave makes `turns` turns over the original length
    auto index_of = [&](double turns) { return (double)p->rot_dim * log(p->original_length / (turns * two_pi)) / (2.0 * log(p->base)); };
    double lo = 0.0, hi = 1.0;
    if (p->kind == WAR_ROPE_RAMP) {
        lo = fmax(floor(index_of(p->fast)), 0.0);
        hi = fmin(ceil(index_of(p->slow)), (double)p->rot_dim - 1.0);
        if (hi <= lo) hi = lo + 0.001;
    }
    for (int i = 0; i < n; ++i) {
        double f = pow(base, -2.0 * i / (double)p->rot_dim);
        if (p->kind == WAR_ROPE_LINEAR) f /= p->scale;
        if (p->kind == WAR_ROPE_RAMP) {
            const double slow_share = fmin(fmax(((double)i - lo) / (hi - lo), 0.0), 1.0);
            f = f / p->scale * slow_share + f * (1.0 - slow_share);
        }
        if (p->kind == WAR_ROPE_BANDS) {
            const double turns = p->original_length * f / two_pi;          // of this wave over the original length
            const double fast_share = fmin(fmax((turns - p->slow) / (p->fast - p->slow), 0.0), 1.0);
            f = f / p->scale * (1.0 - fast_share) + f * fast_share;
        }
        h_inv_freq[i] = (float)f;
    }
    if (h_factor) *h_factor = p->kind == WAR_ROPE_RAMP ? (float)(0.1 * log(p->scale) + 1.0) : 1.f;
    return WAR_OK;
}
