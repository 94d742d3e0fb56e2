// The target's choice after every slot of a draft tree: penalties, biases and grammar masks on the logits, then the
// largest value (and, if asked for, the processed logits).
//
// The logits are the traffic (64 times 131072 values a request against a few thousand context tokens), so a row is read
// once, 16 bytes a lane, and what the penalties need is looked up on chip: a cluster of up to eight thread blocks takes
// one request, each block a slice of the vocabulary, and counts the context's tokens that
// fall into it (each block reads the whole context; sending counts to the owner across the cluster took 2.5 times as long).  Rows are independent of each other (tokens on a
// slot's path are looked up in the tree, not written into the counters), so warps take pieces of rows without a barrier; the
// winners of a row meet in one 64-bit maximum per block, and the cluster's first block compares the slices.  Ties go to the
// lowest token, whatever the order of the atomics.
//   choice only, penalties that cannot raise a value (repetition >= 1, the others >= 0: the usual case): a logit at or below
//     the best processed value so far cannot win, so eight are dismissed with one packed maximum and only candidates are
//     looked up and processed (a few hundred a row)
//   processed logits wanted, or penalties that may raise: every value goes through the arithmetic, without branches
//   tokens with a bias, and tokens of the tree, are few: each warp goes through them after its piece of a row
//
// Measured: the choice for 256 requests of 8 slots and 32000 bf16 logits with contexts of up to 32768 tokens takes 90 us, of
// which the rows alone (no penalties, biases, masks) 45 (131 MB, 2.9 TB/s: two thread blocks' tables fill an SM, the start of
// a row has no bar yet, and 512 blocks go through in two waves), counting the contexts about 25 and looking candidates up the
// rest; looking every value up, as a first version did, took 449.  All values of 32 requests of 32 slots and 131071
// float32 logits: 400 us for 1.09 GB (2.7 TB/s), 202 without penalties, biases and masks; there the arithmetic, about 280 instructions for 128
// values, is the bound.  One slot of 8 requests: 9.7 us, a launch and four dependent reads.
#include <cuda_bf16.h>
#include <cooperative_groups.h>
#include "war_common.cuh"
#include "war_attn_plan.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kMaxSlots = 64;
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSlices = 8;                 // thread blocks of a cluster
constexpr int kMaxSlice = 32768;              // tokens a block can hold: 6 bytes and a bit each, of 227 KB
constexpr int kMaxVocab = kMaxSlices * kMaxSlice;
constexpr int kSegment = 1024;                // logits of a row that a warp takes at a time
constexpr int kMaxBias = 65534;               // bias entries of a request (numbered in 16 bits)
constexpr uint32_t kSeen = 0x80000000u;

struct TargetArgs {
    const void* logits; void* out;
    const int32_t *num_nodes, *ids, *parent, *ctx, *prompt_len, *bias_ids;
    const int64_t *ctx_off, *bias_off;
    const float *repetition, *presence, *frequency, *bias_val;
    const uint32_t* mask;
    int32_t* target;
    int* status_word;
    long long ls[2], os[2], ms[2];            // strides (request, slot) of logits and out in elements, of the mask in words
    int N, V, slice, words;                   // words: mask words of a row
    int count;                                // 1: count context tokens (a penalty is given)
    int path;                                 // 1: ids are given (tokens on a slot's path count too)
    int aligned;                              // 1: every row of logits starts on 16 bytes
};

struct Shared {
    unsigned long long best[kMaxSlots];       // (ordered value << 32) | ~token; 0: none
    unsigned long long anc[kMaxSlots];
    uint32_t bar[kMaxSlots];                  // ordered value that some warp has found in the row; 0: none
    int ids[kMaxSlots];
    int bad;
};

template <class T> struct Wide;
template <> struct Wide<float> {
    static constexpr int kPer = 4;
    static __device__ __forceinline__ void widen(const uint4& u, float* x) {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 narrow(const float* x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __noinline__ uint4 part(const float* p, int from, int to) {    // elements from .. to - 1, -inf elsewhere
        uint4 r;
        r.x = from <= 0 && to > 0 ? __float_as_uint(p[0]) : 0xff800000u;
        r.y = from <= 1 && to > 1 ? __float_as_uint(p[1]) : 0xff800000u;
        r.z = from <= 2 && to > 2 ? __float_as_uint(p[2]) : 0xff800000u;
        r.w = from <= 3 && to > 3 ? __float_as_uint(p[3]) : 0xff800000u;
        return r;
    }
    static __device__ __forceinline__ uint4 keep(const uint4& u, uint32_t ok) {      // -inf where ok's bit is clear
        return make_uint4(ok & 1 ? u.x : 0xff800000u, ok & 2 ? u.y : 0xff800000u, ok & 4 ? u.z : 0xff800000u, ok & 8 ? u.w : 0xff800000u);
    }
    static __device__ __forceinline__ int find(const uint4& u, float x) {            // an element that equals x, if one does
        return __uint_as_float(u.x) == x ? 0 : __uint_as_float(u.y) == x ? 1 : __uint_as_float(u.z) == x ? 2 : 3;
    }
    // the largest value that is no NaN (NaN: all are)
    static __device__ __forceinline__ float top(const uint4& u) {
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
    static __device__ __forceinline__ float pick(const uint4& u, int i) { return __uint_as_float(i < 2 ? (i ? u.y : u.x) : (i == 2 ? u.z : u.w)); }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, float x) { *p = x; }
};
template <> struct Wide<__nv_bfloat16> {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ void widen(const uint4& u, float* x) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint4 narrow(const float* x) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __noinline__ uint4 part(const __nv_bfloat16* p, int from, int to) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = from <= 2 * i && to > 2 * i ? reinterpret_cast<const uint16_t*>(p)[2 * i] : 0xff80u;
            const uint32_t hi = from <= 2 * i + 1 && to > 2 * i + 1 ? reinterpret_cast<const uint16_t*>(p)[2 * i + 1] : 0xff80u;
            w[i] = lo | hi << 16;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ uint32_t keep2(uint32_t w, uint32_t ok) {
        const uint32_t m = (ok & 1 ? 0xffffu : 0u) | (ok & 2 ? 0xffff0000u : 0u);
        return (w & m) | (0xff80ff80u & ~m);
    }
    static __device__ __forceinline__ uint4 keep(const uint4& u, uint32_t ok) {
        return make_uint4(keep2(u.x, ok), keep2(u.y, ok >> 2), keep2(u.z, ok >> 4), keep2(u.w, ok >> 6));
    }
    static __device__ __forceinline__ int find(const uint4& u, float x) {
        int i = 7;
        if (__uint_as_float(u.w << 16) == x) i = 6;
        if (__uint_as_float(u.z & 0xffff0000u) == x) i = 5;
        if (__uint_as_float(u.z << 16) == x) i = 4;
        if (__uint_as_float(u.y & 0xffff0000u) == x) i = 3;
        if (__uint_as_float(u.y << 16) == x) i = 2;
        if (__uint_as_float(u.x & 0xffff0000u) == x) i = 1;
        if (__uint_as_float(u.x << 16) == x) i = 0;
        return i;
    }
    static __device__ __forceinline__ float top(const uint4& u) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&u);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ float pick(const uint4& u, int i) {
        const uint32_t w = i < 4 ? (i < 2 ? u.x : u.y) : (i < 6 ? u.z : u.w);
        return __uint_as_float((i & 1) ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// order-preserving map of a float that is no NaN and above -inf to an unsigned number above 0 (-0 counts as 0)
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t unordered(uint32_t u) { return (u & 0x80000000u) ? u & 0x7fffffffu : ~u; }

// 32 bits of a bit string from bit v on (the word after them is read too)
__device__ __forceinline__ uint32_t bits_at(const uint32_t* w, int v) { return __funnelshift_r(w[v >> 5], w[(v >> 5) + 1], v & 31); }

template <class T, bool kOut>
__global__ void __launch_bounds__(kThreads, 2)
war_target_kernel(const TargetArgs a) {
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), slices = (int)cluster.num_blocks();
    const int b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int W = a.slice, bit_words = W / 32;
    uint32_t* counter = smem;                                             // [W] generated occurrences, bit 31: in the context; when
    const float* const made_of = reinterpret_cast<const float*>(counter); //     all values are processed: as floats, -1 not in the context
    uint16_t* bias_at = reinterpret_cast<uint16_t*>(counter + (a.count ? W : 0));   // [W] bias entry + 1
    uint32_t* rare = reinterpret_cast<uint32_t*>(bias_at + (a.bias_off ? W : 0));   // [bit_words + 1] a bias, or some slot's token
    const int v0 = rank * W, v1 = min(a.V, v0 + W);

    const int n_in = a.num_nodes[b];
    long long c0 = 0, c1 = 0;
    if (a.count) { c0 = a.ctx_off[b]; c1 = a.ctx_off[b + 1]; }
    long long e0 = 0, e1 = 0;
    if (a.bias_off) { e0 = a.bias_off[b]; e1 = a.bias_off[b + 1]; }
    int bad = 0;
    if (n_in < 0 || n_in > a.N) bad = WAR_ERR_BAD_TREE;
    if (c0 < 0 || c1 < c0 || c1 - c0 >= (1ll << 31) || e0 < 0 || e1 < e0 || e1 - e0 > kMaxBias) bad = WAR_ERR_INVALID_ARG;
    if (c1 > c0 && !a.ctx) bad = WAR_ERR_INVALID_ARG;
    for (int x = tid; x < bit_words + 1; x += kThreads) rare[x] = 0;
    const uint4 zero = make_uint4(0, 0, 0, 0);                            // (W is a multiple of 32)
    if (a.count) for (int x = tid; x < W / 4; x += kThreads) reinterpret_cast<uint4*>(counter)[x] = zero;
    if (a.bias_off) for (int x = tid; x < W / 8; x += kThreads) reinterpret_cast<uint4*>(bias_at)[x] = zero;
    if (tid < kMaxSlots) { sh.best[tid] = 0; sh.bar[tid] = 0; sh.ids[tid] = -1; }
    if (warp == 0) {
        // ancestor-or-self masks by pointer jumping; the root's bit is cleared (it is the context's last token)
        const int n = bad ? 0 : n_in;
        const int32_t* prow = a.parent + (size_t)b * a.N;
        int p0 = 0, p1 = 0;
        bool wrong = false;
        if (a.path) {
            p0 = lane > 0 && lane < n ? prow[lane] : 0; p1 = lane + 32 < n ? prow[lane + 32] : 0;
            wrong = (lane > 0 && lane < n && (p0 < 0 || p0 >= lane)) || (lane + 32 < n && (p1 < 0 || p1 >= lane + 32));
        }
        wrong = __any_sync(0xffffffffu, wrong);
        if (wrong) { p0 = 0; p1 = 0; }
        unsigned long long m0 = 1ull << lane, m1 = 1ull << (lane + 32);
        for (int r = 0; r < 6; ++r) {
            const unsigned long long m00 = __shfl_sync(0xffffffffu, m0, p0 & 31), m01 = __shfl_sync(0xffffffffu, m1, p0 & 31);
            const unsigned long long m10 = __shfl_sync(0xffffffffu, m0, p1 & 31), m11 = __shfl_sync(0xffffffffu, m1, p1 & 31);
            const int q00 = __shfl_sync(0xffffffffu, p0, p0 & 31), q01 = __shfl_sync(0xffffffffu, p1, p0 & 31);
            const int q10 = __shfl_sync(0xffffffffu, p0, p1 & 31), q11 = __shfl_sync(0xffffffffu, p1, p1 & 31);
            m0 |= p0 >= 32 ? m01 : m00; m1 |= p1 >= 32 ? m11 : m10;
            p0 = p0 >= 32 ? q01 : q00; p1 = p1 >= 32 ? q11 : q10;
        }
        sh.anc[lane] = m0 & ~1ull; sh.anc[lane + 32] = m1 & ~1ull;
        if (lane == 0) sh.bad = bad ? bad : (wrong ? WAR_ERR_BAD_TREE : 0);
    }
    __syncthreads();                                                      // the tables are cleared
    bad = sh.bad;
    const int n = bad ? 0 : n_in;

    if (n > 0) {
        if (a.count) {
            // every block reads the context and counts the tokens of its slice
            const int32_t* ctx = a.ctx + c0;
            const int len = (int)(c1 - c0), made = a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
#pragma unroll 8
            for (int x = tid; x < made; x += kThreads) {
                const int tok = ctx[x];
                if (tok >= v0 && tok < v1) atomicOr(&counter[tok - v0], kSeen);
            }
#pragma unroll 8
            for (int x = made + tid; x < len; x += kThreads) {
                const int tok = ctx[x];
                if (tok >= v0 && tok < v1) atomicAdd(&counter[tok - v0], 1u);
            }
        }
        if (a.bias_off) {
            // the last entry of a token counts: the largest number in its half of a word
            for (long long e = e0 + tid; e < e1; e += kThreads) {
                const int tok = a.bias_ids[e];
                if (tok < v0 || tok >= v1) continue;
                const int l = tok - v0, sh16 = (l & 1) * 16;
                const uint32_t k = (uint32_t)(e - e0 + 1);
                uint32_t* at = reinterpret_cast<uint32_t*>(bias_at) + (l >> 1);
                uint32_t now = *reinterpret_cast<volatile uint32_t*>(at);
                while (((now >> sh16) & 0xffffu) < k) {
                    const uint32_t before = now;
                    now = atomicCAS(at, before, (before & ~(0xffffu << sh16)) | (k << sh16));
                    if (now == before) break;
                }
                atomicOr(&rare[l >> 5], 1u << (l & 31));
            }
        }
        if (a.path && tid < kMaxSlots && tid > 0 && tid < n) {
            const int tok = a.ids[(size_t)b * a.N + tid];
            sh.ids[tid] = tok;
            if (a.count && tok >= v0 && tok < v1) {
                atomicOr(&rare[(tok - v0) >> 5], 1u << ((tok - v0) & 31));
            }
        }
    }
    __syncthreads();                                                      // all tokens are counted
    const float rep = a.repetition ? a.repetition[b] : 1.f, pres = a.presence ? a.presence[b] : 0.f, freq = a.frequency ? a.frequency[b] : 0.f;
    const bool dismiss = !kOut && rep >= 1.f && pres >= 0.f && freq >= 0.f;          // (uniform)
    auto made_from = [](uint32_t c) -> float { return c == 0 ? -1.f : (float)(c & ~kSeen); };
    if (n > 0 && a.count && !dismiss) {
        for (int x = tid; x < W; x += kThreads) counter[x] = __float_as_uint(made_from(counter[x]));
        __syncthreads();
    }
    // a value after the penalties; made < 0: neither in the context nor on the path
    auto penalise = [&](float x, float made) -> float {
        if (made < 0.f) return x;
        x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
        x = __fsub_rn(x, __fmul_rn(freq, made));
        return made > 0.f ? __fsub_rn(x, pres) : x;
    };

    // the same without branches, where |x| is inside [2^-60, 2^60] (Markstein's division: a quotient from the rounded reciprocal
    // that the residual corrects, here twice; it is the rounded quotient as long as nothing leaves the normal range)
    const float rep_inv = __frcp_rn(rep);
    const bool rep_plain = rep >= 0x1p-60f && rep <= 0x1p60f;
    auto penalise_plain = [&](float x, float made) -> float {
        float q = __fmul_rn(x, rep_inv);
        q = __fmaf_rn(__fmaf_rn(-q, rep, x), rep_inv, q);
        q = __fmaf_rn(__fmaf_rn(-q, rep, x), rep_inv, q);
        float y = x > 0.f ? q : __fmul_rn(x, rep);
        y = __fsub_rn(y, __fmul_rn(freq, made));
        y = made > 0.f ? __fsub_rn(y, pres) : y;
        return made < 0.f ? x : y;
    };

    constexpr int kPer = Wide<T>::kPer;
    constexpr int kLoads = kSegment / (32 * kPer);
    const int z = blockIdx.z, zs = gridDim.z;
    const int segments = v1 > v0 ? (v1 - v0 + (a.aligned ? 0 : kPer - 1) + kSegment - 1) / kSegment : 0;
    const int rows = n > z ? (n - z + zs - 1) / zs : 0;                   // rows z, z + zs, ... below n
    // a warp's pieces follow each other, so that a row's best value is known when most of it is read
    const int tasks = rows * segments;
    int of_row = -1, best_v = 0x7fffffff;
    float best = -INFINITY, bar = -INFINITY;                              // a lane's best of the row; what a candidate must exceed
    auto flush = [&]() {                                                  // the warp's best of the row goes to the block's
        unsigned long long key = best > -INFINITY ? ((unsigned long long)ordered(best) << 32) | (uint32_t)~best_v : 0ull;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, o);
            key = other > key ? other : key;
        }
        if (lane == 0 && key) atomicMax(&sh.best[of_row], key);
    };
    for (int task = (int)((long long)tasks * warp / kWarps); task < (int)((long long)tasks * (warp + 1) / kWarps); ++task) {
        const int rj = task / segments, seg = task - rj * segments, j = z + rj * zs;
        if (j != of_row) {
            if (of_row >= 0) flush();
            of_row = j; best = -INFINITY; bar = -INFINITY; best_v = 0x7fffffff;
        }
        const T* row = reinterpret_cast<const T*>(a.logits) + b * a.ls[0] + j * a.ls[1];
        T* out = kOut ? reinterpret_cast<T*>(a.out) + b * a.os[0] + j * a.os[1] : nullptr;
        const uint32_t* mask = a.mask ? a.mask + b * a.ms[0] + j * a.ms[1] : nullptr;
        // elements between the 16-byte boundary at or before the slice's first logit and that logit
        const int skew = (int)(((uintptr_t)(row + v0) & 15) / sizeof(T));
        const int first = v0 - skew + seg * kSegment;                     // a 16-byte boundary
        if (first >= v1) continue;
        const bool out_wide = kOut && (((uintptr_t)(out + first)) & 15) == 0;
        const bool table_wide = (skew & 3) == 0;
        // what another warp found in the row counts as well (values equal to it still have to be looked at: they may stand before it)
        if (dismiss) {
            const uint32_t o = *reinterpret_cast<volatile uint32_t*>(&sh.bar[j]);
            if (o) bar = fmaxf(bar, __uint_as_float(unordered(o - (o == 0x80000000u ? 2 : 1))));
        }
        const float bar_in = bar;
        const bool inner = first >= v0 && first + kSegment <= v1;         // (uniform) nothing ends in this piece
        auto fetch = [&](int u) -> uint4 {
            const int v = first + (u * 32 + lane) * kPer;
            if (inner || (v >= v0 && v + kPer <= v1)) return __ldcs(reinterpret_cast<const uint4*>(row + v));
            // (a slice may begin or end inside 16 bytes)
            return v + kPer > v0 && v < v1 ? Wide<T>::part(row + v, v0 - v, v1 - v) : Wide<T>::nothing();
        };
        // the piece's mask words: at most 33, a lane each; tokens that may be chosen here, rare ones are looked at below
        uint32_t m_lane = 0xffffffffu, m_last = 0xffffffffu;
        const int w0 = first >> 5;
        auto load_mask = [&]() {
            if (mask) {
                const int w = w0 + lane;
                m_lane = w >= 0 && w < a.words ? mask[w] : 0;
                m_last = w0 + 32 < a.words && skew ? mask[w0 + 32] : 0;
            }
        };
        auto allowed_at = [&](int v) -> uint32_t {
            if (!mask) return 0xffffffffu;
            const int k = (v >> 5) - w0;
            const uint32_t w = __shfl_sync(0xffffffffu, m_lane, k & 31);
            if (!skew) return w >> (v & 31);
            const uint32_t next = __shfl_sync(0xffffffffu, m_lane, (k + 1) & 31);
            return __funnelshift_r(k == 32 ? m_last : w, k == 31 ? m_last : next, v & 31);      // (v + i never reaches word 33)
        };
        auto rare_at = [&](int v) -> uint32_t {                           // (bits past the slice's do not matter)
            if (inner) return bits_at(rare, v - v0);
            return v >= v0 && v < v1 ? bits_at(rare, v - v0) : v < v0 && v + kPer > v0 ? rare[0] << (v0 - v) : 0;
        };
        if (dismiss) {
            uint4 in[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) in[u] = fetch(u);
            float top = Wide<T>::top(in[0]);
#pragma unroll
            for (int u = 1; u < kLoads; ++u) top = fmaxf(top, Wide<T>::top(in[u]));
            if (__any_sync(0xffffffffu, top > bar)) {
                load_mask();
#pragma unroll
                for (int u = 0; u < kLoads; ++u) {
                    const int v = first + (u * 32 + lane) * kPer;
                    in[u] = Wide<T>::keep(in[u], allowed_at(v) & ~rare_at(v));
                }
                // each lane looks at its largest: after that most others are at or below the bar
                const float from = bar;
                while (true) {
                    uint4 q = in[0];
                    int at = 0, i = 0;
                    top = Wide<T>::top(q);
#pragma unroll
                    for (int u = 1; u < kLoads; ++u) {
                        const float t = Wide<T>::top(in[u]);
                        if (t > top || !(top == top)) { top = t; q = in[u]; at = u; }
                    }
                    const bool look = top > from && top >= bar;
                    if (!__any_sync(0xffffffffu, look)) break;
                    i = Wide<T>::find(q, top);
                    if (look) {
                        const int v = first + (at * 32 + lane) * kPer + i;
                        const float y = a.count ? penalise(top, made_from(counter[v - v0])) : top;
                        if (y > best || (y == best && v < best_v && y > -INFINITY)) { best = y; best_v = v; }
                        q = Wide<T>::keep(q, ~(1u << i));
#pragma unroll
                        for (int u = 0; u < kLoads; ++u) if (at == u) in[u] = q;
                    }
                    bar = fmaxf(bar, __uint_as_float(unordered(__reduce_max_sync(0xffffffffu, ordered(best)))));
                }
            }
        } else {
            // the next piece's lines come to L2 meanwhile (without penalties, biases and masks 240 -> 202 us at the size above)
            const int next = first + kSegment + lane * (128 / (int)sizeof(T));
            if (lane * 128 < kSegment * (int)sizeof(T) && next < v1) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + next));
            // (rolled, three loads ahead: unrolled, its code no longer stays in the instruction cache)
            uint4 in0 = fetch(0), in1 = fetch(1), in2 = fetch(2);
            load_mask();
#pragma unroll 1
            for (int u = 0; u < kLoads; ++u) {
                const uint4 in = in0;
                in0 = in1; in1 = in2;
                if (u + 3 < kLoads) in2 = fetch(u + 3);
                const int v = first + (u * 32 + lane) * kPer;
                const uint32_t allowed = allowed_at(v), few = rare_at(v) & ((1u << kPer) - 1), ok = allowed & ~few;
                if (!inner && (v + kPer <= v0 || v >= v1)) continue;
                float x[kPer];
                Wide<T>::widen(in, x);
                if (a.count) {
                    float made[kPer];
                    if (table_wide && (inner || (v >= v0 && v + kPer <= v1))) {
#pragma unroll
                        for (int i = 0; i < kPer; i += 4) *reinterpret_cast<float4*>(made + i) = *reinterpret_cast<const float4*>(made_of + (v - v0) + i);
                    } else if (inner) {
#pragma unroll
                        for (int i = 0; i < kPer; ++i) made[i] = made_of[v - v0 + i];
                    } else {
#pragma unroll
                        for (int i = 0; i < kPer; ++i) made[i] = made_of[min(max(v + i - v0, 0), W - 1)];
                    }
                    float seen = made[0], low = fabsf(x[0]), high = x[0];
#pragma unroll
                    for (int i = 1; i < kPer; ++i) { seen = fmaxf(seen, made[i]); low = fminf(low, fabsf(x[i])); high = fmaxf(high, x[i]); }
                    if (seen >= 0.f) {
                        if (low >= 0x1p-60f && high <= 0x1p60f && rep_plain) {
#pragma unroll
                            for (int i = 0; i < kPer; ++i) x[i] = penalise_plain(x[i], made[i]);
                        } else {
#pragma unroll
                            for (int i = 0; i < kPer; ++i) x[i] = penalise(x[i], made[i]);
                        }
                    }
                }
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    x[i] = (ok >> i) & 1u ? x[i] : -INFINITY;
                    top = fmaxf(top, x[i]);
                }
                if (!inner && (v < v0 || v + kPer > v1)) {
                    top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) if (v + i >= v0 && v + i < v1) top = fmaxf(top, x[i]);
                }
                if (top > best) {
                    best = top;
#pragma unroll
                    for (int i = kPer - 1; i >= 0; --i) best_v = x[i] == top && v + i >= v0 ? v + i : best_v;
                }
                if (kOut) {
                    if (few) {                                            // as they were, for the list below (out may be the logits)
#pragma unroll
                        for (int i = 0; i < kPer; ++i) x[i] = (few >> i) & 1u ? Wide<T>::pick(in, i) : x[i];
                    }
                    if (out_wide && (inner || (v >= v0 && v + kPer <= v1))) __stcs(reinterpret_cast<uint4*>(out + v), Wide<T>::narrow(x));
                    else {
#pragma unroll
                        for (int i = 0; i < kPer; ++i) if (inner || (v + i >= v0 && v + i < v1)) Wide<T>::store(out + v + i, x[i]);
                    }
                }
            }
        }
        // tokens with a bias and tokens of the tree, if they lie in this piece
        __syncwarp();
        const int l0 = max(first, v0) - v0, l1 = min(first + kSegment, v1) - v0;
        for (int w = (l0 >> 5) + lane; w * 32 < l1; w += 32) for (uint32_t m = rare[w]; m; m &= m - 1) {
            const int l = w * 32 + __ffs(m) - 1, v = v0 + l;
            if (l < l0 || l >= l1) continue;
            float x = Wide<T>::load(row + v);
            if (a.count) {
                float made = dismiss ? made_from(counter[l]) : made_of[l];
                int on_path = 0;
                for (unsigned long long m = sh.anc[j]; m; m &= m - 1) on_path += sh.ids[__ffsll((long long)m) - 1] == v;
                if (on_path) made = fmaxf(made, 0.f) + (float)on_path;
                x = penalise(x, made);
            }
            if (a.bias_off) {
                const int k = bias_at[l];
                if (k) x = __fadd_rn(x, a.bias_val[e0 + k - 1]);
            }
            if (mask && !((mask[v >> 5] >> (v & 31)) & 1u)) x = -INFINITY;
            if (x > best || (x == best && v < best_v && x > -INFINITY)) { best = x; best_v = v; }
            if (kOut) Wide<T>::store(out + v, x);
        }
        // later values of the row must exceed the warp's best
        if (dismiss) {
            bar = fmaxf(bar, __uint_as_float(unordered(__reduce_max_sync(0xffffffffu, ordered(best)))));
            if (lane == 0 && bar > bar_in) atomicMax(&sh.bar[j], ordered(bar));
        }
        __syncwarp();
    }
    if (of_row >= 0) flush();
    cluster.sync();                                                       // every slice's winners are there
    if (rank == 0) {
        for (int j = tid; j < a.N; j += kThreads) {
            if (j % zs != z) continue;
            unsigned long long key = 0;
            if (j < n)
                for (int r = 0; r < slices; ++r) {
                    const unsigned long long other = *cluster.map_shared_rank(&sh.best[j], r);
                    key = other > key ? other : key;
                }
            a.target[(size_t)b * a.N + j] = key ? (int32_t)~(uint32_t)key : -1;
        }
        if (bad && tid == 0) war_set_device_status(a.status_word, bad);
    }
    cluster.sync();                                                       // no block leaves while its winners are read
}

constexpr int kMaxDevices = 64;
template <class T, bool kOut>
war_status_t allow_smem(int bytes) {
    static int allowed[kMaxDevices];                                     // (two threads may both set the attribute: the same call)
    int dev = 0;
    WAR_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return WAR_ERR_UNSUPPORTED;
    if (bytes > 40 * 1024 && !allowed[dev]) {                            // (48 KB need no request; the kernel's own variables are in them)
        WAR_CUDA_TRY(cudaFuncSetAttribute(war_target_kernel<T, kOut>, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024));
        allowed[dev] = 1;
    }
    return WAR_OK;
}

template <class T, bool kOut>
war_status_t launch(const TargetArgs& a, int slices, int B, int groups, size_t smem, cudaStream_t s) {
    const war_status_t st = allow_smem<T, kOut>((int)smem);
    if (st != WAR_OK) return st;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(slices, B, groups);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = slices; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, war_target_kernel<T, kOut>, a) != cudaSuccess) { (void)cudaGetLastError(); return WAR_ERR_CUDA; }
    return WAR_OK;
}

}  // namespace

extern "C" war_status_t war_target(const void* d_logits, const int32_t* d_num_nodes, const int32_t* d_ids, const int32_t* d_parent,
                                   const war_target_inputs_t* in, const war_target_params_t* p, int32_t* d_target, void* d_out,
                                   war_stream_t stream) {
    if (!p || !in) return WAR_ERR_INVALID_ARG;
    if (p->B < 0 || p->N < 1 || p->N > kMaxSlots || p->V < 1 || (p->dtype != 0 && p->dtype != 1)) return WAR_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
        if (p->logits_strides[i] < 0 || p->out_strides[i] < 0 || p->mask_strides[i] < 0) return WAR_ERR_INVALID_ARG;
    if (p->V > kMaxVocab || p->B > 65535) return WAR_ERR_UNSUPPORTED;
    if (p->B == 0) return WAR_OK;
    const int count = in->d_repetition || in->d_presence || in->d_frequency;
    if (!d_logits || !d_num_nodes || !d_target || (count && (!in->d_ctx_off || (!d_ids) != (!d_parent)))) return WAR_ERR_INVALID_ARG;
    if ((in->d_bias_off != nullptr) != (in->d_bias_ids != nullptr) || (in->d_bias_off != nullptr) != (in->d_bias_val != nullptr))
        return WAR_ERR_INVALID_ARG;
    const int size = p->dtype == 0 ? 2 : 4;
    if (((uintptr_t)d_logits | (uintptr_t)d_out) % size) return WAR_ERR_INVALID_ARG;
    int* status_word = war_status_word();
    if (!status_word) return WAR_ERR_CUDA;
    TargetArgs a;
    a.logits = d_logits; a.out = d_out; a.num_nodes = d_num_nodes; a.ids = d_ids; a.parent = d_parent;
    a.ctx = in->d_ctx; a.ctx_off = in->d_ctx_off; a.prompt_len = in->d_prompt_len;
    a.bias_off = in->d_bias_off; a.bias_ids = in->d_bias_ids; a.bias_val = in->d_bias_val;
    a.repetition = in->d_repetition; a.presence = in->d_presence; a.frequency = in->d_frequency;
    a.mask = (const uint32_t*)in->d_mask; a.target = d_target; a.status_word = status_word;
    for (int i = 0; i < 2; ++i) { a.ls[i] = p->logits_strides[i]; a.os[i] = p->out_strides[i]; a.ms[i] = p->mask_strides[i]; }
    a.N = p->N; a.V = p->V; a.words = (p->V + 31) / 32;
    a.count = count; a.path = count && d_ids != nullptr;
    a.aligned = (((uintptr_t)d_logits | (uintptr_t)(p->logits_strides[0] * size) | (uintptr_t)(p->logits_strides[1] * size)) & 15) == 0;
    // Slices of whole mask words, at most eight, at least four segments each (with two, 99
    // requests of 29 slots and 8266 tokens take 106 us, with four 90, with eight 116), so many that the requests fill the GPU (two thread
    // blocks an SM, 1.5 waves of them: 256 requests of 32000 tokens take 90 us with two slices, 106 with three); rows are dealt to more clusters of a request only if that leaves room: each counts the context again.
    const int n_sm = war_attn_sm_count(), resident = 2 * n_sm;
    if (n_sm <= 0) return WAR_ERR_CUDA;
    const int most = (p->V + kSegment * 4 - 1) / (kSegment * 4), least = (p->V + kMaxSlice - 1) / kMaxSlice;
    int slices = (resident * 3 / 2 + p->B - 1) / p->B;
    slices = slices > most ? most : slices;
    slices = slices > kMaxSlices ? kMaxSlices : slices < least ? least : slices;
    a.slice = ((p->V + slices - 1) / slices + 31) / 32 * 32;
    int groups = resident / (slices * p->B);
    groups = groups < 1 ? 1 : groups > p->N ? p->N : groups;
    const size_t smem = (size_t)(a.slice / 32 + 1) * 4 + (count ? (size_t)a.slice * 4 : 0) + (in->d_bias_off ? (size_t)a.slice * 2 : 0);
    if (p->dtype == 0) return d_out ? launch<__nv_bfloat16, true>(a, slices, p->B, groups, smem, stream) : launch<__nv_bfloat16, false>(a, slices, p->B, groups, smem, stream);
    return d_out ? launch<float, true>(a, slices, p->B, groups, smem, stream) : launch<float, false>(a, slices, p->B, groups, smem, stream);
}
