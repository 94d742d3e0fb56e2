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
// move.  A thread block works for one request: it fills a table of (c, s) for the request's slots (shared by all heads
// and both roles), and its warps then take tasks,
//   rows    one slot, up to kHeadsPerTask heads: half a warp per row, eight elements (16 bytes) a lane, the partner
//           element eight lanes' worth away comes by shuffle; the lane's (c, s) stay in registers over the heads
//   blocks  (8-bit pools) one head's K or V rows of one scale block: largest magnitude first, then the scale, the
//           re-encoding of older rows if the scale has grown, and the new rows (read again, from L1)
// and the request's tasks are dealt over several thread blocks when there are few requests.
#include <cuda_bf16.h>
#include <math.h>
#include "war_common.cuh"
#include "war_quant.cuh"

namespace {

constexpr int kMaxSlots = 64;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kHeadsPerTask = 8;
constexpr int kTargetBlocks = 148 * 6;        // thread blocks that keep a B200 busy with rows

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
};

struct Row { float x[8]; };

__device__ __forceinline__ Row widen(const uint4 u) {
    Row r;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.x[2 * i] = __uint_as_float(w[i] << 16); r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    return r;
}
__device__ __forceinline__ uint4 narrow(const Row& r) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(r.x[2 * i], r.x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// This lane's eight (c, s): elements 8 * sub .. 8 * sub + 7 of a head.  Elements that do not rotate get (1, 0).
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn load_turn(const float2* table, int sub, int half, int interleaved) {
    Turn t;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = sub * 8 + i;
        const int pair = interleaved ? e >> 1 : (e < half ? e : e - half);
        float2 cs = make_float2(1.f, 0.f);
        if (e < 2 * half) cs = table[pair];
        const bool first = interleaved ? !(e & 1) : e < half;
        t.c[i] = cs.x;
        t.s[i] = first ? -cs.y : cs.y;
    }
    return t;
}

// Rotates a row held by 16 lanes, eight elements each; `scratch`: 128 floats of this half-warp, used only when the
// partner of an element does not sit at the same place of another lane.  All 32 lanes call it together.
__device__ __forceinline__ void rotate(Row& r, const Turn& t, int sub, int lane, int half, int interleaved, float* scratch) {
    Row p;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p.x[i] = r.x[i ^ 1];
    } else if ((half & 7) == 0) {
        const int off = half >> 3;                                        // lanes between a pair's two elements
        const int src = (lane & 16) | ((sub < off ? sub + off : sub - off) & 15);
#pragma unroll
        for (int i = 0; i < 8; ++i) p.x[i] = __shfl_sync(0xffffffffu, r.x[i], src);
    } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) scratch[sub * 8 + i] = r.x[i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = sub * 8 + i;
            const int o = e < half ? e + half : (e < 2 * half ? e - half : e);
            p.x[i] = scratch[o];
        }
    }
    // separate roundings of the two products: the value does not depend on which of them a fused operation would keep
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __fadd_rn(__fmul_rn(r.x[i], t.c[i]), __fmul_rn(p.x[i], t.s[i]));
        r.x[i] = sub * 8 + i < 2 * half ? y : r.x[i];
    }
}

__global__ void __launch_bounds__(kThreads)
war_rope_store_kernel(const StoreArgs a, const int kv, const int parts) {
    extern __shared__ float2 s_table[];                                   // [N][half]
    __shared__ int s_depth[kMaxSlots];
    __shared__ float s_scratch[kWarps][2][128];
    const int b = blockIdx.x, part = blockIdx.y;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, sub = lane & 15, side = lane >> 4;
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
    for (int x = tid; x < n * a.half; x += kThreads) {
        const int j = x / a.half, i = x - j * a.half;
        const double turns = (double)(pl + s_depth[j]) * ((double)a.inv_freq[i] * 0.15915494309189533577);
        double s, c;
        sincospi(2.0 * (turns - rint(turns)), &s, &c);
        s_table[x] = make_float2((float)(c * (double)a.factor), (float)(s * (double)a.factor));
    }
    __syncthreads();

    const int32_t* pt = a.page_table + (size_t)b * a.max_pages;
    const int first_block = pl / a.block;
    const int blocks = kv == kKvBf16 ? 0 : (pl + n - 1) / a.block - first_block + 1;
    const int block_tasks = 2 * a.Hkv * blocks;
    const int heads = a.Hq + (kv == kKvBf16 ? 2 * a.Hkv : 0);             // heads the row tasks cover: q, then k and v of a bf16 pool
    const int chunks = (heads + kHeadsPerTask - 1) / kHeadsPerTask;
    const int tasks = block_tasks + n * chunks;
    float* scratch = s_scratch[warp][side];

    for (int task = part * kWarps + warp; task < tasks; task += parts * kWarps) {
        if (task >= block_tasks) {
            const int r = task - block_tasks, j = r / chunks, h0 = (r - j * chunks) * kHeadsPerTask;
            const Turn turn = load_turn(s_table + j * a.half, sub, a.half, a.interleaved);
            const int h1 = min(h0 + kHeadsPerTask, heads);
            uint4 in[kHeadsPerTask / 2];
#pragma unroll
            for (int u = 0; u < kHeadsPerTask / 2; ++u) {
                const int h = h0 + 2 * u + side;
                in[u] = make_uint4(0, 0, 0, 0);
                if (h < h1) {
                    const __nv_bfloat16* src = h < a.Hq ? a.q + b * a.qs[0] + j * a.qs[1] + h * a.qs[2]
                                             : h < a.Hq + a.Hkv ? a.k + b * a.ks[0] + j * a.ks[1] + (h - a.Hq) * a.ks[2]
                                                                : a.v + b * a.vs[0] + j * a.vs[1] + (h - a.Hq - a.Hkv) * a.vs[2];
                    in[u] = *reinterpret_cast<const uint4*>(src + sub * 8);
                }
            }
#pragma unroll
            for (int u = 0; u < kHeadsPerTask / 2; ++u) {
                if (h0 + 2 * u >= h1) break;                              // (uniform: both halves of the warp rotate together)
                const int h = h0 + 2 * u + side;
                Row row = widen(in[u]);
                rotate(row, turn, sub, lane, a.half, a.interleaved, scratch);
                if (h >= h1) continue;
                const uint4 out = h < a.Hq + a.Hkv ? narrow(row) : in[u];  // v is copied as it is
                if (h < a.Hq) {
                    *reinterpret_cast<uint4*>(a.q_out + (((size_t)b * a.N + j) * a.Hq + h) * 128 + sub * 8) = out;
                } else {
                    const int pos = pl + j;
                    const long long page = pt[pos / a.page_size];
                    if (page < 0 || page >= a.num_pages) {
                        if (sub == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
                        continue;
                    }
                    const bool is_k = h < a.Hq + a.Hkv;
                    const long long* st = is_k ? a.kp : a.vp;
                    const int kh = h - a.Hq - (is_k ? 0 : a.Hkv);
                    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(is_k ? a.kpool : a.vpool) + page * st[0] + kh * st[1] + (long long)(pos % a.page_size) * st[2];
                    *reinterpret_cast<uint4*>(dst + sub * 8) = out;
                }
            }
            continue;
        }
        // ---- one scale block of one head's K or V
        const int which = task & 1, h = (task >> 1) % a.Hkv, t = (task >> 1) / a.Hkv;
        const int pos0 = (first_block + t) * a.block;
        const int j0 = max(0, pos0 - pl), j1 = min(n, pos0 + a.block - pl);
        const long long page = pt[pos0 / a.page_size];
        if (page < 0 || page >= a.num_pages) {
            if (lane == 0) war_set_device_status(a.status_word, WAR_ERR_BAD_PAGE);
            continue;
        }
        const long long* ss = which ? a.vs : a.ks;
        const __nv_bfloat16* src = (which ? a.v : a.k) + b * ss[0] + h * ss[2];
        const long long* ps = which ? a.vp : a.kp;
        const int row0 = pos0 % a.page_size;
        uint8_t* dst = (which ? a.vpool : a.kpool) + page * ps[0] + h * ps[1] + (long long)row0 * ps[2];
        float* scale = (which ? a.vscale : a.kscale) + (page * a.Hkv + h) * a.blocks_per_page + row0 / a.block;
        const int old = min(max(pl - pos0, 0), a.block);                  // rows of earlier tokens in the block
        const float s_old = old > 0 ? *scale : 0.f;
        auto fetch = [&](int j) -> Row {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (j < j1) u = *reinterpret_cast<const uint4*>(src + j * ss[1] + sub * 8);
            Row r = widen(u);
            if (!which) rotate(r, load_turn(s_table + min(j, j1 - 1) * a.half, sub, a.half, a.interleaved), sub, lane, a.half, a.interleaved, scratch);
            return r;
        };
        float top = 0.f;
        for (int j = j0; j < j1; j += 2) {
            const Row r = fetch(j + side);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(r.x[i]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float s_new = fmaxf(s_old, quant::pow2_scale(top, kv));
        if (!(s_new > 0.f)) s_new = 1.f;
        if (s_new != s_old && old > 0) {
            const float ratio = s_old / s_new;
            for (int r = side; r < old; r += 2) {
                uint2* p = reinterpret_cast<uint2*>(dst + r * ps[2]) + sub;
                *p = quant::recode8(*p, ratio, kv);
            }
        }
        for (int j = j0; j < j1; j += 2) {
            const Row r = fetch(j + side);
            if (j + side >= j1) continue;
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = quant::encode2(r.x[4 * i] / s_new, r.x[4 * i + 1] / s_new, kv) |
                       (quant::encode2(r.x[4 * i + 2] / s_new, r.x[4 * i + 3] / s_new, kv) << 16);
            reinterpret_cast<uint2*>(dst + (long long)(pl + j + side - pos0) * ps[2])[sub] = make_uint2(w[0], w[1]);
        }
        if (lane == 0 && s_new != s_old) *scale = s_new;
    }
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
    // how many thread blocks share a request: enough to fill the GPU, no more than there are tasks
    const long long heads = p->Hq + (p->kv_type == kKvBf16 ? 2ll * p->Hkv : 0);
    const long long tasks = (p->kv_type == kKvBf16 ? 0 : 2ll * p->Hkv * ((p->N + a.block - 2) / a.block + 1)) +
                            (long long)p->N * ((heads + kHeadsPerTask - 1) / kHeadsPerTask);
    long long parts = (kTargetBlocks + p->B - 1) / p->B;
    if (parts > (tasks + kWarps - 1) / kWarps) parts = (tasks + kWarps - 1) / kWarps;
    if (parts < 1) parts = 1;
    const size_t table = sizeof(float2) * (size_t)p->N * (size_t)(a.half > 0 ? a.half : 1);
    war_rope_store_kernel<<<dim3(p->B, (unsigned)parts), kThreads, table, stream>>>(a, p->kv_type, (int)parts);
    WAR_LAUNCH_CHECK();
    return WAR_OK;
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
