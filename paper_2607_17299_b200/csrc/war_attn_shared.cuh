// Attention over requests that share the pages of a prefix: what the planning kernel (war_verify_attn_shared.cu) leaves in
// the workspace for the attention kernels and for the merge (library-internal).
//
// A part is what one pass over keys serves: the prefix that the members of a group share (rows of all members, every key
// visible to all) or what a request has for itself (its rows; keys behind the shared ones, its tree among them).  Parts are cut into
// units as in war_attn_plan.cuh: (part, kv head, row block, chunk of 128-key tiles).  Rows of a shared part are the (slot, query head
// of the group) pairs of its members one behind the other, so that row blocks are full whatever the trees' sizes are.  A row block has
// 256 rows, and 128 with the 8-bit kernel up to kQuantWideRows.
#pragma once
#include <cuda_runtime.h>
#include "war_attn_plan.cuh"
#include "war_attn_quant.cuh"

// A unit's partial result: (max, sum) of row r at part_ml[part0 + r], and O in pieces of four columns, piece c of row r at
// part_o[(part0 * 32 + c * part_rows + r) * 4]: a warp that holds a row a lane stores 512 bytes in a row.
struct alignas(16) SharedPart {
    int part0, n_chunks, rows, slot0;    // partial results of (chunk, kv head) begin at part0 + (chunk * Hkv + kv head) * rows;
                                         // slot0: a shared part's first entry in slot_map, -1: the request's own part
    int each, more, whole, req;          // the first `more` chunks have each + 1 tiles, the others `each`; whole: nothing else serves these
                                         // rows, the result is written; the page table's row that is read,
    int page0, n_keys, visible, pad;     // the part's first page in it, its keys, the first of them that every row sees (the tree's mask
                                         // decides for the others)
};
struct SharedReq { int n, group, row0, pad; };                       // group: number of the shared part (-1: none), row0: the request's first row there
struct SharedUnit {
    SharedPart part;
    int kvh, tile_begin, tile_end;
    int row0, rows;                      // the unit's rows of the part
    int part0;                           // partial results of its (chunk, kv head)
};

struct SharedWorkspace {
    int* counters;                  // [0] units handed out behind the first of every CTA, [1] number of units
    int* slot_map;                  // [B * N] request * N + slot, group by group
    uint2* units;                   // part | chunk << 16, kv head | row block << 16
    SharedPart* parts;              // [B + B / 2] the requests' own parts, then the shared ones
    SharedReq* reqs;                // [B]
    float* part_ml;                 // [rows, 2]
    float* part_o;                  // [rows, D]
    long long max_units, max_rows;
    size_t bytes;
};

constexpr int kSharedBlock = 256, kSharedQuantBlock = 128;           // rows of a row block
inline SharedWorkspace war_attn_shared_layout(const war_attn_params_t* p, void* base) {
    SharedWorkspace w;
    const long long G = p->Hq / p->Hkv, B = p->B, R = G * p->N;
    const long long own_blocks = (R + kRowBlock - 1) / kRowBlock, group_blocks = (B * R + kRowBlock - 1) / kRowBlock + B / 2;
    // chunks of at least 1 / kTargetUnits of all work: no more than kTargetUnits units above one for every (part, kv head, row block),
    // and a unit has no more rows than a block
    w.max_units = kTargetUnits + p->Hkv * (B * own_blocks + group_blocks);
    w.max_rows = (long long)kTargetUnits * kSharedBlock + 2 * B * R * p->Hkv;
    auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
    size_t at = 0;
    char* b = (char*)base;
    auto take = [&](size_t bytes) { void* q = b + at; at += align(bytes); return q; };
    w.counters = (int*)take(64 * sizeof(int));
    w.slot_map = (int*)take(sizeof(int) * (size_t)(B * p->N));
    w.units = (uint2*)take(sizeof(uint2) * (size_t)w.max_units);
    w.parts = (SharedPart*)take(sizeof(SharedPart) * (size_t)(B + B / 2));
    w.reqs = (SharedReq*)take(sizeof(SharedReq) * (size_t)B);
    w.part_ml = (float*)take(sizeof(float) * 2 * (size_t)w.max_rows);
    w.part_o = (float*)take(sizeof(float) * 128 * (size_t)w.max_rows);
    w.bytes = at;
    return w;
}

// The attention kernels on such a plan: war_verify_attn_shared_sm100.cu; war_verify_attn_quant_many.cu up to kQuantWideRows query rows per request
// and kv head, above war_verify_attn_shared_quant_sm100.cu.  The latter has twice the rows in a unit, the former more of a cache in flight where
// memory is the bound, the requests' own keys.  In turn on one GPU (us, former / latter): 4 rows, 4K to 8K own keys 504 / 645; 32 rows
// 16 prompts of 4 338 / 347, one of 16 264 / 240; 64 rows, 8K own keys 257 / 290, 4 prompts of 4 with 32K 271 / 236; 68 and 80 rows, 8K own keys
// 300 / 308, 304 / 312, with 4 rollouts of 12K shared 376 / 366; 128 rows 331 / 329, 721 / 637, 517 / 460; 256 rows 562 / 495, 680 / 588.  The rule sees a
// request's rows, which the host knows, and not the lengths, which it does not: with shared keys alone the latter can be ahead at 32 and 64 rows
// (264 / 240, 271 / 236), with long own keys the former still at 68 and 80 (300 / 308, 304 / 312).
constexpr int kQuantWideRows = 64;
war_status_t war_attn_shared_launch(const void* q, const void* k, const void* v, const int32_t* page_table, const int32_t* parent,
                                    const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                    int* status_word, cudaStream_t s);
war_status_t war_attn_quant_launch_shared(const void* q, const AttnQuantPools& pools, const int32_t* page_table, const int32_t* parent,
                                          const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                          int* status_word, cudaStream_t s);
war_status_t war_attn_quant_launch_shared_wide(const void* q, const AttnQuantPools& pools, const int32_t* page_table, const int32_t* parent,
                                          const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                          int* status_word, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ SharedUnit shared_unit(const uint2* units, const SharedPart* parts, int u, int Hkv, int block) {
    SharedUnit x;
    const uint2 at = units[u];
    x.part = parts[at.x & 0xffffu];
    const int c = (int)(at.x >> 16);
    x.kvh = (int)(at.y & 0xffffu);
    x.row0 = (int)(at.y >> 16) * block; x.rows = min(block, x.part.rows - x.row0);
    x.tile_begin = c * x.part.each + min(c, x.part.more); x.tile_end = x.tile_begin + x.part.each + (c < x.part.more ? 1 : 0);
    x.part0 = x.part.part0 + (c * Hkv + x.kvh) * x.part.rows;
    return x;
}

// The loads of a unit of T tiles are K0, K1, V0, K2, V1, ..., K(T-1), V(T-2), V(T-1); ld0: loads before the unit.
__device__ __forceinline__ uint32_t load_k(uint32_t ld0, int t) { return t == 0 ? ld0 : ld0 + 2u * t - 1u; }
__device__ __forceinline__ uint32_t load_v(uint32_t ld0, int t, int T) { return t == T - 1 ? ld0 + 2u * T - 1u : ld0 + 2u * t + 2u; }

// a number twice, as a packed pair; the sum of four packed pairs
__device__ __forceinline__ uint64_t pair_of(float x) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float sum_of(uint64_t s0, uint64_t s1, uint64_t s2, uint64_t s3) {
    float r;
    asm("{\n.reg .f32 a, b;\nadd.rn.f32x2 %1, %1, %2;\nadd.rn.f32x2 %3, %3, %4;\nadd.rn.f32x2 %1, %1, %3;\nmov.b64 {a, b}, %1;\nadd.rn.f32 %0, a, b;\n}\n"
        : "=f"(r), "+l"(s0), "+l"(s1), "+l"(s2), "+l"(s3));
    return r;
}
#endif
