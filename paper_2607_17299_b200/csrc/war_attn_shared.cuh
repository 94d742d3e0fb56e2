// Attention over requests that share the pages of a prefix: what the planning kernel (war_verify_attn_shared.cu) leaves in
// the workspace for the attention kernels and for the merge (library-internal).
//
// A part is what one pass over keys serves: the prefix that the members of a group share (rows of all members, every key
// visible to all) or what a request has for itself (its rows; keys behind the shared ones, its tree among them).  Parts are cut into
// units as in war_attn_plan.cuh: (part, kv head, row block, chunk of 128-key tiles).  Rows of a shared part are the (slot, query head
// of the group) pairs of its members one behind the other, so that row blocks are full whatever the trees' sizes are.
#pragma once
#include "war_attn_plan.cuh"
#include "war_attn_quant.cuh"

struct SharedUnit {
    int req, page0;                 // the page table's row that is read, and the part's first page in it
    int kvh, rb, tile_begin, tile_end;
    int n_keys;                     // keys of the part
    int visible;                    // the first keys, that every row sees; behind them the tree's mask decides
    int rows;                       // rows of the part
    int slot0;                      // shared part: its first entry in slot_map; -1: the request's own part
    int part0;                      // where the unit's first row goes in the partial results
    int whole;                      // 1: nothing else serves these rows, the result is written
};
struct SharedPart { int part0, n_chunks, rows, n_tiles; };           // partial of (chunk, kv head, row): part0 + (chunk * Hkv + kv head) * rows + row
struct SharedReq { int n, group, row0, pad; };                       // group: number of the shared part (-1: none), row0: the request's first row there

struct SharedWorkspace {
    int* counters;                  // [1] number of units
    uint64_t* anc;                  // [B, N]
    int* slot_map;                  // [B * N] request * N + slot, group by group
    SharedUnit* units;
    SharedPart* parts;              // [B + B / 2] the requests' own parts, then the shared ones
    SharedReq* reqs;                // [B]
    float* part_ml;                 // [rows, 2]
    float* part_o;                  // [rows, D]
    long long max_units, max_rows;
    size_t bytes;
};

inline SharedWorkspace war_attn_shared_layout(const war_attn_params_t* p, void* base) {
    SharedWorkspace w;
    const long long G = p->Hq / p->Hkv, B = p->B, R = G * p->N;
    const long long own_blocks = (R + kRowBlock - 1) / kRowBlock, group_blocks = (B * R + kRowBlock - 1) / kRowBlock + B / 2;
    // chunks of at least total / kTargetUnits tiles: no more than kTargetUnits units above one for every (part, kv head, row block),
    // and a unit has no more rows than a block, nor a request's own unit than its trees
    w.max_units = kTargetUnits + p->Hkv * (B * own_blocks + group_blocks);
    w.max_rows = (long long)kTargetUnits * kRowBlock + 2 * B * R * p->Hkv;
    auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
    size_t at = 0;
    char* b = (char*)base;
    auto take = [&](size_t bytes) { void* q = b + at; at += align(bytes); return q; };
    w.counters = (int*)take(64 * sizeof(int));
    w.anc = (uint64_t*)take(sizeof(uint64_t) * (size_t)(B * p->N));
    w.slot_map = (int*)take(sizeof(int) * (size_t)(B * p->N));
    w.units = (SharedUnit*)take(sizeof(SharedUnit) * (size_t)w.max_units);
    w.parts = (SharedPart*)take(sizeof(SharedPart) * (size_t)(B + B / 2));
    w.reqs = (SharedReq*)take(sizeof(SharedReq) * (size_t)B);
    w.part_ml = (float*)take(sizeof(float) * 2 * (size_t)w.max_rows);
    w.part_o = (float*)take(sizeof(float) * 128 * (size_t)w.max_rows);
    w.bytes = at;
    return w;
}

// The attention kernels on such a plan (war_verify_attn_sm100.cu, war_verify_attn_quant_many.cu).
war_status_t war_attn_launch_sm100_shared(const void* q, const void* k, const void* v, const int32_t* page_table,
                                          const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                          int* status_word, cudaStream_t s);
war_status_t war_attn_quant_launch_shared(const void* q, const AttnQuantPools& pools, const int32_t* page_table,
                                          const war_attn_params_t* p, const SharedWorkspace& w, void* out, float* lse,
                                          int* status_word, cudaStream_t s);
