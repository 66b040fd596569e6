// Norm and rotation of queries and keys, the paged cache in 8 bits or bf16, attention of drafted tokens over
// it: what the launches take.  Pointers are device pointers unless they say otherwise.
#pragma once
#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime_api.h>

#include "kernels.h"

namespace pk {

constexpr int kMostPairs = 128;                     // rotated pairs of a row
constexpr int kMostDrafts = 64;                     // drafted tokens of a request: bits of its mask words

struct RowsView {                                   // [token][head][d], strides in elements, columns contiguous
    void* data; int64_t token_stride, head_stride;
};

// The cache: K [blocks][Hkv][page][d], V [blocks][Hkv][page / 4][d][4], scales [blocks][Hkv][2][page] (K, V)
struct CacheView {
    void* k; void* v; uint8_t* scales;
    int64_t num_blocks; int page, Hkv, d, f8;
};

struct TokenRowsArgs {
    RowsView q, k, v, q_out, k_out;                 // no k_out: K and V go into the cache
    const void* q_weight; const void* k_weight;     // null: no norm
    float eps;
    const float* table; const int32_t* positions;   // [max_pos][2][pairs]; [axes][tokens]
    int64_t axis_stride; int32_t max_pos; int pairs; int interleaved;
    uint8_t pair_axis[kMostPairs];
    CacheView cache; const int64_t* slots;
    int64_t tokens; int Hq, Hkv, d;
    int in_f32, out_f32;
    // set by the launch
    int splits, axes_by_four; FastDiv by_splits; double by_d;       // waves that share a token's heads; whether four pairs in a row have one axis
};
int launch_token_rows(TokenRowsArgs a, void* stream);

struct CacheReadArgs {
    CacheView cache; const int32_t* block_table; int32_t max_blocks;
    const int32_t* kv_lens; const int32_t* row_start; int32_t n;
    RowsView k_out, v_out; int64_t rows; int out_f32;
    int splits; FastDiv by_splits;                  // set by the launch: workgroups that share the heads of 64 tokens
};
int launch_cache_read(CacheReadArgs a, void* stream);

struct CacheKeepArgs {
    CacheView cache; const int32_t* block_table; int32_t max_blocks;
    const int32_t* kv_lens; const int32_t* q_start; int32_t n;
    const int32_t* keep; int32_t max_keep; const int32_t* keep_count; int32_t* new_lens;
    FastDiv by_page;
};
int launch_cache_keep(CacheKeepArgs a, void* stream);

// How a launch takes the rows of a (request, KV head): `chunks` workgroups of up to `rows` of them for every piece of the request's keys; `items` workgroups of a
// KV head run at once; of more requests than that a piece has at most 4 / rounds of what a workgroup's place gets to do.
struct TreeShape {
    int rows, chunks, items, rounds, alone_chunks;  // alone_chunks: chunks of 32 rows (16 with no more), where a wave has a request
    // both grow with n and max_q, so that a workspace serves every call of one head shape that is not larger than what it was made for
    size_t count_bytes(int64_t n, int Hkv) const { return static_cast<size_t>((n * Hkv * chunks * 4 + 255) / 256 * 256 + (n * 8 + 255) / 256 * 256); }
    size_t partial_bytes(int Hkv, int d, int compute_units) const;
    static TreeShape of(int max_q, int Hq, int Hkv, int compute_units);
};

struct TreeArgs {
    CacheView cache; const int32_t* block_table; int32_t max_blocks;
    const void* q; const int32_t* q_start; int64_t total_q; int32_t max_q;
    const uint64_t* mask;                           // [total_q]; null: every drafted token sees those before it and itself
    const int32_t* kv_lens; int32_t n;
    void* out; int out_f32; float scale; int Hq;
    uint32_t* arrived;                              // [n][Hkv][chunks], zero between launches (arrival.h)
    int2* pieces_of;                                // [n] pieces of a request and slot of the first one, for the merge in a launch of its own
    float* part_lse; float* part_o;                 // [slots][Hkv][rows], [..][d]
    // set by the launch
    int heads_per_kv, subs, most_keys, chunk_shift, chunks, items, slices, whole;  // subs: sub-tiles of 16 keys in a page; chunk_shift: rows of a chunk, log2
    float rounds, least_per_share, least_per_many;
    FastDiv by_hkv, by_chunks;
    FastDiv by_r, by_subs;
};
int launch_tree_attn(TreeArgs a, const TreeShape& s, void* stream);

}  // namespace pk
