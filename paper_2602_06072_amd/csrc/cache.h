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
    int64_t rows_of_slots(int Hkv, int compute_units) const { return slots(rounds, Hkv, compute_units) * rows; }
    size_t partial_bytes(int Hkv, int d, int compute_units) const { return whole256(rows_of_slots(Hkv, compute_units) * (d + 1) * 4); }
    // Counts of arrivals, one for every slot where up to 16 rows are joined in the launch.  They come first in a workspace, and how many there are depends
    // neither on n nor on max_q: no call, whatever the others were, has its counts where another one has written something else.
    static size_t count_bytes(int Hkv, int compute_units) { return whole256(slots(kRoundsOfFewRows, Hkv, compute_units) * 4); }
    static size_t pieces_bytes(int64_t n) { return whole256(n * 8); }
    static TreeShape of(int max_q, int Hq, int Hkv, int compute_units);

    static constexpr int kRoundsOfFewRows = 8;      // (of up to 32 rows)

private:
    // Pieces of cut requests, all KV heads together.  A piece has at least 4 / (items * rounds) of all tiles, and only requests of more than that are cut:
    // twice as many slots hold the pieces of all.
    static int64_t slots(int rounds, int Hkv, int compute_units) {
        const int64_t most = Hkv > 2 * compute_units ? Hkv : 2 * compute_units;
        return (rounds + 1) / 2 * most + 64;
    }
    static size_t whole256(int64_t bytes) { return static_cast<size_t>((bytes + 255) / 256 * 256); }
};

struct TreeArgs {
    CacheView cache; const int32_t* block_table; int32_t max_blocks;
    const void* q; const int32_t* q_start; int64_t total_q; int32_t max_q;
    const uint64_t* mask;                           // [total_q]; null: every drafted token sees those before it and itself
    const int32_t* kv_lens; int32_t n;
    void* out; int out_f32; float scale; int Hq;
    uint32_t* arrived;                              // [slots][Hkv], a request's at its first slot; zero between launches (arrival.h)
    int2* pieces_of;                                // [n] pieces of a request and slot of the first one, for the merge in a launch of its own
    float* part_lse; float* part_o;                 // [slots][Hkv][rows], [..][d]
    // set by the launch
    int heads_per_kv, subs, most_keys, chunk_shift, chunks, items, slices, whole;  // subs: sub-tiles of 16 keys in a page; chunk_shift: rows of a chunk, log2
    float rounds, least_per_share, least_per_many;
    FastDiv by_hkv, by_chunks;
    FastDiv by_r, by_subs;
    // where requests share pages: tokens that a request shares with its family (a multiple of 64; [n]), and a family's first request ([families])
    const int32_t* shared_of; const int32_t* first_of;
    const int32_t* places;                          // instead of `items`, for shared keys
};
int launch_tree_attn(TreeArgs a, const TreeShape& s, void* stream);

}  // namespace pk
