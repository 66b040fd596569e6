// Attention of drafted tokens where requests share pages: what its launches take.
#pragma once
#include "cache.h"

namespace pk {

struct SharedArgs {
    TreeArgs tree;                                  // as for pk_tree_attn; partial results of the requests' own keys
    const int32_t* family_start; int32_t families;
    uint32_t* arrived; int32_t* missing;            // zero between calls: workgroups that are done; [families] 1 + the keys of a table that a family does not share, 0: it has no rows
    int32_t* family_of; int32_t* shared_of;         // [n]
    int32_t* first_of; int32_t* q_start_of; int32_t* len_of;       // [families (+ 1)]: first request, rows of q, shared tokens
    int32_t* places;                                // [1] workgroups of a KV head that the shared keys are cut for
    int few_rows, at_once;                          // set by the launch: up to 32 rows a request; workgroups of a KV head that run at once
    int2* pieces_of_family; float* family_lse; float* family_o;    // partial results of the shared keys
};
int launch_shared_tree_attn(SharedArgs s, const TreeShape& shape, void* stream);

// Where things are in a workspace.  What has to be zero between calls comes first, at places that depend on Hkv alone.
struct SharedWorkspace {
    static constexpr int64_t kMostFamilies = 65536;
    int64_t own_slots, family_slots;                // of a KV head
    size_t counts, plain, arrays, own, family, bytes;              // begin of: arrivals of pk_tree_attn's pieces; its other parts, or the arrays and both parts here

    static SharedWorkspace of(const int64_t n, const int64_t total_q, const TreeShape& s, const int Hq, const int Hkv, const int d, const int compute_units) {
        SharedWorkspace w;
        const int64_t row = 4 * (d + 1);
        // (share_of in tree_body.hip.h: no more pieces than chunks and twice what runs at once, and some for the rounding of its sums)
        w.own_slots = n * s.chunks + 4 * 2 * s.items + 64;            // (four waves of a workgroup with pieces of their own)
        w.family_slots = total_q * (Hq / Hkv) / 128 + n / 2 + 1 + 3 * s.items + 64;
        w.counts = 256 + kMostFamilies * 4;
        w.plain = w.counts + TreeShape::count_bytes(Hkv, compute_units);
        w.arrays = w.plain;
        w.own = w.arrays + whole256(4 * (5 * n + 16) + 16 * n);
        w.family = w.own + whole256(w.own_slots * Hkv * s.rows * row);
        const size_t here = w.family + whole256(w.family_slots * Hkv * 128 * row);
        const size_t there = w.plain + s.partial_bytes(Hkv, d, compute_units) + TreeShape::pieces_bytes(n);
        w.bytes = here > there ? here : there;
        return w;
    }
    static size_t whole256(const int64_t bytes) { return static_cast<size_t>((bytes + 255) / 256 * 256); }
};

}  // namespace pk
