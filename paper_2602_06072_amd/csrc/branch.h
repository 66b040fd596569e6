// Pages of the paged cache (forking, reserving, compacting, copying) and the judging of drafted tokens: what the launches take.
// Pointers are device pointers.
#pragma once
#include <cstddef>
#include <cstdint>

#include "cache.h"

namespace pk {

struct PagesSelectArgs {
    const int32_t* table; const int32_t* lens; const int32_t* pages; int32_t n; int32_t max_blocks;
    const int32_t* from; int32_t n_new; int32_t* new_table; int32_t* new_lens; int32_t* new_pages;
    int32_t* refs; int32_t num_blocks; int32_t page;
};
int launch_pages_select(const PagesSelectArgs& a, void* stream);

// A workspace of the page calls: for every 1024 blocks three times 1024 words and a cache line's worth for one more.  The first two thousand are zero between calls, and which words these are
// does not depend on num_blocks: no call has its zeros where one for a smaller pool has written something else.
struct PagesWorkspace {
    static constexpr int kSegment = 1024;           // blocks that a workgroup looks at
    static constexpr int kWriters = kSegment, kNumbers = 2 * kSegment, kUsed = 3 * kSegment, kWords = kUsed + 64;     // (whole cache lines)
    static size_t bytes(const int64_t num_blocks) { return static_cast<size_t>((num_blocks + kSegment - 1) / kSegment) * kWords * 4; }
    // of block b's words the first
    static constexpr int64_t at(const uint32_t b) { return static_cast<int64_t>(b / kSegment) * kWords + b % kSegment; }
};

struct PagesReserveArgs {
    int32_t* table; const int32_t* lens; int32_t* pages; int32_t n; int32_t max_blocks;
    const int32_t* grow; int32_t* refs; int32_t num_blocks; int32_t page;
    int32_t* served; int32_t* copy_src; int32_t* copy_dst;
    // at PagesWorkspace::at of a block; zero between calls: number + 1 of the last request that would write it though it is shared; how many would
    int32_t* last_writer; int32_t* writers;
    int32_t* free;                                  // (the same) the free blocks that are handed out, by rising number
};
int launch_pages_reserve(const PagesReserveArgs& a, void* stream);

struct PagesCompactArgs {
    const int32_t* table; const int32_t* pages; int32_t n; int32_t max_blocks;
    const int32_t* refs; int32_t num_blocks; int32_t* new_table; int32_t* new_refs;
    int32_t* copy_src; int32_t* copy_dst; int32_t max_moves;
    int32_t* to;                                    // at PagesWorkspace::at: new number of every block; -1 - k: that of move k
    int32_t* used_of;                               // blocks in use of every segment, kWords apart
};
int launch_pages_compact(const PagesCompactArgs& a, void* stream);

struct CacheCopyArgs {
    CacheView from, to; const int32_t* src; const int32_t* dst; int32_t count;
    int parts;                                      // set by the launch: waves that share a block's keys, and its values
};
int launch_cache_copy(CacheCopyArgs a, void* stream);

// Sum of the weights of a piece of a row of logits, relative to that of the logit `top`; or the largest logit and where it stands first
struct RowPart { double sum; float top; int32_t at; };

// What a token with children decides: which of them stays (-1: none), c, and 1 / the sums of its rows with what they are relative to.  Until then: workgroups that are done
// (zero from the launch in front), and what each of them has of the first sum of what is left.
struct VerifyChoice {
    static constexpr int kMostParts = 8;
    int32_t token;
    double c, of_target, of_draft;
    float top, draft_top;
    uint32_t arrived;
    double left[kMostParts];
};

// How a launch cuts rows of logits: `pieces` of a row where all rows with children are looked at; where one of each request is, `spans`, each of span_rounds times 1024 elements,
// for `groups` workgroups, group_spans for each
struct VerifyShape {
    int pieces, length;                             // length in elements, a multiple of kStep
    int spans, span_rounds, groups, group_spans, last_stride;
    static constexpr int kStep = 4096;              // elements that a workgroup takes at a time
    static constexpr int kRows = 2048, kMostPieces = 64;           // pieces of all rows together, about; of a row (the lanes that put them together)
    static constexpr int kSpan = 1024, kMostSpans = 256;           // elements of a round of a span; spans (the threads that put them together)
    static constexpr size_t kCountBytes = 65536 * 4;               // arrivals of a request's pieces, zero between calls: in front of everything, as many for every call
    static VerifyShape of(int64_t n, int64_t total_q, int32_t vocab);
    // Room for as much as any call of up to so many tokens, requests and logits takes, so that a workspace of the largest batch serves all smaller ones: `pieces` and
    // `last_stride` fall where a row is cut into fewer, longer parts.  Rows have up to 2048 / total_q + 1 pieces, of a step and more, and up to 64; last_stride is up to 256
    // spans of 1024 logits.
    static size_t part_bytes(const int64_t total_q, const int32_t vocab) {
        const int64_t steps = (vocab + kStep - 1) / kStep, each = total_q * (steps < kMostPieces ? steps : kMostPieces), all = kRows + total_q;
        return whole256(2 * (each < all ? each : all) * static_cast<int64_t>(sizeof(RowPart)));
    }
    static size_t last_bytes(const int64_t n, const int32_t vocab) {
        const int64_t spans = (vocab + kSpan - 1) / kSpan;
        return whole256(n * (spans < 2 ? 2 : spans < kMostSpans ? spans : kMostSpans) * static_cast<int64_t>(sizeof(RowPart)));
    }
    static size_t choice_bytes(const int64_t total_q) { return whole256(total_q * static_cast<int64_t>(sizeof(VerifyChoice))); }
    static size_t bytes(const int64_t n, const int64_t total_q, const int32_t vocab) {
        return kCountBytes + part_bytes(total_q, vocab) + last_bytes(n, vocab) + choice_bytes(total_q);
    }

private:
    static size_t whole256(const int64_t bytes) { return static_cast<size_t>((bytes + 255) / 256 * 256); }
};

struct VerifyArgs {
    const void* target; int64_t target_stride; const void* draft; int64_t draft_stride; int f32; int32_t vocab;
    const int32_t* tokens; const int32_t* q_start; int64_t total_q; int32_t max_q; const uint64_t* mask; int32_t n;
    const float* temperature; const float* accept_u; const float* sample_u;
    int32_t* keep; int32_t max_keep; int32_t* keep_count; int32_t* next_token;
    VerifyShape shape;
    uint32_t* arrived;                              // [n], zero between calls
    RowPart* parts;                                 // [total_q][2][pieces]: of the target's rows, of the draft's
    RowPart* last_parts;                            // [n][last_stride]
    VerifyChoice* choices;                          // [total_q]
    int choice_parts;                               // set by the launch: workgroups that share the first sum of what is left
};
int launch_draft_verify(const VerifyArgs& a, void* stream);

}  // namespace pk
