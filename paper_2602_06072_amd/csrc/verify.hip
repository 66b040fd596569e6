// Judging of drafted tokens: which of them stay, and the token behind them.
//
// With target P and draft Q of the last token that stays, its k-th child x stays if P(x) > (c + u Z) Q(x).  That is the usual rule of rejection sampling, r(x) / Q(x) >
// u with the residual r = max(P - c Q, 0) / Z: each refusal takes r to max(r - Q, 0) over its sum, and max(max(P - c Q, 0) / Z - Q, 0) = max(P - (c + Z) Q, 0) / Z, so
// that a node's whole state is two numbers.
//
// A row of V logits is read once for its maximum and sum; rows without children (and the draft of tokens without children) are not read for that.  The row that the
// next token is drawn from is read once more, in pieces, and a piece of it a third time.  Probabilities and their sums have 64 bits: a draw is the place of a number
// between V borders, and with sums of 32 bits every tenth draw of a flat row of 100000 would fall on the other side of one.  (Vector instructions of 64 bits run
// at the rate of those of 32 here.)
#include "branch.h"
#include "common.hip.h"

namespace pk {
namespace {

constexpr int kThreads = 256, kVector = 8, kStep = VerifyShape::kStep;
static_assert(kStep == kThreads * kVector, "a step is a vector of every thread");
constexpr float kMostLogit = 3.402823466e38f;

// Eight logits from number `at` on; those behind the row's end are -inf, NaN is -inf, inf the largest number.  Rows of odd length begin anywhere: the loads
// are 16 bytes long at addresses of any alignment.
template <bool F32>
__device__ __forceinline__ void load_logits(const void* base, const int64_t row_at, const int at, const int vocab, float (&x)[kVector]) {
    if (at + kVector <= vocab) {
        if constexpr (F32) {
            __builtin_memcpy(x, static_cast<const float*>(base) + row_at + at, 32);
        } else {
            uint32_t w[4];
            __builtin_memcpy(w, static_cast<const uint16_t*>(base) + row_at + at, 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[e] << 16);
                x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            x[e] = -INFINITY;
            if (at + e < vocab) x[e] = F32 ? static_cast<const float*>(base)[row_at + at + e] : bf16_bits_to_float(static_cast<const uint16_t*>(base)[row_at + at + e]);
        }
    }
#pragma unroll
    for (int e = 0; e < kVector; ++e) x[e] = fminf(fmaxf(x[e], -INFINITY), kMostLogit);
}
template <bool F32>
__device__ __forceinline__ float load_logit(const void* base, const int64_t at) {
    const float x = F32 ? static_cast<const float*>(base)[at] : bf16_bits_to_float(static_cast<const uint16_t*>(base)[at]);
    return fminf(fmaxf(x, -INFINITY), kMostLogit);
}

// 2^y for y <= 0: y = n + f, |f| <= 1/2, and the series of exp(f ln 2) up to the 11th power (6e-15 of its value behind it).  0 for -inf.
__device__ __forceinline__ double exp2_of(const double y) {
    const double n = rint(y), f = y - n;
    constexpr double L = 0.69314718055994530942;
    constexpr double C2 = L * L / 2, C3 = C2 * L / 3, C4 = C3 * L / 4, C5 = C4 * L / 5, C6 = C5 * L / 6, C7 = C6 * L / 7, C8 = C7 * L / 8, C9 = C8 * L / 9,
                     C10 = C9 * L / 10, C11 = C10 * L / 11;
    double p = C11;
    p = fma(p, f, C10); p = fma(p, f, C9); p = fma(p, f, C8); p = fma(p, f, C7); p = fma(p, f, C6); p = fma(p, f, C5);
    p = fma(p, f, C4); p = fma(p, f, C3); p = fma(p, f, C2); p = fma(p, f, L); p = fma(p, f, 1.0);
    return y < -1100.0 ? 0.0 : ldexp(p, static_cast<int>(n));
}
// weight of a logit against the largest one; per: log2 e / temperature
__device__ __forceinline__ double weight_of(const float x, const float top, const double per) {
    return x == -INFINITY ? 0.0 : exp2_of((static_cast<double>(x) - static_cast<double>(top)) * per);
}
constexpr double kLog2eWide = 1.4426950408889634074;

// Temperature of a request; 0: the largest logit is taken
__device__ __forceinline__ float temperature_of(const VerifyArgs& a, const int i) {
    const float t = a.temperature ? a.temperature[i] : 1.f;
    return t > 0.f ? t : 0.f;
}

// Two parts of a row as one.  Of equal largest logits the first one's place.
__device__ __forceinline__ RowPart joined(const RowPart& x, const RowPart& y, const double per) {
    RowPart z;
    z.top = fmaxf(x.top, y.top);
    z.at = x.top > y.top || (x.top == y.top && x.at < y.at) ? x.at : y.at;
    z.sum = (x.sum > 0 ? x.sum * weight_of(x.top, z.top, per) : 0.0) + (y.sum > 0 ? y.sum * weight_of(y.top, z.top, per) : 0.0);
    return z;
}
__device__ __forceinline__ RowPart of_lane(const RowPart& x, const int mask) { return {__shfl_xor(x.sum, mask, 64), __shfl_xor(x.top, mask, 64), __shfl_xor(x.at, mask, 64)}; }

// Whether a row's tokens have children, and where a request's tokens are: a lane has a token
struct Tree {
    int64_t q0;
    int tokens, parent;                             // parent of this lane's token, -1: none
    uint64_t inner;                                 // tokens with children
};
__device__ __forceinline__ Tree tree_of(const VerifyArgs& a, const int i) {
    Tree t;
    const int lane = threadIdx.x & 63, q0 = a.q_start[i], q1 = a.q_start[i + 1];
    t.q0 = min(max(static_cast<int64_t>(q0), int64_t{0}), a.total_q);
    t.tokens = static_cast<int>(max(min(min(static_cast<int64_t>(q1), a.total_q) - t.q0, static_cast<int64_t>(a.max_q)), int64_t{0}));
    uint64_t before = 0;                            // ancestors
    if (lane < t.tokens) before = (a.mask ? a.mask[t.q0 + lane] : ~uint64_t{0}) & ((uint64_t{1} << lane) - 1);
    t.parent = before ? 63 - __builtin_clzll(before) : -1;
    uint64_t mine = t.parent >= 0 ? uint64_t{1} << t.parent : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine |= __shfl_xor(static_cast<unsigned long long>(mine), o, 64);
    t.inner = mine;
    return t;
}

// A piece of a row, all threads: elements [first, end)
template <bool F32>
__device__ __forceinline__ RowPart part_of_row(const void* base, const int64_t row_at, const int first, const int end, const int vocab, const double per, RowPart* lds) {
    RowPart y{0.0, -INFINITY, 0x7FFFFFFF};
    constexpr int AHEAD = 4;
    for (int at0 = first + static_cast<int>(threadIdx.x) * kVector; at0 < end; at0 += AHEAD * kStep) {
        float x[AHEAD][kVector];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load_logits<F32>(base, row_at, at0 + u * kStep, at0 + u * kStep < end ? vocab : 0, x[u]);
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int e = 0; e < kVector; ++e) top = fmaxf(top, x[u][e]);
        if (top > y.top) {
            if (y.sum > 0) y.sum *= weight_of(y.top, top, per);
            y.top = top;
            bool found = false;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int e = 0; e < kVector; ++e)
                    if (!found && x[u][e] == top) { y.at = at0 + u * kStep + e; found = true; }
        }
        if (top == -INFINITY) continue;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int e = 0; e < kVector; ++e) y.sum += weight_of(x[u][e], y.top, per);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) y = joined(y, of_lane(y, o), per);
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[wave] = y;
    __syncthreads();
    y = lds[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) y = joined(y, lds[w], per);
    return y;
}
__device__ __forceinline__ double sum_of_all(double x, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double y = lds[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) y += lds[w];
    return y;
}

// Statistics of the rows of tokens with children (a request's only token counts as one): a workgroup for (request, token, target or draft, piece)
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_rows_kernel(VerifyArgs a) {
    __shared__ RowPart lds[kThreads / 64];
    int64_t rest = blockIdx.x;
    const auto take = [&](const int of) { const int x = static_cast<int>(rest % of); rest /= of; return x; };
    const int piece = take(a.shape.pieces), of_draft = a.draft ? take(2) : 0, token = take(a.max_q), i = static_cast<int>(rest);
    const Tree t = tree_of(a, i);
    if (token >= t.tokens || !(t.inner >> token & 1 || (t.tokens == 1 && !of_draft))) return;
    const float warm = temperature_of(a, i);
    if (of_draft && warm == 0.f) return;
    const int64_t row = t.q0 + token;
    const int first = piece * a.shape.length, end = min(first + a.shape.length, a.vocab);
    const RowPart y = part_of_row<F32>(of_draft ? a.draft : a.target, row * (of_draft ? a.draft_stride : a.target_stride), first, end, a.vocab,
                                       warm > 0.f ? kLog2eWide / warm : 0.0, lds);
    if (threadIdx.x == 0) a.parts[(row * 2 + of_draft) * a.shape.pieces + piece] = y;
}

// What is left of a token's weight
struct LeftWeight {
    double per, c, of_target, of_draft;
    float top, draft_top;
    __device__ __forceinline__ double operator()(const float x, const float y) const {
        return max(of_target * weight_of(x, top, per) - (c > 0 ? c * of_draft * weight_of(y, draft_top, per) : 0.0), 0.0);
    }
};
// Sum over elements [first, end) of two rows
template <bool F32>
__device__ __forceinline__ double left_in(const VerifyArgs& a, const int64_t row, const int first, const int end, const LeftWeight& w, double* lds) {
    double sum = 0;
    for (int at = first + static_cast<int>(threadIdx.x) * kVector; at < end; at += kStep) {
        float x[kVector], y[kVector];
        load_logits<F32>(a.target, row * a.target_stride, at, a.vocab, x);
        load_logits<F32>(a.draft, row * a.draft_stride, at, a.vocab, y);
#pragma unroll
        for (int e = 0; e < kVector; ++e) sum += w(x[e], y[e]);
    }
    return sum_of_all(sum, lds);
}

// The walk along the drafted tokens that stay: a workgroup for a request, every wave the same (a lane has a token)
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(VerifyArgs a) {
    __shared__ double lds[kThreads / 64];
    const int i = blockIdx.x, lane = threadIdx.x & 63;
    const Tree t = tree_of(a, i);
    const float warm = temperature_of(a, i);
    const double per = warm > 0.f ? kLog2eWide / warm : 0.0;
    const bool greedy = warm == 0.f, drawn = a.draft && !greedy;
    int32_t* keep = a.keep + static_cast<int64_t>(i) * a.max_keep;
    if (t.tokens == 0) {
        for (int k = threadIdx.x; k < a.max_keep; k += kThreads) keep[k] = -1;
        if (threadIdx.x == 0) { a.keep_count[i] = 0; a.next_token[i] = -1; a.left[i].kind = kNone; }
        return;
    }
    // this lane's row: its pieces put together
    const bool known = lane < t.tokens && (t.inner >> lane & 1 || t.tokens == 1);
    RowPart p{0.0, -INFINITY, 0x7FFFFFFF}, q = p;
    for (int z = 0; z < a.shape.pieces; ++z) {
        if (known) p = joined(p, a.parts[(t.q0 + lane) * 2 * a.shape.pieces + z], per);
        if (known && drawn && t.tokens > 1) q = joined(q, a.parts[((t.q0 + lane) * 2 + 1) * a.shape.pieces + z], per);
    }
    // this lane's token: its probabilities in its parent's rows
    const int from = max(t.parent, 0), token = lane < t.tokens ? a.tokens[t.q0 + lane] : -1;
    const bool able = t.parent >= 0 && token >= 0 && token < a.vocab;
    const float u = able ? a.accept_u[t.q0 + lane] : 0.f;
    double mine_p = 0, mine_q = 0;
    {
        const float top_p = __shfl(p.top, from, 64), top_q = __shfl(q.top, from, 64);
        const double sum_p = __shfl(p.sum, from, 64), sum_q = __shfl(q.sum, from, 64);
        if (able && sum_p > 0) mine_p = weight_of(load_logit<F32>(a.target, (t.q0 + from) * a.target_stride + token), top_p, per) / sum_p;
        if (able && drawn && sum_q > 0) mine_q = weight_of(load_logit<F32>(a.draft, (t.q0 + from) * a.draft_stride + token), top_q, per) / sum_q;
    }
    int at = 0, count = 1;
    uint64_t kept = 1;
    double c = 0, Z = 1;
    bool refused = false;
    uint64_t gone = 0;                              // children of `at` that were refused
    for (int s = 1; s < t.tokens && count < a.max_keep; ++s) {
        if (__shfl(t.parent, s, 64) != at || !__shfl(static_cast<int>(able), s, 64)) continue;
        const int x = __shfl(token, s, 64);
        const double px = __shfl(mine_p, s, 64), qx = __shfl(mine_q, s, 64), us = __shfl(u, s, 64);
        const bool before = __ballot((gone >> lane & 1) && token == x) != 0;       // (the same token again)
        const bool ok = greedy ? __shfl(p.top, at, 64) > -INFINITY && __shfl(p.at, at, 64) == x : drawn ? px > (c + us * Z) * qx : !before && px > us * Z;
        if (ok) {
            at = s; kept |= uint64_t{1} << s; ++count;
            c = 0; Z = 1; refused = false; gone = 0;
            continue;
        }
        if (greedy) continue;
        refused = true;
        gone |= uint64_t{1} << s;
        if (!drawn) { Z -= before ? 0.0 : px; continue; }
        c += Z;
        // what is left is summed up only for a sibling's sake
        if (__ballot(lane > s && lane < t.tokens && t.parent == at && able) == 0) continue;
        const double sum_p = __shfl(p.sum, at, 64), sum_q = __shfl(q.sum, at, 64);
        const LeftWeight w{per, c, sum_p > 0 ? 1 / sum_p : 0.0, sum_q > 0 ? 1 / sum_q : 0.0, __shfl(p.top, at, 64), __shfl(q.top, at, 64)};
        Z = left_in<F32>(a, t.q0 + at, 0, a.vocab, w, lds);
    }
    if (threadIdx.x >= 64) return;
    for (int k = lane; k < a.max_keep; k += 64)
        if (k >= count) keep[k] = -1;
    if (kept >> lane & 1) keep[__popcll(kept & ((uint64_t{1} << lane) - 1))] = lane;
    const bool here = __shfl(static_cast<int>(known), at, 64);
    const double sum_p = __shfl(p.sum, at, 64), sum_q = __shfl(q.sum, at, 64);
    const float top = __shfl(p.top, at, 64), draft_top = __shfl(q.top, at, 64);
    const int largest = __shfl(p.at, at, 64);
    if (lane != 0) return;
    a.keep_count[i] = count;
    Leftover y;
    y.row = t.q0 + at;
    y.pieces = here ? a.shape.pieces : a.shape.last_pieces;
    y.c = drawn ? c : 0;
    y.of_target = sum_p > 0 ? 1 / sum_p : 0.0;
    y.of_draft = sum_q > 0 ? 1 / sum_q : 0.0;
    y.top = top; y.draft_top = draft_top;
    y.kind = greedy ? (here ? kNone : kLargest) : !here ? kUnknown : top == -INFINITY ? kNone : !refused ? kKnown : drawn ? kResidual : kRemoved;
    if (here && (greedy || top == -INFINITY)) a.next_token[i] = top == -INFINITY ? -1 : largest;
    if (y.kind == kResidual || y.kind == kRemoved) y.pieces = a.shape.last_pieces;
    a.left[i] = y;
}

// Tokens of the last one's children, all of them refused (kRemoved): in LDS, and how many
__device__ __forceinline__ int removed_tokens(const VerifyArgs& a, const int i, const int64_t row, int* list, int* count) {
    const Tree t = tree_of(a, i);
    const int lane = threadIdx.x & 63, at = static_cast<int>(row - t.q0);
    const uint64_t gone = __ballot(lane < t.tokens && t.parent == at);
    if (threadIdx.x < 64 && gone >> lane & 1) list[__popcll(gone & ((uint64_t{1} << lane) - 1))] = a.tokens[t.q0 + lane];
    if (threadIdx.x == 0) *count = __popcll(gone);
    __syncthreads();
    return *count;
}

// Weights of eight tokens from number `at` on
template <bool F32>
__device__ __forceinline__ void left_weights(const VerifyArgs& a, const Leftover& y, const LeftWeight& w, const int at, const int* list, const int removed, double (&v)[kVector]) {
    float x[kVector], z[kVector];
    load_logits<F32>(a.target, y.row * a.target_stride, at, a.vocab, x);
    if (w.c > 0) load_logits<F32>(a.draft, y.row * a.draft_stride, at, a.vocab, z);
#pragma unroll
    for (int e = 0; e < kVector; ++e) v[e] = w(x[e], w.c > 0 ? z[e] : 0.f);
    for (int r = 0; r < removed; ++r)
#pragma unroll
        for (int e = 0; e < kVector; ++e)
            if (list[r] == at + e) v[e] = 0;
}
__device__ __forceinline__ LeftWeight weight_left(const Leftover& y, const double per) { return {per, y.kind == kResidual ? y.c : 0.0, y.of_target, y.of_draft, y.top, y.draft_top}; }

// Sums of the row that is drawn from, where they are not known: a workgroup for (request, piece)
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_left_kernel(VerifyArgs a) {
    __shared__ RowPart lds[kThreads / 64];
    __shared__ double sums[kThreads / 64];
    __shared__ int list[kMostDrafts], count;
    const int i = blockIdx.x / a.shape.last_pieces, piece = blockIdx.x - i * a.shape.last_pieces;
    const Leftover y = a.left[i];
    if (y.kind == kNone || y.kind == kKnown) return;
    const float warm = temperature_of(a, i);
    const double per = warm > 0.f ? kLog2eWide / warm : 0.0;
    const int first = piece * a.shape.last_length, end = min(first + a.shape.last_length, a.vocab);
    RowPart* to = a.last_parts + static_cast<int64_t>(i) * a.shape.last_pieces + piece;
    if (y.kind == kUnknown || y.kind == kLargest) {
        const RowPart p = part_of_row<F32>(a.target, y.row * a.target_stride, first, end, a.vocab, per, lds);
        if (threadIdx.x == 0) *to = p;
        return;
    }
    const int removed = y.kind == kRemoved ? removed_tokens(a, i, y.row, list, &count) : 0;
    const LeftWeight w = weight_left(y, per);
    double sum = 0;
    for (int at = first + static_cast<int>(threadIdx.x) * kVector; at < end; at += kStep) {
        double v[kVector];
        left_weights<F32>(a, y, w, at, list, removed, v);
#pragma unroll
        for (int e = 0; e < kVector; ++e) sum += v[e];
    }
    sum = sum_of_all(sum, sums);
    if (threadIdx.x == 0) *to = {sum, 0.f, 0};
}

// The draw: a workgroup for a request finds the piece, then the place in it
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyArgs a) {
    __shared__ double sums[kThreads / 64];
    __shared__ int list[kMostDrafts], count;
    __shared__ int found, last_positive;
    const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Leftover y = a.left[i];
    if (y.kind == kNone) return;
    const float warm = temperature_of(a, i);
    const double per = warm > 0.f ? kLog2eWide / warm : 0.0;
    const RowPart* parts = a.last_parts + static_cast<int64_t>(i) * a.shape.last_pieces;
    int pieces = a.shape.last_pieces, length = a.shape.last_length;
    double whole = 0;
    if (y.kind == kResidual || y.kind == kRemoved) {
        for (int z = 0; z < pieces; ++z) whole += parts[z].sum;
        if (!(whole > 0)) y.kind = kKnown;          // nothing is left: from P
    }
    if (y.kind == kKnown) {
        parts = a.parts + y.row * 2 * a.shape.pieces;
        pieces = a.shape.pieces; length = a.shape.length;
    }
    if (y.kind == kKnown || y.kind == kUnknown || y.kind == kLargest) {
        RowPart p{0.0, -INFINITY, 0x7FFFFFFF};
        for (int z = 0; z < pieces; ++z) p = joined(p, parts[z], per);
        if (p.top == -INFINITY || y.kind == kLargest) {
            if (tid == 0) a.next_token[i] = p.top == -INFINITY ? -1 : p.at;
            return;
        }
        y.top = p.top; y.of_target = 1; y.c = 0;
        whole = p.sum;
    }
    const bool relative = y.kind == kKnown || y.kind == kUnknown;                  // (sums of pieces are relative to each one's largest)
    const int removed = y.kind == kRemoved ? removed_tokens(a, i, y.row, list, &count) : 0;
    const LeftWeight w = weight_left(y, per);
    const double goal = min(max(static_cast<double>(a.sample_u[i]), 0.0), 1.0) * whole;            // (NaN: max gives 0)
    // the first piece whose cumulative sum is over the goal; the last one that has any weight where rounding leaves none
    double before = 0, of_piece = 0, upto = 0;
    int piece = 0;
    for (int z = 0; z < pieces; ++z) {
        const double s = parts[z].sum > 0 ? parts[z].sum * (relative ? weight_of(parts[z].top, y.top, per) : 1.0) : 0.0;
        if (!(s > 0)) continue;
        before = upto; upto += s; of_piece = s; piece = z;
        if (upto > goal) break;
    }
    (void)of_piece;
    const int first = piece * length, end = min(first + length, a.vocab);
    if (tid == 0) { found = 0x7FFFFFFF; last_positive = -1; }
    for (int at0 = first; at0 < end; at0 += kStep) {
        const int at = at0 + tid * kVector;
        double v[kVector];
        if (at < end) left_weights<F32>(a, y, w, at, list, removed, v);
        double mine = 0;
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            if (at >= end) v[e] = 0;
            mine += v[e];
        }
        double to_here = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double z = __shfl_up(to_here, o, 64);
            to_here += lane >= o ? z : 0;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = to_here;
        __syncthreads();
        double all = 0, in_front = before;
#pragma unroll
        for (int z = 0; z < kThreads / 64; ++z) {
            in_front += z < wave ? sums[z] : 0;
            all += sums[z];
        }
        double x = in_front + (to_here - mine);
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            x += v[e];
            if (v[e] > 0 && x > goal) { atomicMin(&found, at + e); break; }
        }
#pragma unroll
        for (int e = kVector - 1; e >= 0; --e)
            if (v[e] > 0) { atomicMax(&last_positive, at + e); break; }
        before += all;
        __syncthreads();
        if (found != 0x7FFFFFFF) break;
    }
    if (tid == 0) a.next_token[i] = found != 0x7FFFFFFF ? found : last_positive;
}

template <bool F32>
int launch(const VerifyArgs& a, hipStream_t st) {
    const int64_t rows = static_cast<int64_t>(a.n) * a.max_q * (a.draft ? 2 : 1) * a.shape.pieces, left = static_cast<int64_t>(a.n) * a.shape.last_pieces;
    if (rows > 0x7FFFFFFF || left > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const dim3 block(kThreads);
    hipLaunchKernelGGL((verify_rows_kernel<F32>), dim3(static_cast<unsigned>(rows)), block, 0, st, a);
    hipLaunchKernelGGL((verify_walk_kernel<F32>), dim3(static_cast<unsigned>(a.n)), block, 0, st, a);
    hipLaunchKernelGGL((verify_left_kernel<F32>), dim3(static_cast<unsigned>(left)), block, 0, st, a);
    hipLaunchKernelGGL((verify_draw_kernel<F32>), dim3(static_cast<unsigned>(a.n)), block, 0, st, a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

VerifyShape VerifyShape::of(const int64_t n, const int64_t total_q, const int32_t vocab) {
    const auto cut = [&](const int64_t rows, int& pieces, int& length) {
        const int64_t steps = (static_cast<int64_t>(vocab) + kStep - 1) / kStep, wanted = 2048 / (rows > 0 ? rows : 1) + 1;
        const int64_t each = (steps + (wanted < steps ? wanted : steps) - 1) / (wanted < steps ? wanted : steps);
        length = static_cast<int>(each * kStep < 0x7FFFF000 ? each * kStep : 0x7FFFF000);
        pieces = static_cast<int>((steps + each - 1) / each);
    };
    VerifyShape s;
    cut(total_q, s.pieces, s.length);
    cut(n, s.last_pieces, s.last_length);
    return s;
}

int launch_draft_verify(const VerifyArgs& a, void* stream) {
    return a.f32 ? launch<true>(a, static_cast<hipStream_t>(stream)) : launch<false>(a, static_cast<hipStream_t>(stream));
}

}  // namespace pk
