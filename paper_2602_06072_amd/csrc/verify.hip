// Judging of drafted tokens: which of them stay, and the token behind them.
//
// With target P and draft Q of the last token that stays, its k-th child x stays if P(x) > (c + u Z) Q(x).  That is the usual rule of rejection sampling, r(x) / Q(x) >
// u with the residual r = max(P - c Q, 0) / Z: each refusal takes r to max(r - Q, 0) over its sum, and max(max(P - c Q, 0) / Z - Q, 0) = max(P - (c + Z) Q, 0) / Z, so
// that a node's whole state is two numbers.  What a node decides depends on its own rows alone: all are looked at at once, and the tokens that stay are
// found by going from one choice to the next.
//
// Three launches.  Sums of the rows of tokens with children, target and draft (V logits each, in pieces); the choices of these tokens; then, of every request, the row that the
// next token is drawn from, in pieces again, the last of which to finish finds the place.  One token a request: the last launch alone.
//
// Probabilities and their sums have 64 bits: a draw is the place of a number between V borders, and with sums of 32 bits every tenth draw of a flat row of 100000
// would fall on the other side of one.  Vector instructions of 64 bits run at the rate of those of 32 here; a weight takes about 20 of them, 80 cycles for 64 logits, and
// at 2 10^12 logits a second that, not memory (3 10^12 of bf16), bounds the launches over rows.
#include "arrival.h"
#include "branch.h"
#include "common.hip.h"

namespace pk {
namespace {

constexpr int kThreads = 256, kVector = 16, kStep = VerifyShape::kStep;
static_assert(kStep == kThreads * kVector, "a step is a vector of every thread");
constexpr float kMostLogit = 3.402823466e38f;

// NaN becomes -inf, inf the largest number
__device__ __forceinline__ float plain_logit(const float x) { return fminf(fmaxf(x, -INFINITY), kMostLogit); }

// Sixteen logits from number `at` on, and the largest of them; those behind the row's end are -inf, inf is the largest number.  NaN stays: it is no largest one, and has no
// weight.  Rows of odd length begin anywhere: the loads are 16 bytes long at addresses of any alignment.
// (as they are in memory, so that what is asked for ahead is not waited for)
template <bool F32> struct Raw { uint32_t w[F32 ? kVector : kVector / 2]; };
template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const void* base, const int64_t at) {
    Raw<F32> r;
    __builtin_memcpy(r.w, static_cast<const char*>(base) + at * (F32 ? 4 : 2), sizeof r.w);
    return r;
}
template <bool F32>
__device__ __forceinline__ void unpack(const Raw<F32>& r, float (&x)[kVector]) {
#pragma unroll
    for (int e = 0; e < kVector; ++e) x[e] = __uint_as_float(F32 ? r.w[F32 ? e : 0] : e % 2 == 0 ? r.w[e / 2] << 16 : r.w[e / 2] & 0xFFFF0000u);
}
template <bool F32>
__device__ __forceinline__ void load_last(const void* base, const int64_t row_at, const int at, const int vocab, float (&x)[kVector]) {
#pragma unroll
    for (int e = 0; e < kVector; ++e) {
        x[e] = -INFINITY;
        if (at + e < vocab) x[e] = F32 ? static_cast<const float*>(base)[row_at + at + e] : bf16_bits_to_float(static_cast<const uint16_t*>(base)[row_at + at + e]);
    }
}
template <bool F32>
__device__ __forceinline__ void load_logits(const void* base, const int64_t row_at, const int at, const int vocab, float (&x)[kVector]) {
    if (at + kVector <= vocab) unpack<F32>(load_raw<F32>(base, row_at + at), x);
    else load_last<F32>(base, row_at, at, vocab, x);
}
__device__ __forceinline__ float largest_of(float (&x)[kVector]) {
    // (three at a time, which fmaxf, with its care for signalling NaN, is not compiled to: such a NaN becomes the result, and is seen to below)
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < kVector; e += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(top) : "v"(x[e]), "v"(x[e + 1]));
    if (!(top < INFINITY)) {
        top = -INFINITY;
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            x[e] = plain_logit(x[e]);
            top = fmaxf(top, x[e]);
        }
    }
    return top;
}
template <bool F32>
__device__ __forceinline__ float load_logit(const void* base, const int64_t at) {
    return plain_logit(F32 ? static_cast<const float*>(base)[at] : bf16_bits_to_float(static_cast<const uint16_t*>(base)[at]));
}

// 2^y for y up to 1000; 0 below -1074 and for a NaN.  y = n + f with |f| <= 1/2: adding 1.5 2^52 leaves n in the low bits.  The polynomial has the least largest
// relative error of its degree with p(0) = 1, 8.1e-13 (fitted to 2^f by least squares with weights that follow the error): equal logits of 0 count exactly.
__device__ __forceinline__ double exp2_of(const double y) {
    constexpr double kRound = 6755399441055744.0;
    const double in = fmax(y, -1100.0), t = in + kRound, f = in - (t - kRound);
    double p = 0x1.61c4f0ed5f063p-20;
    p = fma(p, f, 0x1.00d85341b87d0p-16);
    p = fma(p, f, 0x1.430aa882ba307p-13);
    p = fma(p, f, 0x1.5d874d06fe487p-10);
    p = fma(p, f, 0x1.3b2ab5ed6fb84p-7);
    p = fma(p, f, 0x1.c6b08dced3566p-5);
    p = fma(p, f, 0x1.ebfbdff8ede86p-3);
    p = fma(p, f, 0x1.62e42fef89d1ep-1);
    p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, __double2loint(t));
}
// weight of a logit relative to that of `ref`; per: log2 e / temperature
__device__ __forceinline__ double weight_of(const float x, const float ref, const double per) { return exp2_of((static_cast<double>(x) - static_cast<double>(ref)) * per); }
constexpr double kLog2e64 = 1.4426950408889634074;

// Temperature of a request; 0: the largest logit is taken
__device__ __forceinline__ float temperature_of(const VerifyArgs& a, const int i) {
    const float t = a.temperature ? a.temperature[i] : 1.f;
    return t > 0.f ? t : 0.f;
}

// Two parts of a row as one.  Sums are relative to the weight of `top` (any logit that is near enough to the largest for 64 bits; -inf: nothing can be drawn); with
// LARGEST `top` is the largest logit and `at` its first place.
template <bool LARGEST>
__device__ __forceinline__ RowPart joined(const RowPart& x, const RowPart& y, const double per) {
    RowPart z{0.0, fmaxf(x.top, y.top), 0};
    if constexpr (LARGEST) z.at = x.top > y.top || (x.top == y.top && x.at < y.at) ? x.at : y.at;
    else if (x.top == y.top) z.sum = x.sum + y.sum;
    else z.sum = x.top > y.top ? x.sum + (y.top > -INFINITY ? y.sum * weight_of(y.top, x.top, per) : 0.0) : y.sum + (x.top > -INFINITY ? x.sum * weight_of(x.top, y.top, per) : 0.0);
    return z;
}
template <bool LARGEST>
__device__ __forceinline__ RowPart of_wave(RowPart y, const double per) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) y = joined<LARGEST>(y, {__shfl_xor(y.sum, o, 64), __shfl_xor(y.top, o, 64), __shfl_xor(y.at, o, 64)}, per);
    return y;
}
// ... of all threads, in every thread
struct WaveParts { double sum[kThreads / 64]; float top[kThreads / 64]; int at[kThreads / 64]; };
template <bool LARGEST>
__device__ __forceinline__ RowPart of_all(RowPart y, const double per, WaveParts& lds) {
    y = of_wave<LARGEST>(y, per);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        const int wave = threadIdx.x >> 6;
        lds.sum[wave] = y.sum; lds.top[wave] = y.top; lds.at[wave] = y.at;
    }
    __syncthreads();
    y = {lds.sum[0], lds.top[0], lds.at[0]};
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) y = joined<LARGEST>(y, {lds.sum[w], lds.top[w], lds.at[w]}, per);
    return y;
}
constexpr RowPart kNoPart{0.0, -INFINITY, 0x7FFFFFFF};

// Where a request's tokens are: a lane has a token
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
    if (!a.mask) {                                  // one behind the other
        t.parent = lane < t.tokens ? lane - 1 : -1;
        t.inner = t.tokens > 1 ? ~uint64_t{0} >> (65 - t.tokens) : 0;
        return t;
    }
    uint64_t before = 0;                            // ancestors
    if (lane < t.tokens) before = a.mask[t.q0 + lane] & ((uint64_t{1} << lane) - 1);
    t.parent = before ? 63 - __builtin_clzll(before) : -1;
    uint64_t mine = t.parent >= 0 ? uint64_t{1} << t.parent : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine |= __shfl_xor(static_cast<unsigned long long>(mine), o, 64);
    t.inner = mine;
    return t;
}

// A piece of a row, all threads: elements [first, end).  A thread's reference is 0 unless weights would leave the range of 64 bits.
template <bool F32, bool LARGEST>
__device__ __forceinline__ RowPart part_of_row(const void* base, const int64_t row_at, const int first, const int end, const int vocab, const double per, WaveParts& lds) {
    RowPart y = kNoPart;
    constexpr float kFar = 500.f;                   // octaves
    const float octaves = static_cast<float>(per);
    const auto take = [&](float (&x)[kVector], const int at) {
        const float top = largest_of(x);
        if constexpr (LARGEST) {
            if (!(top > y.top)) return;
            y.top = top;
            int place = kVector;
#pragma unroll
            for (int e = kVector - 1; e >= 0; --e) place = x[e] == top ? e : place;
            y.at = at + place;
        } else {
            if (top == -INFINITY) return;
            if (y.top == -INFINITY) {
                y.top = fabsf(top) * octaves <= kFar ? 0.f : top;
            } else if ((top - y.top) * octaves > kFar) {
                y.sum *= weight_of(y.top, top, per);
                y.top = top;
            }
            double sums[2] = {};
            if (__all(y.top == 0.f)) {              // (as nearly always: a subtraction less)
#pragma unroll
                for (int e = 0; e < kVector; ++e) sums[e % 2] += exp2_of(static_cast<double>(x[e]) * per);
            } else {
#pragma unroll
                for (int e = 0; e < kVector; ++e) sums[e % 2] += weight_of(x[e], y.top, per);
            }
            y.sum += sums[0] + sums[1];
        }
    };
    int at = first + static_cast<int>(threadIdx.x) * kVector;
    Raw<F32> ahead;
    if (at + kVector <= end) ahead = load_raw<F32>(base, row_at + at);
    for (; at + kVector <= end; at += kStep) {
        float x[kVector];
        unpack<F32>(ahead, x);
        if (at + kStep + kVector <= end) ahead = load_raw<F32>(base, row_at + at + kStep);
        take(x, at);
    }
    if (at < end) {                                 // the end of a row
        float x[kVector];
        load_last<F32>(base, row_at, at, vocab, x);
        take(x, at);
    }
    return of_all<LARGEST>(y, per, lds);
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

// Sums of the rows of tokens with children: a workgroup for (piece, target or draft; token; request)
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_rows_kernel(VerifyArgs a) {
    __shared__ WaveParts lds;
    const int of_draft = blockIdx.x >= static_cast<unsigned>(a.shape.pieces) ? 1 : 0, piece = blockIdx.x - of_draft * a.shape.pieces, token = blockIdx.y, i = blockIdx.z;
    const Tree t = tree_of(a, i);
    if (!(t.inner >> token & 1)) return;
    const float warm = temperature_of(a, i);
    if (of_draft && warm == 0.f) return;
    const int64_t row = t.q0 + token;
    const int first = piece * a.shape.length, end = min(first + a.shape.length, a.vocab);
    const RowPart y = warm == 0.f ? part_of_row<F32, true>(a.target, row * a.target_stride, first, end, a.vocab, 0.0, lds)
                                  : part_of_row<F32, false>(of_draft ? a.draft : a.target, row * (of_draft ? a.draft_stride : a.target_stride), first, end, a.vocab, kLog2e64 / warm, lds);
    if (threadIdx.x == 0) {
        RowPart& to = a.parts[(row * 2 + of_draft) * a.shape.pieces + piece];
        to.sum = y.sum; to.top = y.top; to.at = y.at;
    }
}

// Weights that are left of a row: max(P - c Q, 0)
struct LeftWeight {
    double per, c, of_target, of_draft;             // 1 / sums of the rows, relative to
    float top, draft_top;
    __device__ __forceinline__ double target(const float x) const { return of(x, top, of_target); }
    __device__ __forceinline__ double draft(const float x) const { return of(x, draft_top, of_draft); }
    __device__ __forceinline__ double of(const float x, const float ref, const double share) const { return share * weight_of(x, ref, per); }
    __device__ __forceinline__ double operator()(const float x, const float y) const { return fmax(target(x) - c * draft(y), 0.0); }
};

// What a token with children decides: a workgroup for (token, request), every wave the same (a lane has a token)
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_choice_kernel(VerifyArgs a) {
    __shared__ double lds[kThreads / 64];
    const int token = blockIdx.x, i = blockIdx.y, lane = threadIdx.x & 63;
    const Tree t = tree_of(a, i);
    if (!(t.inner >> token & 1)) return;
    const float warm = temperature_of(a, i);
    const bool greedy = warm == 0.f, drawn = a.draft && !greedy;
    const double per = greedy ? 0.0 : kLog2e64 / warm;
    const int64_t row = t.q0 + token;
    // this lane's piece of the row (there are no more than 64), its child if its token is one
    const bool child = lane < t.tokens && t.parent == token;
    const int x = child ? a.tokens[t.q0 + lane] : -1;
    const bool able = child && x >= 0 && x < a.vocab;
    const float u = able ? a.accept_u[t.q0 + lane] : 0.f;
    const float xp = able ? load_logit<F32>(a.target, row * a.target_stride + x) : -INFINITY;
    const float xq = able && drawn ? load_logit<F32>(a.draft, row * a.draft_stride + x) : -INFINITY;
    const bool there = lane < a.shape.pieces;
    RowPart p = there ? a.parts[row * 2 * a.shape.pieces + lane] : kNoPart, q = kNoPart;
    if (there && drawn) q = a.parts[(row * 2 + 1) * a.shape.pieces + lane];
    p = greedy ? of_wave<true>(p, per) : of_wave<false>(p, per);
    q = of_wave<false>(q, per);
    LeftWeight w{per, 0.0, p.sum > 0 ? 1 / p.sum : 0.0, q.sum > 0 ? 1 / q.sum : 0.0, p.top, q.top};
    const double mine_p = able ? w.target(xp) : 0.0, mine_q = able && drawn ? w.draft(xq) : 0.0;
    uint64_t left = __ballot(able), gone = 0;       // children to be looked at; those that were refused
    int choice = -1;
    double Z = 1;
    while (left != 0) {
        const int s = __builtin_ctzll(left);
        left &= left - 1;
        const int of = __builtin_amdgcn_readlane(x, s);
        const double px = __shfl(mine_p, s, 64), qx = __shfl(mine_q, s, 64), us = __shfl(u, s, 64);
        const bool before = __ballot((gone >> lane & 1) && x == of) != 0;          // (the same token again)
        if (greedy ? p.top > -INFINITY && p.at == of : drawn ? px > (w.c + us * Z) * qx : !before && px > us * Z) { choice = s; break; }
        if (greedy) continue;
        gone |= uint64_t{1} << s;
        if (!drawn) { Z -= before ? 0.0 : px; continue; }
        w.c += Z;
        if (left == 0) break;                       // (what is left is summed up only for a sibling's sake)
        double sum = 0;
        for (int at = static_cast<int>(threadIdx.x) * kVector; at < a.vocab; at += kStep) {
            float vp[kVector], vq[kVector];
            load_logits<F32>(a.target, row * a.target_stride, at, a.vocab, vp);
            load_logits<F32>(a.draft, row * a.draft_stride, at, a.vocab, vq);
            largest_of(vp);
            largest_of(vq);
#pragma unroll
            for (int e = 0; e < kVector; ++e) sum += w(vp[e], vq[e]);
        }
        Z = sum_of_all(sum, lds);
    }
    if (threadIdx.x == 0) a.choices[row] = {choice, drawn && gone != 0 ? w.c : 0.0, w.of_target, w.of_draft, w.top, w.draft_top};
}

// Sums of pieces of the row that a request's next token is drawn from, and the draw: a workgroup for (piece, request), the last of a request to finish goes on
enum { kPlain, kResidual, kRemoved };               // weights: P; max(P - c Q, 0); P without the tokens that were refused
struct LastCount {
    uint32_t* x;
    __device__ __forceinline__ uint32_t next(const uint32_t limit) const { return __builtin_amdgcn_atomic_inc32(x, limit, __ATOMIC_RELAXED, "agent"); }
};
template <bool F32>
__device__ __forceinline__ void left_weights(const VerifyArgs& a, const int64_t row, const int kind, const LeftWeight& w, const int at, const int* list, const int removed, double (&v)[kVector]) {
    float x[kVector], z[kVector];
    load_logits<F32>(a.target, row * a.target_stride, at, a.vocab, x);
    if (kind == kResidual) {
        load_logits<F32>(a.draft, row * a.draft_stride, at, a.vocab, z);
        largest_of(x);
        largest_of(z);
#pragma unroll
        for (int e = 0; e < kVector; ++e) v[e] = w(x[e], z[e]);
        return;
    }
    largest_of(x);
#pragma unroll
    for (int e = 0; e < kVector; ++e) v[e] = w.target(x[e]);
    if (kind == kRemoved)
        for (int r = 0; r < removed; ++r)
#pragma unroll
            for (int e = 0; e < kVector; ++e)
                if (list[r] == at + e) v[e] = 0;
}
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyArgs a) {
    __shared__ WaveParts lds;
    __shared__ double sums[kThreads / 64];
    __shared__ int list[kMostDrafts];
    __shared__ int last, found, last_positive, the_piece;
    __shared__ double the_begin;
    const int pieces = a.shape.last_pieces, piece = blockIdx.x, i = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Tree t = tree_of(a, i);
    const float warm = temperature_of(a, i);
    const bool greedy = warm == 0.f;
    const double per = greedy ? 0.0 : kLog2e64 / warm;
    // the tokens that stay: from one choice to the next
    int at = 0, count = 1;
    uint64_t kept = 1;
    const int chosen = lane < t.tokens ? a.choices[t.q0 + lane].token : -1, choice = t.inner >> lane & 1 ? chosen : -1;       // (asked for beside the masks)
    for (; count < a.max_keep; ++count) {
        const int next = __builtin_amdgcn_readlane(choice, at);
        if (next < 0) break;
        at = next;
        kept |= uint64_t{1} << at;
    }
    if (t.tokens == 0) count = 0, kept = 0;
    if (piece == 0 && wave == 0) {
        int32_t* keep = a.keep + static_cast<int64_t>(i) * a.max_keep;
        for (int k = count + lane; k < a.max_keep; k += 64) keep[k] = -1;
        if (kept >> lane & 1) keep[__popcll(kept & ((uint64_t{1} << lane) - 1))] = lane;
        if (lane == 0) a.keep_count[i] = count;
        if (lane == 0 && t.tokens == 0) a.next_token[i] = -1;
    }
    if (t.tokens == 0) return;
    // what is left of the last one's row
    const int64_t row = t.q0 + at;
    const bool judged = !greedy && (t.inner >> at & 1) && __builtin_amdgcn_readlane(choice, at) < 0;         // all of its children were refused
    LeftWeight w{per, 0.0, 1.0, 0.0, 0.f, 0.f};
    int kind = kPlain, removed = 0;
    if (judged) {
        const VerifyChoice c = a.choices[row];
        if (a.draft) {
            if (c.c > 0) kind = kResidual;          // (0: none of them is a token)
        } else {
            kind = kRemoved;
            const uint64_t gone = __ballot(lane < t.tokens && t.parent == at);
            removed = __popcll(gone);
            if (wave == 0 && (gone >> lane & 1)) list[__popcll(gone & ((uint64_t{1} << lane) - 1))] = a.tokens[t.q0 + lane];
            __syncthreads();
        }
        w = {per, c.c, kind == kRemoved ? 1.0 : c.of_target, c.of_draft, c.top, c.draft_top};
    }
    const int first = piece * a.shape.last_length, end = min(first + a.shape.last_length, a.vocab);
    RowPart mine{0.0, 0.f, 0};
    if (kind == kPlain) {
        mine = greedy ? part_of_row<F32, true>(a.target, row * a.target_stride, first, end, a.vocab, per, lds)
                      : part_of_row<F32, false>(a.target, row * a.target_stride, first, end, a.vocab, per, lds);
    } else {
        double sum = 0;
        for (int n = first + tid * kVector; n < end; n += kStep) {
            double v[kVector];
            left_weights<F32>(a, row, kind, w, n, list, removed, v);
#pragma unroll
            for (int e = 0; e < kVector; ++e) sum += v[e];
        }
        mine.sum = sum_of_all(sum, sums);
    }
    if (pieces > 1) {
        // (decode_body.hip.h on the order of such stores and the count)
        uint64_t* to = reinterpret_cast<uint64_t*>(a.last_parts + static_cast<int64_t>(i) * pieces);
        if (tid == 0) {
            __hip_atomic_store(to + 2 * piece, static_cast<uint64_t>(__double_as_longlong(mine.sum)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(to + 2 * piece + 1, static_cast<uint64_t>(__float_as_uint(mine.top)) | static_cast<uint64_t>(static_cast<uint32_t>(mine.at)) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0)
            last = arrives_last(LastCount{a.arrived + i}, static_cast<uint32_t>(pieces));
        }
        __syncthreads();
        if (last == 0) return;
        mine = kNoPart;
        if (tid < pieces) {
            mine.sum = __longlong_as_double(static_cast<long long>(__hip_atomic_load(to + 2 * tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
            const uint64_t more = __hip_atomic_load(to + 2 * tid + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            mine.top = __uint_as_float(static_cast<uint32_t>(more));
            mine.at = static_cast<int>(more >> 32);
        }
    } else if (tid > 0) {
        mine = kNoPart;
    }
    // a thread has a piece: the whole row
    RowPart all = greedy ? of_all<true>(mine, per, lds) : of_all<false>(mine, per, lds);
    if (greedy || (kind == kPlain && all.top == -INFINITY)) {
        if (tid == 0) a.next_token[i] = all.top == -INFINITY ? -1 : all.at;
        return;
    }
    int from = 0, to = a.vocab;
    double before = 0, goal = fmin(fmax(static_cast<double>(a.sample_u[i]), 0.0), 1.0);            // (NaN: 0)
    if (kind != kPlain && !(all.sum > 0)) {
        // nothing is left: from P, all of it anew
        kind = kPlain;
        all = part_of_row<F32, false>(a.target, row * a.target_stride, 0, a.vocab, a.vocab, per, lds);
        w.of_target = 1.0; w.top = all.top;
        if (all.top == -INFINITY) {
            if (tid == 0) a.next_token[i] = -1;
            return;
        }
        goal *= all.sum;
    } else {
        if (kind == kPlain) { w.top = all.top; w.of_target = 1.0; }
        goal *= all.sum;
        // the first piece whose cumulative sum is over the goal; the last one that has any weight where rounding leaves none
        const double weight = mine.top == -INFINITY ? 0.0 : kind == kPlain && mine.top != all.top ? mine.sum * weight_of(mine.top, all.top, per) : mine.sum;
        double upto = weight;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double z = __shfl_up(upto, o, 64);
            upto += lane >= o ? z : 0.0;
        }
        if (tid == 0) { found = 0x7FFFFFFF; last_positive = -1; }
        __syncthreads();
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        for (int v = 0; v < wave; ++v) upto += sums[v];
        if (weight > 0) {
            atomicMax(&last_positive, tid);
            if (upto > goal) atomicMin(&found, tid);
        }
        __syncthreads();
        if (tid == (found != 0x7FFFFFFF ? found : last_positive)) { the_piece = tid; the_begin = upto - weight; }
        __syncthreads();
        from = the_piece * a.shape.last_length;
        to = min(from + a.shape.last_length, a.vocab);
        before = the_begin;
    }
    __syncthreads();
    if (tid == 0) { found = 0x7FFFFFFF; last_positive = -1; }
    for (int n0 = from; n0 < to; n0 += kStep) {
        const int n = n0 + tid * kVector;
        double v[kVector], here = 0;
        if (n < to) left_weights<F32>(a, row, kind, w, n, list, removed, v);
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            if (n >= to) v[e] = 0;
            here += v[e];
        }
        double upto = here;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double z = __shfl_up(upto, o, 64);
            upto += lane >= o ? z : 0.0;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        double step = 0, in_front = before;
#pragma unroll
        for (int z = 0; z < kThreads / 64; ++z) {
            in_front += z < wave ? sums[z] : 0.0;
            step += sums[z];
        }
        double x = in_front + (upto - here);
        int hit = 0x7FFFFFFF, positive = -1;
#pragma unroll
        for (int e = 0; e < kVector; ++e) {
            x += v[e];
            if (v[e] > 0) {
                positive = n + e;
                if (x > goal && hit == 0x7FFFFFFF) hit = n + e;
            }
        }
        if (hit != 0x7FFFFFFF) atomicMin(&found, hit);
        if (positive >= 0) atomicMax(&last_positive, positive);
        before += step;
        __syncthreads();
        if (found != 0x7FFFFFFF) break;
    }
    if (tid == 0) a.next_token[i] = found != 0x7FFFFFFF ? found : last_positive;
}

template <bool F32>
int launch(const VerifyArgs& a, hipStream_t st) {
    const dim3 block(kThreads);
    const unsigned n = static_cast<unsigned>(a.n), tokens = static_cast<unsigned>(a.max_q);
    if (a.max_q > 1) {
        hipLaunchKernelGGL((verify_rows_kernel<F32>), dim3(static_cast<unsigned>(a.shape.pieces * (a.draft ? 2 : 1)), tokens, n), block, 0, st, a);
        hipLaunchKernelGGL((verify_choice_kernel<F32>), dim3(tokens, n), block, 0, st, a);
    }
    hipLaunchKernelGGL((verify_draw_kernel<F32>), dim3(static_cast<unsigned>(a.shape.last_pieces), n), block, 0, st, a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

VerifyShape VerifyShape::of(const int64_t n, const int64_t total_q, const int32_t vocab) {
    const auto cut = [&](const int64_t rows, const int64_t groups, const int64_t most, int& pieces, int& length) {
        const int64_t steps = (static_cast<int64_t>(vocab) + kStep - 1) / kStep;
        int64_t wanted = groups / (rows > 0 ? rows : 1) + 1;
        wanted = wanted < most ? wanted : most;
        wanted = wanted < steps ? wanted : steps;
        const int64_t each = (steps + wanted - 1) / wanted;
        length = static_cast<int>(each * kStep);
        pieces = static_cast<int>((steps + each - 1) / each);
    };
    VerifyShape s;
    cut(total_q, 2048, 64, s.pieces, s.length);           // (a lane for each in verify_choice_kernel,
    cut(n, 1024, kThreads, s.last_pieces, s.last_length); //  a thread for each in verify_draw_kernel)
    return s;
}

int launch_draft_verify(const VerifyArgs& a, void* stream) {
    return a.f32 ? launch<true>(a, static_cast<hipStream_t>(stream)) : launch<false>(a, static_cast<hipStream_t>(stream));
}

}  // namespace pk
