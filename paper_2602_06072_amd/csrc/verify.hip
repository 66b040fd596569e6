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
// Where a choice takes no sums of what is left (one child each, or no draft), the first sums have terms of 32 bits, which are near enough for nearly every choice (kCoarse), and
// what the draw needs in 64 bits, the sums of one row of each request, is found in a launch in front of it (chains of 64 requests, 640 rows of 128256 logits: 73 us in
// 64 bits and 97 for the call, when a weight took 20 instructions).
//
// Probabilities and their sums have 64 bits: a draw is the place of a number between V borders, and with sums of 32 bits every tenth draw of a flat row of 100000
// would fall on the other side of one.  Vector instructions of 64 bits run at the rate of those of 32 here; a weight takes about 22 of them, 100 cycles for 64 logits, and
// at 1.6 10^12 logits a second at most that, not memory (3 10^12 of bf16), bounds the launches over rows in 64 bits; terms of 32 bits reach 2.5 10^12, 5.1 TB/s.
#include <algorithm>

#include "arrival.h"
#include "branch.h"
#include "common.hip.h"

namespace pk {
namespace {

constexpr int kThreads = 256, kVector = 16, kStep = VerifyShape::kStep;
static_assert(kStep == kThreads * kVector, "a step is a vector of every thread");
static_assert(VerifyShape::kSpan == 64 * kVector && VerifyShape::kMostSpans == kThreads && VerifyShape::kMostPieces == 64, "lanes and threads that put parts together");
constexpr float kMostLogit = 3.402823466e38f;

// NaN becomes -inf, inf the largest number
__device__ __forceinline__ float plain_logit(const float x) { return fminf(fmaxf(x, -INFINITY), kMostLogit); }

// Sixteen logits as they are in memory, so that what is asked for ahead is not waited for.  Rows of odd length begin anywhere: the loads are 16 bytes long at addresses
// of any alignment.
template <bool F32> struct Raw { uint32_t w[F32 ? kVector : kVector / 2]; };
template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const void* base, const int64_t at) {
    Raw<F32> r;
    __builtin_memcpy(r.w, static_cast<const char*>(base) + at * (F32 ? 4 : 2), sizeof r.w);
    return r;
}
template <bool F32>
__device__ __forceinline__ float logit_of(const Raw<F32>& r, const int e) {
    return __uint_as_float(F32 ? r.w[F32 ? e : 0] : e % 2 == 0 ? r.w[e / 2] << 16 : r.w[e / 2] & 0xFFFF0000u);
}
// The last sixteen of a row, those in front of number `at` hidden (-inf), for a vector that begins there and has fewer
template <bool F32>
__device__ __forceinline__ Raw<F32> load_last(const void* base, const int64_t row_at, const int at, const int vocab) {
    Raw<F32> r;
    if (vocab >= kVector) {
        r = load_raw<F32>(base, row_at + vocab - kVector);
    } else {
#pragma unroll 1
        for (int e = vocab - kVector; e < vocab; e += F32 ? 1 : 2) {               // (a word at a time, from the front)
            const auto half = [&](const int n) { return n >= 0 ? static_cast<uint32_t>(static_cast<const uint16_t*>(base)[row_at + n]) : 0xFF80u; };
            const uint32_t w = F32 ? (e >= 0 ? static_cast<const uint32_t*>(base)[row_at + e] : 0xFF800000u) : half(e) | half(e + 1) << 16;
#pragma unroll
            for (int n = 0; n + 1 < static_cast<int>(sizeof r.w / 4); ++n) r.w[n] = r.w[n + 1];
            r.w[sizeof r.w / 4 - 1] = w;
        }
    }
    const int hidden = at - (vocab - kVector);      // 1 .. 15
#pragma unroll
    for (int n = 0; n < static_cast<int>(sizeof r.w / 4); ++n) {
        if constexpr (F32) r.w[n] = n < hidden ? 0xFF800000u : r.w[n];
        else r.w[n] = (2 * n < hidden ? 0xFF80u : r.w[n] & 0xFFFFu) | (2 * n + 1 < hidden ? 0xFF800000u : r.w[n] & 0xFFFF0000u);
    }
    return r;
}
// The vector that begins at number `at`; `begin`: number of its first logit (some of those in front of `at` are hidden)
template <bool F32>
__device__ __forceinline__ Raw<F32> load_vector(const void* base, const int64_t row_at, const int at, const int vocab, int& begin) {
    const bool whole = at + kVector <= vocab;
    begin = whole ? at : vocab - kVector;
    return whole ? load_raw<F32>(base, row_at + at) : load_last<F32>(base, row_at, at, vocab);
}
// each(four logits, number of the first one among the sixteen): for code that is short (a launch of little work waits for its instructions, too), which four logits
// at a time keep as busy as sixteen.  NaN becomes -inf, inf the largest number, but with AS_IS.
template <bool F32, int UNROLL = 1, bool AS_IS = false, class Each>
__device__ __forceinline__ void by_four(Raw<F32> r, Each each) {
#pragma unroll UNROLL
    for (int e = 0; e < kVector; e += 4) {
        float x[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) x[n] = AS_IS ? logit_of<F32>(r, n) : plain_logit(logit_of<F32>(r, n));
        each(x, e);
#pragma unroll
        for (int n = 0; n + (F32 ? 4 : 2) < static_cast<int>(sizeof r.w / 4); ++n) r.w[n] = r.w[n + (F32 ? 4 : 2)];
    }
}
// The largest of sixteen logits.  NaN is none; inf and NaN have been replaced where `odd` comes back.
template <bool F32>
__device__ __forceinline__ float largest_of(const Raw<F32>& r, bool& odd) {
    // (three at a time, which fmaxf, with its care for signalling NaN, is not compiled to: such a NaN becomes the result, and is seen to below)
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < kVector; e += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(top) : "v"(logit_of<F32>(r, e)), "v"(logit_of<F32>(r, e + 1)));
    odd = !(top < INFINITY);
    if (odd) {
        top = -INFINITY;
        by_four<F32>(r, [&](const float (&x)[4], int) { top = fmaxf(fmaxf(top, fmaxf(x[0], x[1])), fmaxf(x[2], x[3])); });
    }
    return top;
}
template <bool F32>
__device__ __forceinline__ float load_logit(const void* base, const int64_t at) {
    return plain_logit(F32 ? static_cast<const float*>(base)[at] : bf16_bits_to_float(static_cast<const uint16_t*>(base)[at]));
}

// A constant in scalar registers.  Left alone, the compiler holds those of a single weight in vector registers over the loop that it stands in: twenty more, with which the
// first sums in terms of 32 bits spill (chains of 64 requests 87.5 us instead of 84.5).
__device__ __forceinline__ double scalar(double x) {
    asm("" : "+s"(x));
    return x;
}
// 2^y for y up to 1000; 0 below -1074 and for a NaN.  y = n + f with |f| <= 1/2: adding 1.5 2^52 leaves n in the low bits.  The polynomial has the least largest
// relative error of its degree with p(0) = 1, 2.2e-16 (exchange of extremal points, 60 digits), so that what is left are roundings of 64 bits; equal logits of 0 count exactly.
// (Degree 8, 8.1e-13, saves two instructions of 22: 81 us instead of 82.5 for chains of 64 requests, 74 instead of 79 for trees, 44.3 instead of 45.5 for looked-up tokens.  But a
// number within 1e-13 of a border then falls to its other side.)
__device__ __forceinline__ double exp2_of(const double y) {
    constexpr double kRound = 6755399441055744.0;
    const double in = fmax(y, -1100.0), t = in + kRound, f = in - (t - kRound);
    double p = 0x1.e3a9046bc2ff4p-28;
    p = fma(p, f, scalar(0x1.b671b2f14537ap-24));
    p = fma(p, f, scalar(0x1.62c147a4afdfcp-20));
    p = fma(p, f, scalar(0x1.ffcb58ca31191p-17));
    p = fma(p, f, scalar(0x1.4309126c00bdfp-13));
    p = fma(p, f, scalar(0x1.5d87fe9b8efd1p-10));
    p = fma(p, f, scalar(0x1.3b2ab6fbd6d05p-7));
    p = fma(p, f, scalar(0x1.c6b08d703e17ap-5));
    p = fma(p, f, scalar(0x1.ebfbdff82c431p-3));
    p = fma(p, f, scalar(0x1.62e42fefa3a12p-1));
    p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, __double2loint(t));
}
// weight of a logit relative to that of `ref`; that of a logit of 0 and less than inf, the same to the last bit where ref is 0
__device__ __forceinline__ double weight_of(const float x, const float ref, const double per) { return exp2_of((static_cast<double>(x) - static_cast<double>(ref)) * per); }
__device__ __forceinline__ double weight_of(const float x, const double per) { return exp2_of(static_cast<double>(x) * per); }
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
    if constexpr (!LARGEST) {
        if (__all(y.top == 0.f || y.top == -INFINITY)) {           // (as nearly always)
            y.top = __any(y.top == 0.f) ? 0.f : -INFINITY;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) y.sum += __shfl_xor(y.sum, o, 64);
            return y;
        }
    }
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

// Sixteen logits, the first of them number `begin`, to what a thread has of a row.  Its reference is 0 unless weights would leave the range of 64 bits.  kFast: many of them.
// kCoarse: terms of 32 bits where none is over 2^60 or, of the largest, under 2^-60.  With exponents y of two: y has two roundings of 2^-24 (of the factor and the product), which
// are 60 ln 2 2^-23 = 5e-6 of a term; the exponential has 2^-23, sums of sixteen 16 2^-24: together 6.1e-6 of the sum.  (Terms further below weigh nothing.)
enum Sums64 { kExact, kFast, kCoarse };
constexpr double kCoarseError = 6.1e-6;
template <bool F32, Sums64 HOW>
__device__ __forceinline__ void add_weights(RowPart& y, const Raw<F32>& r, const double per, const float octaves) {
    constexpr float kFar = 500.f;
    bool odd;
    const float top = largest_of<F32>(r, odd);
    if (top == -INFINITY) return;
    if (y.top == -INFINITY) {
        y.top = fabsf(top) * octaves <= kFar ? 0.f : top;
    } else if ((top - y.top) * octaves > kFar) {
        y.sum *= weight_of(y.top, top, per);
        y.top = top;
    }
    if (HOW == kCoarse && __all(y.top == 0.f && !odd && fabsf(top) * octaves <= 60.f)) {
        float coarse[2] = {};
#pragma unroll
        for (int e = 0; e < kVector; ++e) coarse[e % 2] += __builtin_amdgcn_exp2f(logit_of<F32>(r, e) * octaves);
        const float sum = coarse[0] + coarse[1];
        if (sum == sum) {                           // (no NaN among them)
            y.sum += static_cast<double>(sum);
            return;
        }
    }
    double sums[2] = {};
    const bool near = __all(y.top == 0.f && !odd);  // (as nearly always: a subtraction less)
    if (HOW == kFast && near) {
#pragma unroll
        for (int e = 0; e < kVector; ++e) sums[e % 2] += weight_of(logit_of<F32>(r, e), per);
    } else {
        by_four<F32>(r, [&](const float (&x)[4], int) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[e % 2] += weight_of(x[e], y.top, per);
        });
    }
    y.sum += sums[0] + sums[1];
}
template <bool F32>
__device__ __forceinline__ void add_largest(RowPart& y, const Raw<F32>& r, const int begin) {
    bool odd;
    const float top = largest_of<F32>(r, odd);
    if (!(top > y.top)) return;
    y.top = top;
    int place = kVector;
    by_four<F32>(r, [&](const float (&x)[4], const int e) {
#pragma unroll
        for (int n = 3; n >= 0; --n) place = x[n] == top ? min(place, e + n) : place;
    });
    y.at = begin + place;
}

// A piece of a row, all threads: elements [first, end)
template <bool F32, bool LARGEST, Sums64 HOW = kFast>
__device__ __forceinline__ RowPart part_of_row(const void* base, const int64_t row_at, const int first, const int end, const int vocab, const double per, WaveParts& lds) {
    RowPart y = kNoPart;
    const float octaves = static_cast<float>(per);
    int at = first + static_cast<int>(threadIdx.x) * kVector;
    Raw<F32> ahead;
    if (at + kVector <= end) ahead = load_raw<F32>(base, row_at + at);
#pragma unroll 1
    for (; at < end; at += kStep) {
        const bool whole = at + kVector <= end;
        Raw<F32> r = ahead;
        if (!whole) r = load_last<F32>(base, row_at, at, vocab);                   // (the end of a row: pieces are multiples of a vector)
        else if (at + kStep + kVector <= end) ahead = load_raw<F32>(base, row_at + at + kStep);
        if constexpr (LARGEST) add_largest<F32>(y, r, whole ? at : vocab - kVector);
        else add_weights<F32, HOW>(y, r, per, octaves);
    }
    return of_all<LARGEST>(y, per, lds);
}
template <int THREADS>
__device__ __forceinline__ double sum_of_all(double x, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double y = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) y += lds[w];
    return y;
}

// Sums of the rows of tokens with children: a workgroup for (piece, target or draft; token; request).  Chains of 64 requests (640 rows of 128256 logits) 32 us with terms of
// 32 bits, 5.1 TB/s; 581 rows of 50257 logits that begin at any address 16, 3.7 TB/s; trees (612 rows of 32000 in fp32) in 64 bits 25.
template <bool F32, Sums64 HOW>
__global__ __launch_bounds__(kThreads, F32 ? 5 : 6) void verify_rows_kernel(VerifyArgs a) {
    __shared__ WaveParts lds;
    const int of_draft = blockIdx.x >= static_cast<unsigned>(a.shape.pieces) ? 1 : 0, piece = blockIdx.x - of_draft * a.shape.pieces, token = blockIdx.y, i = blockIdx.z;
    const Tree t = tree_of(a, i);
    if (!(t.inner >> token & 1)) return;
    const float warm = temperature_of(a, i);
    if (of_draft && warm == 0.f) return;
    const int64_t row = t.q0 + token;
    const int first = piece * a.shape.length, end = min(first + a.shape.length, a.vocab);
    const RowPart y = warm == 0.f ? part_of_row<F32, true>(a.target, row * a.target_stride, first, end, a.vocab, 0.0, lds)
                                  : part_of_row<F32, false, HOW>(of_draft ? a.draft : a.target, row * (of_draft ? a.draft_stride : a.target_stride), first, end, a.vocab, kLog2e64 / warm, lds);
    if (threadIdx.x == 0) {
        RowPart& to = a.parts[(row * 2 + of_draft) * a.shape.pieces + piece];
        to.sum = y.sum; to.top = y.top; to.at = y.at;
        if (HOW == kFast && !of_draft && piece == 0) a.choices[row].arrived = 0;
    }
}

// Weights that are left of a row: max(P - c Q, 0).  `near`: both rows' sums are relative to logits of 0, and neither row has an inf (weights of less than 2^500 with such a
// scale); then a weight is max(e^x - ratio e^y, 0) times 1 / sum.
struct LeftWeight {
    double per, c, of_target, of_draft;             // 1 / sums of the rows, relative to
    float top, draft_top;
    double ratio;
    bool near;
    __device__ __forceinline__ void set() {         // (behind any change)
        near = top == 0.f && (c == 0 || draft_top == 0.f) && of_target > 0 && per >= 1e-30;
        ratio = c == 0 ? 0.0 : c * of_draft / of_target;
    }
    __device__ __forceinline__ double target(const float x) const { return of_target * weight_of(x, top, per); }
    __device__ __forceinline__ double draft(const float x) const { return of_draft * weight_of(x, draft_top, per); }
    __device__ __forceinline__ double left(const float x, const float y) const {
        return near ? of_target * fmax(fma(-ratio, weight_of(y, per), weight_of(x, per)), 0.0) : fmax(target(x) - c * draft(y), 0.0);
    }
};

// Sum of what is left of sixteen tokens, the first of them number `begin`
template <bool F32, int UNROLL = 1>
__device__ __forceinline__ double left_of(const Raw<F32>& p, Raw<F32> q, const bool of_two, const LeftWeight& w, const int begin, const int* list, const int removed) {
    double sum = 0;
    const auto add = [&](double (&v)[4], const int e) {
        for (int r = 0; r < removed; ++r)
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = list[r] == begin + e + n ? 0.0 : v[n];
#pragma unroll
        for (int n = 0; n < 4; ++n) sum += v[n];
    };
    const auto next_of_q = [&] {
#pragma unroll
        for (int n = 0; n + (F32 ? 4 : 2) < static_cast<int>(sizeof q.w / 4); ++n) q.w[n] = q.w[n + (F32 ? 4 : 2)];
    };
    if (w.near) {
        by_four<F32, UNROLL, true>(p, [&](const float (&x)[4], const int e) {
            double v[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = weight_of(x[n], w.per);
            if (of_two) {
#pragma unroll
                for (int n = 0; n < 4; ++n) v[n] = fmax(fma(-w.ratio, weight_of(logit_of<F32>(q, n), w.per), v[n]), 0.0);
                next_of_q();
            }
            add(v, e);
        });
        return w.of_target * sum;
    }
    by_four<F32>(p, [&](const float (&x)[4], const int e) {
        double v[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = w.target(x[n]);
        if (of_two) {
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = fmax(v[n] - w.c * w.draft(plain_logit(logit_of<F32>(q, n))), 0.0);
            next_of_q();
        }
        add(v, e);
    });
    return sum;
}

struct LastCount {
    uint32_t* x;
    __device__ __forceinline__ uint32_t next(const uint32_t limit) const { return __builtin_amdgcn_atomic_inc32(x, limit, __ATOMIC_RELAXED, "agent"); }
};

// What a token with children decides: a workgroup for (token, request), every wave the same (a lane has a token).  Without sums of what is left 6 us, loads one behind the
// other; each of them is a pass over two rows by one unit, 64000 weights in 8 us, and a token's siblings need them one after the other, which bounds the launch for trees.
// THREADS: where sums of what is left are to be expected (a mask and a draft), 512, as the one workgroup of a token waits for its loads: 16 trees of 16 to 48 tokens, 32000
// logits of 32 bits, 40 us (256: 48, 1024: 41).  Without such sums 256, which begin sooner.
// MORE: workgroups share the first of those sums, and the last one to finish goes on, where tokens are too few for the machine: 4 trees of 16 tokens, 128256 logits, 80 -> 53 us
// for the whole call, one of 64 tokens 100 -> 69, 16 of 32 215 -> 199; 16 of 24 with 32000 logits 63 either way; with four parts for every token 16 trees of 16 to 48 73 -> 76.
// (Both sides with weights of 20 instructions.)  Terms of 32 bits: registers for four workgroups a unit, looked-up tokens 46.9 -> 45.5.
template <bool F32, Sums64 HOW, int THREADS, bool MORE = false>
__global__ __launch_bounds__(THREADS, MORE || HOW == kCoarse ? 4 : 1) void verify_choice_kernel(VerifyArgs a) {
    __shared__ double lds[THREADS / 64];
    __shared__ WaveParts parts_lds;
    __shared__ int last;
    const int token = blockIdx.x, i = blockIdx.y, part = MORE ? blockIdx.z : 0, lane = threadIdx.x & 63;
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
    LeftWeight w{per};
    double mine_p = 0, mine_q = 0, Z = 1;
    uint64_t left = 0, gone = 0;                    // children to be looked at; those that were refused
    int choice = -1;
    bool exact = HOW != kCoarse;
    const auto begin_with = [&] {
        w = {per, 0.0, p.sum > 0 ? 1 / p.sum : 0.0, q.sum > 0 ? 1 / q.sum : 0.0, p.top, q.top};
        mine_p = able ? w.target(xp) : 0.0;
        mine_q = able && drawn ? w.draft(xq) : 0.0;
        left = __ballot(able);
        gone = 0;
        Z = 1;
    };
    begin_with();
    bool together = MORE && drawn && __popcll(left) > 1;           // (none of the sums has been begun)
    if (part > 0 && !together) return;
    while (left != 0) {
        const int s = __builtin_ctzll(left);
        left &= left - 1;
        const int of = __builtin_amdgcn_readlane(x, s);
        const double px = __shfl(mine_p, s, 64), qx = __shfl(mine_q, s, 64), us = __shfl(u, s, 64);
        const bool before = __ballot((gone >> lane & 1) && x == of) != 0;          // (the same token again)
        const double least = drawn ? (w.c + us * Z) * qx : us * Z;
        // Sums of 32 bits that do not decide it: of P(x) and of Q(x), or of what has left P, each is off by kCoarseError at most.  The row anew, in 64 bits.
        if (HOW == kCoarse && !exact && !greedy && fabs(px - least) <= 4 * kCoarseError * (px + (drawn ? least : us))) {
            p = part_of_row<F32, false>(a.target, row * a.target_stride, 0, a.vocab, a.vocab, per, parts_lds);
            if (drawn) q = part_of_row<F32, false>(a.draft, row * a.draft_stride, 0, a.vocab, a.vocab, per, parts_lds);
            exact = true;
            begin_with();
            continue;
        }
        if (greedy ? p.top > -INFINITY && p.at == of : drawn ? px > least : !before && px > least) { choice = s; break; }
        if (greedy) continue;
        gone |= uint64_t{1} << s;
        if (!drawn) { Z -= before ? 0.0 : px; continue; }
        w.c += Z;
        w.set();
        if (HOW == kCoarse || left == 0) break;     // (what is left is summed up only for a sibling's sake)
        double sum = 0;
        constexpr int STEP = THREADS * kVector;
#pragma unroll 1
        for (int at = (together ? part * STEP : 0) + static_cast<int>(threadIdx.x) * kVector; at < a.vocab; at += together ? a.choice_parts * STEP : STEP) {
            int begin;
            const Raw<F32> vp = load_vector<F32>(a.target, row * a.target_stride, at, a.vocab, begin), vq = load_vector<F32>(a.draft, row * a.draft_stride, at, a.vocab, begin);
            sum += left_of<F32, 4>(vp, vq, true, w, begin, nullptr, 0);
        }
        Z = sum_of_all<THREADS>(sum, lds);
        if (MORE && together) {
            VerifyChoice& c = a.choices[row];
            if (threadIdx.x == 0) {                // (decode_body.hip.h on the order of such stores and the count)
                __hip_atomic_store(reinterpret_cast<uint64_t*>(c.left + part), static_cast<uint64_t>(__double_as_longlong(Z)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0)
                last = arrives_last(LastCount{&c.arrived}, a.choice_parts);
            }
            __syncthreads();
            if (last == 0) return;
            together = false;
            Z = 0;
            for (int n = 0; n < a.choice_parts; ++n)
                Z += __longlong_as_double(static_cast<long long>(__hip_atomic_load(reinterpret_cast<uint64_t*>(c.left + n), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
        }
    }
    if (part > 0 && together) return;              // (a child stays, and no sum was needed)
    if (threadIdx.x == 0) {
        VerifyChoice& c = a.choices[row];
        c.token = choice;
        c.c = drawn && gone != 0 ? w.c : 0.0;
        c.of_target = w.of_target; c.of_draft = w.of_draft;
        c.top = w.top; c.draft_top = w.draft_top;
    }
}

__device__ __forceinline__ double sum_to_here(double x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double z = __shfl_up(x, o, 64);
        x += lane >= o ? z : 0.0;
    }
    return x;
}

// The tokens that stay: from one choice to the next
struct Walk { int at, count; uint64_t kept; };      // the last one, how many, which
__device__ __forceinline__ Walk walk_of(const VerifyArgs& a, const Tree& t) {
    const int lane = threadIdx.x & 63;
    const int chosen = lane < t.tokens && a.max_q > 1 ? a.choices[t.q0 + lane].token : -1;         // (asked for beside the masks)
    const int choice = t.inner >> lane & 1 ? chosen : -1;
    Walk w{0, 1, 1};
    for (; w.count < a.max_keep; ++w.count) {
        const int next = __builtin_amdgcn_readlane(choice, w.at);
        if (next < 0) break;
        w.at = next;
        w.kept |= uint64_t{1} << next;
    }
    if (t.tokens == 0) { w.count = 0; w.kept = 0; }
    return w;
}

// Parts of a row for another workgroup of the launch (decode_body.hip.h on the order of such stores and the count)
__device__ __forceinline__ void store_part(uint64_t* to, const RowPart& y) {
    __hip_atomic_store(to, static_cast<uint64_t>(__double_as_longlong(y.sum)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(to + 1, static_cast<uint64_t>(__float_as_uint(y.top)) | static_cast<uint64_t>(static_cast<uint32_t>(y.at)) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ RowPart load_part(const uint64_t* from) {
    const uint64_t sum = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), more = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return {__longlong_as_double(static_cast<long long>(sum)), __uint_as_float(static_cast<uint32_t>(more)), static_cast<int>(more >> 32)};
}

// In 64 bits, the sums of the rows that are drawn from as max(P - c Q, 0), where the choices had them in 32: workgroups as for the draw.  Up to 64 pairs of rows of
// 128256 logits 19 us, 0.9 10^12 logits a second: half of it the way there and the end.
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyArgs a) {
    __shared__ WaveParts lds;
    __shared__ int last;
    const int i = blockIdx.y, tid = threadIdx.x;
    const Tree t = tree_of(a, i);
    const float warm = temperature_of(a, i);
    const Walk k = walk_of(a, t);
    if (t.tokens == 0 || warm == 0.f || k.count >= a.max_keep || !(t.inner >> k.at & 1)) return;
    const int64_t row = t.q0 + k.at;
    if (!(a.choices[row].c > 0)) return;
    const double per = kLog2e64 / warm;
    const int length = a.shape.group_spans * a.shape.span_rounds * 64 * kVector, first = blockIdx.x * length, end = min(first + length, a.vocab);
    RowPart p = part_of_row<F32, false>(a.target, row * a.target_stride, first, end, a.vocab, per, lds);
    RowPart q = part_of_row<F32, false>(a.draft, row * a.draft_stride, first, end, a.vocab, per, lds);
    if (gridDim.x > 1) {
        uint64_t* parts = reinterpret_cast<uint64_t*>(a.last_parts + static_cast<int64_t>(i) * a.shape.last_stride);
        if (tid == 0) {
            store_part(parts + 4 * blockIdx.x, p);
            store_part(parts + 4 * blockIdx.x + 2, q);
            __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0)
            last = arrives_last(LastCount{a.arrived + i}, gridDim.x);
        }
        __syncthreads();
        if (last == 0) return;
        const bool there = tid < static_cast<int>(gridDim.x);
        p = there ? load_part(parts + 4 * tid) : kNoPart;
        q = there ? load_part(parts + 4 * tid + 2) : kNoPart;
        p = of_all<false>(p, per, lds);
        q = of_all<false>(q, per, lds);
    }
    if (tid == 0) {
        VerifyChoice& c = a.choices[row];
        c.of_target = p.sum > 0 ? 1 / p.sum : 0.0; c.top = p.top;
        c.of_draft = q.sum > 0 ? 1 / q.sum : 0.0; c.draft_top = q.top;
    }
}

// The draw: sums of the row that a request's next token is drawn from, a wave for a span of it (up to 256 spans, of 1024 tokens where V is up to 2^18), a workgroup for some
// of them; the last workgroup of a request to finish finds the span, one wave of it the vector in the span and the token in the vector.  Four rows of 32000 logits 9.7 us,
// the chain of loads and the end; 200 rows of 50257 and 64 pairs of rows of 128256 24, of them 10 to 13 for the weights.
// One token a request of whole batches, 128256 logits of bf16: 64 rows 20 us, 256 rows 53 (10.6 at memory's rate): weights by four, in the form for few rows.  bf16: registers for four workgroups a unit (131
// otherwise, three: chains of 64 requests 84.5 us instead of 82, looked-up tokens 49.5 instead of 47).
enum { kPlain, kResidual, kRemoved };               // weights: P; max(P - c Q, 0); P without the tokens that were refused
template <bool F32>
__global__ __launch_bounds__(kThreads, F32 ? 3 : 4) void verify_draw_kernel(VerifyArgs a) {
    __shared__ WaveParts lds;
    __shared__ double wave_sums[kThreads / 64], begin_of_span;
    __shared__ int list[kMostDrafts];
    __shared__ int last, over_span, positive_span;
    const int i = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Tree t = tree_of(a, i);
    const float warm = temperature_of(a, i);
    const bool greedy = warm == 0.f;
    const double per = greedy ? 0.0 : kLog2e64 / warm;
    const auto [at, count, kept] = walk_of(a, t);
    if (blockIdx.x == 0 && wave == 0) {
        int32_t* keep = a.keep + static_cast<int64_t>(i) * a.max_keep;
        for (int k = count + lane; k < a.max_keep; k += 64) keep[k] = -1;
        if (kept >> lane & 1) keep[__popcll(kept & ((uint64_t{1} << lane) - 1))] = lane;
        if (lane == 0) a.keep_count[i] = count;
        if (lane == 0 && t.tokens == 0) a.next_token[i] = -1;
    }
    if (t.tokens == 0) return;
    // what is left of the last one's row
    const int64_t row = t.q0 + at, target_at = row * a.target_stride, draft_at = row * a.draft_stride;
    const bool judged = !greedy && count < a.max_keep && (t.inner >> at & 1);      // (and none of its children has stayed)
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
        w = {per, kind == kResidual ? c.c : 0.0, kind == kRemoved ? 1.0 : c.of_target, c.of_draft, c.top, c.draft_top};
        w.set();
    }

    const int spans = a.shape.spans, rounds = a.shape.span_rounds;                 // rounds: times 1024 tokens of a span
    const auto first_of = [&](const int span, const int round) { return (span * rounds + round) * (64 * kVector) + lane * kVector; };
    uint64_t* parts = reinterpret_cast<uint64_t*>(a.last_parts + static_cast<int64_t>(i) * a.shape.last_stride);
    RowPart mine, all;
    for (int turn = 0;; ++turn) {
        // (a second turn: nothing is left, and the last workgroup has all of P)
        const int end = turn > 0 ? spans : min((static_cast<int>(blockIdx.x) + 1) * a.shape.group_spans, spans);
        int span = (turn > 0 ? 0 : static_cast<int>(blockIdx.x) * a.shape.group_spans) + wave, round = 0, begin;
        const bool of_two = kind == kResidual;
        Raw<F32> p, q;
        const auto ask = [&](const int n) {
            if (n >= a.vocab) return;
            p = load_vector<F32>(a.target, target_at, n, a.vocab, begin);
            q = p;
            if (of_two) q = load_vector<F32>(a.draft, draft_at, n, a.vocab, begin);
        };
        mine = kind == kPlain ? kNoPart : RowPart{0.0, 0.f, 0};
        if (span < end) ask(first_of(span, 0));
#pragma unroll 1
        while (span < end) {
            const int n = first_of(span, round), this_begin = begin;
            const Raw<F32> r = p, s = q;
            const bool ends = round + 1 == rounds;
            const int next_span = ends ? span + kThreads / 64 : span, next_round = ends ? 0 : round + 1;
            if (next_span < end) ask(first_of(next_span, next_round));
            if (n < a.vocab) {
                if (kind != kPlain) mine.sum += left_of<F32>(r, s, of_two, w, this_begin, list, removed);
                else if (greedy) add_largest<F32>(mine, r, this_begin);
                else add_weights<F32, kExact>(mine, r, per, static_cast<float>(per));
            }
            if (ends) {
                const RowPart y = greedy ? of_wave<true>(mine, per) : of_wave<false>(mine, per);
                if (lane == 0) store_part(parts + 2 * span, y);
                mine = kind == kPlain ? kNoPart : RowPart{0.0, 0.f, 0};
            }
            span = next_span; round = next_round;
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0)
        __syncthreads();
        if (turn == 0 && gridDim.x > 1) {
            if (tid == 0) last = arrives_last(LastCount{a.arrived + i}, gridDim.x);
            __syncthreads();
            if (last == 0) return;
        }
        mine = kNoPart;
        if (tid < spans) mine = load_part(parts + 2 * tid);
        all = greedy ? of_all<true>(mine, per, lds) : of_all<false>(mine, per, lds);
        if (kind == kPlain || all.sum > 0) break;
        kind = kPlain;
        removed = 0;                                // (tokens that were refused have their weights again)
    }
    if (greedy || all.top == -INFINITY) {
        if (tid == 0) a.next_token[i] = all.top == -INFINITY ? -1 : all.at;
        return;
    }
    if (kind == kPlain) { w.top = all.top; w.of_target = 1.0; w.c = 0; w.set(); }
    const double goal = fmin(fmax(static_cast<double>(a.sample_u[i]), 0.0), 1.0) * all.sum;        // (NaN: 0)
    // The first span with a cumulative sum over the goal; the last one with a weight where rounding leaves none.  The same then for vectors and tokens.
    {
        const double weight = mine.top == -INFINITY ? 0.0 : mine.top != all.top ? mine.sum * weight_of(mine.top, all.top, per) : mine.sum;
        double upto = sum_to_here(weight);
        if (lane == 63) wave_sums[wave] = upto;
        if (tid == 0) { over_span = kThreads; positive_span = 0; }
        __syncthreads();
        for (int v = 0; v < wave; ++v) upto += wave_sums[v];
        const uint64_t positive = __ballot(weight > 0), over = __ballot(weight > 0 && upto > goal);
        if (lane == 0 && positive) atomicMax(&positive_span, wave * 64 + 63 - __builtin_clzll(positive));
        if (lane == 0 && over) atomicMin(&over_span, wave * 64 + __builtin_ctzll(over));
        __syncthreads();
        if (tid == (over_span < kThreads ? over_span : positive_span)) begin_of_span = upto - weight;
        __syncthreads();
    }
    if (wave != 0) return;
    bool over_goal = over_span < kThreads;
    const int span = over_goal ? over_span : positive_span;
    double before = begin_of_span;
    int vector = -1;
    bool found = false;
#pragma unroll 1
    for (int round = 0; round < rounds && !found; ++round) {
        const int n = first_of(span, round);
        double weight = 0;
        if (n < a.vocab) {
            int begin;
            const Raw<F32> p = load_vector<F32>(a.target, target_at, n, a.vocab, begin);
            Raw<F32> q = p;
            if (kind == kResidual) q = load_vector<F32>(a.draft, draft_at, n, a.vocab, begin);
            weight = left_of<F32>(p, q, kind == kResidual, w, begin, list, removed);
        }
        const double upto = before + sum_to_here(weight);
        const uint64_t positive = __ballot(weight > 0), over = __ballot(over_goal && weight > 0 && upto > goal);
        const int of = over ? __builtin_ctzll(over) : positive ? 63 - __builtin_clzll(positive) : -1;
        if (of >= 0) vector = __shfl(n, of, 64);
        found = over != 0;
        before = found ? __shfl(upto - weight, of, 64) : __shfl(upto, 63, 64);
    }
    over_goal = over_goal && found;
    const int n = vector + lane;
    double weight = 0;
    if (lane < kVector && vector >= 0 && n < a.vocab) {
        const float x = load_logit<F32>(a.target, target_at + n);
        weight = kind == kResidual ? w.left(x, load_logit<F32>(a.draft, draft_at + n)) : w.target(x);
        for (int r = 0; r < removed; ++r) weight = list[r] == n ? 0.0 : weight;
    }
    const double upto = before + sum_to_here(weight);
    const uint64_t positive = __ballot(weight > 0), over = __ballot(over_goal && weight > 0 && upto > goal);
    if (lane == 0) a.next_token[i] = over ? vector + __builtin_ctzll(over) : positive ? vector + 63 - __builtin_clzll(positive) : -1;
}

constexpr int64_t kCoarseLogits = int64_t{1} << 23;
constexpr int64_t kChoices = 1024;                  // workgroups to be had for the choices of trees
template <bool F32>
int launch(const VerifyArgs& a, hipStream_t st) {
    const dim3 block(kThreads);
    const unsigned n = static_cast<unsigned>(a.n), tokens = static_cast<unsigned>(a.max_q);
    if (a.max_q > 1) {
        const dim3 rows(static_cast<unsigned>(a.shape.pieces * (a.draft ? 2 : 1)), tokens, n), groups(static_cast<unsigned>(a.shape.groups), n);
        // (chains with a draft: what the further launch takes, 6 us and more, has to be saved)
        if (!a.draft || (!a.mask && a.total_q * a.vocab >= kCoarseLogits)) {
            hipLaunchKernelGGL((verify_rows_kernel<F32, kCoarse>), rows, block, 0, st, a);
            hipLaunchKernelGGL((verify_choice_kernel<F32, kCoarse, kThreads>), dim3(tokens, n), block, 0, st, a);
            if (a.draft) hipLaunchKernelGGL((verify_sums_kernel<F32>), groups, block, 0, st, a);
        } else {
            hipLaunchKernelGGL((verify_rows_kernel<F32, kFast>), rows, block, 0, st, a);
            VerifyArgs b = a;
            const int64_t steps = (a.vocab + 512 * kVector - 1) / (512 * kVector), each = kChoices / (a.total_q > 0 ? a.total_q : 1);
            // (two or three parts of a row of few steps save what they cost: 16 trees of 16 to 48 tokens, 32000 logits, 73.1 us, with two 74.4)
            b.choice_parts = each < 4 && steps < 8 ? 1 : static_cast<int>(std::min({steps, each, int64_t{VerifyChoice::kMostParts}}));
            if (a.mask && b.choice_parts > 1) hipLaunchKernelGGL((verify_choice_kernel<F32, kFast, 512, true>), dim3(tokens, n, b.choice_parts), dim3(512), 0, st, b);
            else if (a.mask) hipLaunchKernelGGL((verify_choice_kernel<F32, kFast, 512>), dim3(tokens, n), dim3(512), 0, st, a);
            else hipLaunchKernelGGL((verify_choice_kernel<F32, kFast, kThreads>), dim3(tokens, n), block, 0, st, a);
        }
    }
    hipLaunchKernelGGL((verify_draw_kernel<F32>), dim3(static_cast<unsigned>(a.shape.groups), n), block, 0, st, a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

VerifyShape VerifyShape::of(const int64_t n, const int64_t total_q, const int32_t vocab) {
    const auto up = [](const int64_t x, const int64_t by) { return (x + by - 1) / by; };
    const auto least = [](const int64_t x, const int64_t y) { return x < y ? x : y; };
    VerifyShape s;
    // rows: workgroups for kRows of them together
    const int64_t steps = up(vocab, kStep), each = up(steps, least(least(kRows / (total_q > 0 ? total_q : 1) + 1, kMostPieces), steps));
    s.length = static_cast<int>(each * kStep);
    s.pieces = static_cast<int>(up(steps, each));
    // the draw: workgroups of 4 spans and more, 1024 of them together
    const int64_t thousands = up(vocab, kSpan);
    s.span_rounds = static_cast<int>(up(thousands, kMostSpans));
    s.spans = static_cast<int>(up(thousands, s.span_rounds));
    s.group_spans = static_cast<int>(up(up(s.spans, least(1024 / (n > 0 ? n : 1) + 1, up(s.spans, 4))), 4) * 4);
    s.groups = static_cast<int>(up(s.spans, s.group_spans));
    s.last_stride = s.spans < 2 ? 2 : s.spans;      // (two for a workgroup of verify_sums_kernel, which has four spans and more where there are several)
    return s;
}

int launch_draft_verify(const VerifyArgs& a, void* stream) {
    return a.f32 ? launch<true>(a, static_cast<hipStream_t>(stream)) : launch<false>(a, static_cast<hipStream_t>(stream));
}

}  // namespace pk
