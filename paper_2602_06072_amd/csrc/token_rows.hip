// Rows of a token on their way between the projections, the cache and the attention: norm and rotation of queries and keys, quantised
// writes, reads, and the moves of accepted tokens.  All of it is bound by memory (by latency in a decode step), one pass over the data.
//
// With x the row of a token's head: y = w x / sqrt(mean(x^2) + eps), pairs (a, b) of y turned to (a c - b s, b c + a s); into the cache as codes of E4M3 (nearest, ties to
// even) times 2^E, the smallest E >= -126 that holds the row's largest finite magnitude within 448.  Sums and products have 32 bits, those of cached keys 64.
// Measured (MI355X): 22011 tokens of 32 + 8 heads of 128 columns, bf16, 85 us, 5.4 TB/s; 44354 tokens of 8 heads of K and V into the cache in 8 bits 58 us, 4.8 TB/s (a large
// copy 4.8), 69 to 84 us right behind the read of the whole cache, from fp32 rows 101, into a bf16 cache 71; 307114 tokens of 8 heads read as bf16 rows 365 to 384 us, 5 TB/s, two
// thirds of it stores, as fp32 rows 687, from a bf16 cache 503; norm, rotation and write of 22011 tokens in one launch 140 us, 3.6 TB/s, of 1080 tokens in runs of 4 .. 12 15 to 17,
// where the bytes take 4: values outside of whole cells go one by one.  Stores past the caches take 72 instead of 85 us and cost the next reader of the rows as much and more
// (2048 tokens and a pass over them 18.5 and 19.4 us, 16384 103 and 112).
#include <type_traits>

#include "cache_format.hip.h"

namespace pk {
namespace {

constexpr int kWaves = 4;

// sum and maximum over aligned groups of LPR lanes (8, 16 or 32), in every lane of them
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(const uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
template <int CTRL, class T>
__device__ __forceinline__ T from_lane(const T x) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, dpp<CTRL>(__builtin_bit_cast(uint32_t, x)));
    else {
        const uint2 y = __builtin_bit_cast(uint2, x);
        return __builtin_bit_cast(T, make_uint2(dpp<CTRL>(y.x), dpp<CTRL>(y.y)));
    }
}
template <int LPR, class T, class Op>
__device__ __forceinline__ T over_row(T x, Op op) {
    x = op(x, from_lane<0xB1>(x));                  // quad_perm [1,0,3,2]
    x = op(x, from_lane<0x4E>(x));                  // quad_perm [2,3,0,1]
    x = op(x, from_lane<0x141>(x));                 // row_half_mirror: the other four of eight
    if constexpr (LPR >= 16) x = op(x, from_lane<0x140>(x));       // row_mirror: the other eight of sixteen
    if constexpr (LPR >= 32) x = op(x, __shfl_xor(x, 16, 64));
    return x;
}

// Eight columns of a row: four from column `a` on and four from `b` on
struct Eight { float a[4], b[4]; };
template <bool F32>
struct RawEight { std::conditional_t<F32, u32x4, uint2> a, b; };
template <bool F32, bool ADJACENT = false>
__device__ __forceinline__ RawEight<F32> load_eight(const void* p, const int64_t at, const int a, const int b) {
    using T = decltype(RawEight<F32>::a);
    if constexpr (ADJACENT && !F32) return __builtin_bit_cast(RawEight<F32>, *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at + a));
    if constexpr (F32) {
        const float* x = static_cast<const float*>(p) + at;
        return {*reinterpret_cast<const T*>(x + a), *reinterpret_cast<const T*>(x + b)};
    } else {
        const uint16_t* x = static_cast<const uint16_t*>(p) + at;
        return {*reinterpret_cast<const T*>(x + a), *reinterpret_cast<const T*>(x + b)};
    }
}
__device__ __forceinline__ float low_half(const uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_half(const uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
template <bool F32>
__device__ __forceinline__ Eight widened(const RawEight<F32>& r) {
    if constexpr (F32) return __builtin_bit_cast(Eight, r);
    else return {{low_half(r.a.x), high_half(r.a.x), low_half(r.a.y), high_half(r.a.y)}, {low_half(r.b.x), high_half(r.b.x), low_half(r.b.y), high_half(r.b.y)}};
}
template <bool F32>
__device__ __forceinline__ void store_eight(void* p, const int64_t at, const int a, const int b, const Eight& x) {
    if constexpr (F32) {
        float* o = static_cast<float*>(p) + at;
        *reinterpret_cast<floatx4*>(o + a) = floatx4{x.a[0], x.a[1], x.a[2], x.a[3]};
        *reinterpret_cast<floatx4*>(o + b) = floatx4{x.b[0], x.b[1], x.b[2], x.b[3]};
    } else {
        uint16_t* o = static_cast<uint16_t*>(p) + at;
        *reinterpret_cast<uint2*>(o + a) = make_uint2(pack_bf16x2(x.a[0], x.a[1]), pack_bf16x2(x.a[2], x.a[3]));
        *reinterpret_cast<uint2*>(o + b) = make_uint2(pack_bf16x2(x.b[0], x.b[1]), pack_bf16x2(x.b[2], x.b[3]));
    }
}

// permlane swaps: rows 16..31 of x with rows 0..15 of y (and 48..63 with 32..47); the upper half of x with the lower half of y
__device__ __forceinline__ void swap16(uint32_t& x, uint32_t& y) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = p[0]; y = p[1];
}
__device__ __forceinline__ void swap32(uint32_t& x, uint32_t& y) {
    const auto p = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = p[0]; y = p[1];
}

// x as a float that rounds to fewer bits as x itself does: toward zero, with an odd last bit where anything was cut off (an infinity where x is out of range)
__device__ __forceinline__ float odd_float(const double x) {
    const float f = static_cast<float>(x);
    const double back = f;
    uint32_t b = __float_as_uint(f);
    if (fabs(back) > fabs(x) && fabsf(f) < INFINITY) b -= 1;
    if (back != x && fabsf(f) < INFINITY) b |= 1;
    return __uint_as_float(b);
}
__device__ __forceinline__ float odd_float(const float x) { return x; }

// Norm and rotation of a lane's eight columns in T
template <class T, int LPR>
__device__ __forceinline__ void norm_and_turn(Eight& row, const bool normed, const Eight& w, const T by_d, const T eps, const bool rotated, const bool interleaved,
                                              const floatx4 cs, const floatx4 sn) {
    T y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { y[e] = row.a[e]; y[4 + e] = row.b[e]; }
    if (normed) {
        T sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fma(y[e], y[e], fma(y[4 + e], y[4 + e], sum));
        sum = over_row<LPR>(sum, [](const T p, const T q) { return p + q; });
        const T inv = T(1) / sqrt(fma(sum, by_d, eps));
#pragma unroll
        for (int e = 0; e < 4; ++e) { y[e] *= inv * w.a[e]; y[4 + e] *= inv * w.b[e]; }
    }
    if (rotated) {
        const auto turn = [&](const int i, const int j, const T c, const T n) {
            const T p = y[i], q = y[j];
            y[i] = fma(p, c, -q * n);
            y[j] = fma(q, c, p * n);
        };
        if (interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) turn(2 * e, 2 * e + 1, cs[e], sn[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) turn(e, 4 + e, cs[e], sn[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) { row.a[e] = odd_float(y[e]); row.b[e] = odd_float(y[4 + e]); }
}

enum Kind { kQuery, kKey, kCachedKey, kCachedCell, kCachedValue };       // (cell: values of four tokens that are interleaved)
struct Place { int64_t t, block; int off; bool ok; };                  // token, and where it goes in the cache
// What a launch does: rows to rows; queries to rows, keys and values into the cache; keys and values into the cache as they are
enum Mode { kRows, kProjected, kWrite };

// One wave for four consecutive tokens (two with LPR = 32), a head of theirs (two with LPR = 8) at a time: LPR lanes share a row, eight columns each.
// A pair's two columns are in one lane (halves: four columns of either half), so that the rotation needs no exchange, and the cosines and sines of a
// token are loaded once for all the heads that a wave takes.  Four tokens at once because the cache interleaves the values of four.
template <int LPR, bool IN_F32, bool OUT_F32, Mode MODE>
__global__ __launch_bounds__(64 * kWaves) void token_rows_kernel(TokenRowsArgs a) {
    constexpr int TOKENS = LPR == 32 ? 2 : 4, HEADS = LPR == 8 ? 2 : 1, BATCH = MODE == kWrite ? 8 : 4;
    constexpr bool CACHED = MODE != kRows;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x * kWaves + (threadIdx.x >> 6))), lane = threadIdx.x & 63;
    const int group = a.by_splits(wave), split = wave - group * a.splits;
    const int64_t t0 = static_cast<int64_t>(group) * TOKENS;
    if (t0 >= a.tokens) return;
    const int sub = lane / (64 / TOKENS), of = HEADS == 1 ? 0 : lane >> 3 & 1, x = lane % LPR;
    const bool token_ok = t0 + sub < a.tokens, columns_ok = 8 * x < a.d;
    const int64_t t = token_ok ? t0 + sub : a.tokens - 1;
    const int steps_q = (a.Hq + HEADS - 1) / HEADS, steps_k = (a.Hkv + HEADS - 1) / HEADS, steps = steps_q + (CACHED ? 2 : 1) * steps_k;
    const int first = static_cast<int>(static_cast<int64_t>(steps) * split / a.splits), last = static_cast<int>(static_cast<int64_t>(steps) * (split + 1) / a.splits);

    // columns of a row that is rotated, and of one that is not
    const bool rotated = x < a.pairs / 4;
    const int plain_a = columns_ok ? 8 * x : 0, plain_b = plain_a + 4;
    const int turn_a = rotated && !a.interleaved ? 4 * x : plain_a, turn_b = rotated && !a.interleaved ? 4 * x + a.pairs : plain_b;
    floatx4 cs = {1.f, 1.f, 1.f, 1.f}, sn = {0.f, 0.f, 0.f, 0.f};
    if (a.table && rotated && first < steps_q + steps_k) {
        const auto row = [&](const int axis) {
            const int pos = a.positions[axis * a.axis_stride + t];
            return a.table + static_cast<int64_t>(min(max(pos, 0), a.max_pos - 1)) * 2 * a.pairs + 4 * x;
        };
        if (a.axes_by_four) {                       // the four pairs of a lane have one axis
            const float* r = row(a.pair_axis[4 * x]);
            cs = *reinterpret_cast<const floatx4*>(r);
            sn = *reinterpret_cast<const floatx4*>(r + a.pairs);
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const float* r = row(a.pair_axis[4 * x + p]);
                cs[p] = r[p];
                sn[p] = r[a.pairs + p];
            }
        }
    }
    // Where the lane's token goes.  Values are interleaved by four: four tokens in a row that fill such a cell go there together, by the wave that has the first of
    // them, whichever tokens the wave has otherwise (prompts behind contexts of any length: 44354 tokens of 8 heads 89 -> 58 us); the others one by one.
    Place own{t, 0, 0, false}, cell{t, 0, 0, false};
    bool any_cell = false, any_single = false, single = false;
    if (CACHED && last > steps_q) {
        const int64_t places = a.cache.num_blocks * a.cache.page, near = t0 - 3 + (lane & 15);
        const int64_t slot = near >= 0 && near < a.tokens && (lane & 15) < 10 ? a.slots[near] : -1;          // of tokens t0 - 3 .. t0 + 6
        const bool inside = slot >= 0 && slot < places;
        const uint32_t begins = __ballot(inside && (slot & 3) == 0), follows = __ballot(__shfl_up(slot, 1, 16) + 1 == slot && (lane & 15) > 0 && inside);
        const uint32_t full = begins & follows >> 1 & follows >> 2 & follows >> 3 & 0x7F, covered = full | full << 1 | full << 2 | full << 3;
        const auto at = [&](Place& p, const int64_t s, const bool ok) {
            p.ok = ok;
            p.block = ok ? s / a.cache.page : 0;
            p.off = ok ? static_cast<int>(s - p.block * a.cache.page) : 0;
        };
        at(own, __shfl(slot, sub + 3, 16), token_ok && __shfl(static_cast<int>(inside), sub + 3, 16));
        single = own.ok && !(covered >> (sub + 3) & 1);
        any_single = __any(single);
        any_cell = (full & 0x78) != 0;
        const int start = any_cell ? __builtin_ctz(full & 0x78) : 3;
        at(cell, __shfl(slot, start, 16) + sub, any_cell);
        cell.t = any_cell ? t0 - 3 + start + sub : t;
    }

    const auto run = [&](auto what, const Place& to_place, const int from, const int to, const int heads, const RowsView& in, const RowsView& out, const void* weight) {
        constexpr Kind KIND = decltype(what)::value;
        constexpr bool turns = KIND < kCachedCell && MODE != kWrite;
        const int ca = turns ? turn_a : plain_a, cb = turns ? turn_b : plain_b;
        Eight w;
        const bool normed = turns && weight != nullptr;
        if (normed && from < to) w = widened<IN_F32>(load_eight<IN_F32>(weight, 0, ca, cb));
        for (int s0 = from; s0 < to; s0 += BATCH) {
            RawEight<IN_F32> raw[BATCH];
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                const int h = min(HEADS * min(s0 + s, to - 1) + of, heads - 1);
                raw[s] = load_eight<IN_F32, !turns>(in.data, to_place.t * in.token_stride + h * in.head_stride, ca, cb);
            }
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                if (s0 + s >= to) break;
                const int h = HEADS * (s0 + s) + of;
                const bool row_ok = columns_ok && h < heads;
                Eight y = widened<IN_F32>(raw[s]);
                if (!columns_ok) y = Eight{};
                // A key of the cache in 64 bits: it is stored with few bits, and one that lies by the middle between two of them goes to the nearer (in 32 bits
                // some three in a million go to the other, which 8 bits hold 6% apart).  A step of 128 requests takes 1 us of 170 for it.
                if (turns && KIND == kCachedKey) norm_and_turn<double, LPR>(y, normed, w, a.by_d, a.eps, rotated, a.interleaved, cs, sn);
                else if (turns) norm_and_turn<float, LPR>(y, normed, w, static_cast<float>(a.by_d), a.eps, rotated, a.interleaved, cs, sn);
                if constexpr (KIND == kQuery || KIND == kKey) {
                    if (row_ok && token_ok) store_eight<OUT_F32>(out.data, t * out.token_stride + h * out.head_stride, ca, cb, y);
                } else {
                    const bool cell_ok = row_ok && to_place.ok;
                    const int off = to_place.off;
                    const int64_t base = (to_place.block * a.cache.Hkv + h) * a.cache.page;
                    if (a.cache.f8) {
                        float top = 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(__uint_as_float(finite_bits(y.a[e])), __uint_as_float(finite_bits(y.b[e]))));
                        top = over_row<LPR>(top, [](float p, float q) { return fmaxf(p, q); });
                        const uint32_t byte = scale_byte(__float_as_uint(top));
                        const float inv = scale_inverse(byte);
                        uint32_t c0 = pack_f8x2(y.a[0], y.a[1], inv) | pack_f8x2(y.a[2], y.a[3], inv) << 16;
                        uint32_t c1 = pack_f8x2(y.b[0], y.b[1], inv) | pack_f8x2(y.b[2], y.b[3], inv) << 16;
                        if (cell_ok && x == 0) a.cache.scales[2 * base + (KIND == kCachedKey ? 0 : a.cache.page) + off] = static_cast<uint8_t>(byte);
                        if constexpr (KIND == kCachedKey) {
                            uint8_t* k = static_cast<uint8_t*>(a.cache.k) + (base + off) * a.d;
                            if (!turns && cell_ok) *reinterpret_cast<uint2*>(k + ca) = make_uint2(c0, c1);
                            if (turns && cell_ok) {
                                *reinterpret_cast<uint32_t*>(k + ca) = c0;
                                *reinterpret_cast<uint32_t*>(k + cb) = c1;
                            }
                        } else if constexpr (KIND == kCachedCell) {
                            // column pairs 0..3 of tokens 0..3 -> lane group s has pair s of all four tokens: 2 columns x 4 tokens, 8 bytes
                            swap32(c0, c1);                        // groups 0, 1: pairs 0, 1 of tokens s, s + 2; groups 2, 3: pairs 2, 3 of tokens s - 2, s
                            uint32_t even = __builtin_amdgcn_perm(c1, c0, 0x05040100u), odd = __builtin_amdgcn_perm(c1, c0, 0x07060302u);
                            swap16(even, odd);                     // pair s of tokens 0, 2 and of tokens 1, 3
                            const uint32_t lo = __builtin_amdgcn_perm(odd, even, 0x06020400u), hi = __builtin_amdgcn_perm(odd, even, 0x07030501u);
                            uint8_t* v = static_cast<uint8_t*>(a.cache.v) + (base + (off & ~3)) * a.d + 4 * (8 * x + 2 * sub);
                            if (cell_ok) *reinterpret_cast<uint2*>(v) = make_uint2(lo, hi);
                        } else if (cell_ok) {
                            uint8_t* v = static_cast<uint8_t*>(a.cache.v) + (base + (off & ~3)) * a.d + 4 * 8 * x + (off & 3);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                v[4 * e] = static_cast<uint8_t>(c0 >> 8 * e);
                                v[16 + 4 * e] = static_cast<uint8_t>(c1 >> 8 * e);
                            }
                        }
                    } else {
                        uint32_t p[4] = {pack_bf16x2(y.a[0], y.a[1]), pack_bf16x2(y.a[2], y.a[3]), pack_bf16x2(y.b[0], y.b[1]), pack_bf16x2(y.b[2], y.b[3])};
                        if constexpr (KIND == kCachedKey) {
                            uint16_t* k = static_cast<uint16_t*>(a.cache.k) + (base + off) * a.d;
                            if (!turns && cell_ok) *reinterpret_cast<u32x4*>(k + ca) = u32x4{p[0], p[1], p[2], p[3]};
                            if (turns && cell_ok) {
                                *reinterpret_cast<uint2*>(k + ca) = make_uint2(p[0], p[1]);
                                *reinterpret_cast<uint2*>(k + cb) = make_uint2(p[2], p[3]);
                            }
                        } else if constexpr (KIND == kCachedCell) {                        // the same with pairs of 32 bits: lane group s has pair s of tokens 0..3
                            swap32(p[0], p[2]);                    // groups 0, 1: pair 0 of tokens s, s + 2; groups 2, 3: pair 2 of tokens s - 2, s
                            swap32(p[1], p[3]);                    // pairs 1, 3
                            swap16(p[0], p[1]);                    // pair s of tokens 0, 1
                            swap16(p[2], p[3]);                    // of tokens 2, 3
                            uint16_t* v = static_cast<uint16_t*>(a.cache.v) + (base + (off & ~3)) * a.d + 4 * (8 * x + 2 * sub);
                            if (cell_ok)
                                *reinterpret_cast<u32x4*>(v) = u32x4{__builtin_amdgcn_perm(p[1], p[0], 0x05040100u), __builtin_amdgcn_perm(p[3], p[2], 0x05040100u),
                                                                     __builtin_amdgcn_perm(p[1], p[0], 0x07060302u), __builtin_amdgcn_perm(p[3], p[2], 0x07060302u)};
                        } else if (cell_ok) {
                            uint16_t* v = static_cast<uint16_t*>(a.cache.v) + (base + (off & ~3)) * a.d + 4 * 8 * x + (off & 3);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                v[8 * e] = static_cast<uint16_t>(p[e]);
                                v[8 * e + 4] = static_cast<uint16_t>(p[e] >> 16);
                            }
                        }
                    }
                }
            }
        }
    };
    if constexpr (MODE != kWrite) run(std::integral_constant<Kind, kQuery>{}, own, min(first, steps_q), min(last, steps_q), a.Hq, a.q, a.q_out, a.q_weight);
    const int k0 = steps_q, k1 = steps_q + steps_k;
    run(std::integral_constant<Kind, CACHED ? kCachedKey : kKey>{}, own, min(max(first, k0), k1) - k0, min(max(last, k0), k1) - k0, a.Hkv, a.k, a.k_out, a.k_weight);
    if constexpr (CACHED) {
        if (any_cell) run(std::integral_constant<Kind, kCachedCell>{}, cell, max(first, k1) - k1, max(last, k1) - k1, a.Hkv, a.v, a.k_out, nullptr);
        own.ok = single;
        if (any_single) run(std::integral_constant<Kind, kCachedValue>{}, own, max(first, k1) - k1, max(last, k1) - k1, a.Hkv, a.v, a.k_out, nullptr);
    }
}

// The request that unit `item` of the launch belongs to, and its number there, where request i has units(i) of them: prefix sums of them all,
// by every workgroup itself.  False: there are fewer.
template <class Units>
__device__ __forceinline__ bool find_unit(const int n, const int item, Units units, int& request, int& unit) {
    __shared__ int sums[kWaves], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (n + 64 * kWaves - 1) / (64 * kWaves), i0 = min(n, tid * each), i1 = min(n, i0 + each);
    int mine = 0;
    for (int i = i0; i < i1; ++i) mine += units(i);
    int before = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(before, o, 64);
        if (lane >= o) before += y;
    }
    if (lane == 63) sums[wave] = before;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    before -= mine;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) before += sums[w];
    if (item >= before && item < before + mine)
        for (int i = i0; i < i1; ++i) {
            const int k = units(i);
            if (item < before + k) { found[0] = i; found[1] = item - before; break; }
            before += k;
        }
    __syncthreads();
    request = __builtin_amdgcn_readfirstlane(found[0]);
    unit = __builtin_amdgcn_readfirstlane(found[1]);
    return request >= 0;
}

template <bool F32, int COUNT>
__device__ __forceinline__ void store_row(void* p, const int64_t at, const float* x) {
    if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < COUNT; e += 4) *reinterpret_cast<floatx4*>(static_cast<float*>(p) + at + e) = floatx4{x[e], x[e + 1], x[e + 2], x[e + 3]};
    } else if constexpr (COUNT % 8 == 0) {
#pragma unroll
        for (int e = 0; e < COUNT; e += 8)
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + at + e) = u32x4{pack_bf16x2(x[e], x[e + 1]), pack_bf16x2(x[e + 2], x[e + 3]), pack_bf16x2(x[e + 4], x[e + 5]), pack_bf16x2(x[e + 6], x[e + 7])};
    } else {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + at) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
}
__device__ __forceinline__ void widen_codes(const uint32_t x, const float scale, float* y) {
    y[0] = __builtin_amdgcn_cvt_f32_fp8(x, 0) * scale;
    y[1] = __builtin_amdgcn_cvt_f32_fp8(x, 1) * scale;
    y[2] = __builtin_amdgcn_cvt_f32_fp8(x, 2) * scale;
    y[3] = __builtin_amdgcn_cvt_f32_fp8(x, 3) * scale;
}

// One workgroup for 64 tokens of a request and some of the heads, one wave for 16 tokens, which lie in one page, a head at a time.  Bound by memory.  Lanes take
// columns so that the wave stores whole lines of the rows, 16 bytes a lane where a row has as many: K as it lies, V all four interleaved tokens of a few columns.
template <int D, bool F8, bool OUT_F32>
__global__ __launch_bounds__(64 * kWaves) void cache_read_kernel(CacheReadArgs a) {
    constexpr int SIZE = F8 ? 1 : 2, PER = OUT_F32 ? 4 : 8, LANES = D / PER, ROWS = 64 / LANES, KC = 16 / ROWS;          // K: columns of a lane, lanes and rows of a load, loads
    constexpr int COLS = OUT_F32 ? 4 : D / 16, GROUPS = D / 16 / COLS, VC = COLS * 4 * SIZE / 16;                        // V: columns in a row of a lane, how often, 16-byte chunks of each
    using KChunk = std::conditional_t<PER * SIZE == 16, u32x4, std::conditional_t<PER * SIZE == 8, uint2, uint32_t>>;
    const CacheView& c = a.cache;
    const int64_t most = static_cast<int64_t>(a.max_blocks) * c.page;
    const auto length = [&](const int i) {          // tokens that have a row
        const int64_t start = a.row_start[i];
        return start < 0 ? 0 : static_cast<int>(max(min(min(static_cast<int64_t>(a.kv_lens[i]), most), a.rows - start), int64_t{0}));
    };
    int i, unit;
    if (!find_unit(a.n, a.by_splits(static_cast<int>(blockIdx.x)), [&](const int y) { return (length(y) + 63) / 64; }, i, unit)) return;
    const int split = static_cast<int>(blockIdx.x) % a.splits, h0 = c.Hkv * split / a.splits, h1 = c.Hkv * (split + 1) / a.splits;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int len = length(i), t0 = unit * 64 + wave * 16;
    if (t0 >= len) return;
    const int page = t0 / c.page, off = t0 - page * c.page;
    const int64_t block = block_of(c, a.block_table + static_cast<int64_t>(i) * a.max_blocks, page);
    const int64_t row0 = static_cast<int64_t>(a.row_start[i]) + t0;
    const auto row_ok = [&](const int token) { return t0 + token < len; };
    const int g = lane >> 4, x = lane & 15;
#pragma unroll 2
    for (int h = h0; h < h1; ++h) {
        const int64_t base = (block * c.Hkv + h) * c.page, at = (base + off) * D * SIZE;
        KChunk k[KC];
        u32x4 v[GROUPS][VC];
        float ks[KC], vs[4];
#pragma unroll
        for (int y = 0; y < KC; ++y) k[y] = *reinterpret_cast<const KChunk*>(static_cast<const unsigned char*>(c.k) + at + static_cast<int>(sizeof(KChunk)) * (lane + 64 * y));
#pragma unroll
        for (int p = 0; p < GROUPS; ++p)
#pragma unroll
            for (int y = 0; y < VC; ++y) v[p][y] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(c.v) + at + g * 4 * D * SIZE + 16 * (VC * (16 * p + x) + y));
        if constexpr (F8) {
#pragma unroll
            for (int y = 0; y < KC; ++y) ks[y] = scale_value(c.scales[2 * base + off + y * ROWS + lane / LANES]);
            const uint32_t four = *reinterpret_cast<const uint32_t*>(c.scales + 2 * base + c.page + off + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) vs[e] = scale_value(four >> 8 * e & 0xFF);
        }
#pragma unroll
        for (int y = 0; y < KC; ++y) {
            uint32_t words[sizeof(KChunk) / 4];
            __builtin_memcpy(words, &k[y], sizeof(KChunk));
            float row[PER];
#pragma unroll
            for (int e = 0; e < static_cast<int>(sizeof(KChunk)) / 4; ++e) {
                if constexpr (F8) widen_codes(words[e], ks[y], row + 4 * e);
                else { row[2 * e] = low_half(words[e]); row[2 * e + 1] = high_half(words[e]); }
            }
            const int token = y * ROWS + lane / LANES;
            if (row_ok(token)) store_row<OUT_F32, PER>(a.k_out.data, (row0 + token) * a.k_out.token_stride + h * a.k_out.head_stride + lane % LANES * PER, row);
        }
#pragma unroll
        for (int p = 0; p < GROUPS; ++p) {
            float rows[4][COLS];
#pragma unroll
            for (int col = 0; col < COLS; ++col) {
                if constexpr (F8) {
                    float four[4];
                    widen_codes(v[p][col / 4][col % 4], 1.f, four);
#pragma unroll
                    for (int e = 0; e < 4; ++e) rows[e][col] = four[e] * vs[e];
                } else {
                    const uint32_t lo = v[p][col / 2][2 * (col % 2)], hi = v[p][col / 2][2 * (col % 2) + 1];
                    rows[0][col] = low_half(lo); rows[1][col] = high_half(lo); rows[2][col] = low_half(hi); rows[3][col] = high_half(hi);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row_ok(4 * g + e)) store_row<OUT_F32, COLS>(a.v_out.data, (row0 + 4 * g + e) * a.v_out.token_stride + h * a.v_out.head_stride + (16 * p + x) * COLS, rows[e]);
        }
    }
}

// One workgroup for a (request, KV head), a lane for a column.  Bound by latency: lengths and numbers, then pages, then the rows, each of them read for eight rows at
// a time.  All of them may be read before the first is stored, since keep rises: a kept row lies behind every place that an earlier one moves to.
template <class T>
__global__ __launch_bounds__(128) void cache_keep_kernel(CacheKeepArgs a) {
    constexpr int BATCH = 8;
    const int i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const CacheView& c = a.cache;
    // (64 bits: whatever the arrays hold, no sum leads past the table)
    const int64_t drafts = static_cast<int64_t>(a.q_start[i + 1]) - a.q_start[i], base = a.kv_lens[i] - drafts;
    const int count = static_cast<int>(min(static_cast<int64_t>(max(min(a.keep_count[i], a.max_keep), 0)), max(drafts, int64_t{0})));
    if (h == 0 && lane == 0) a.new_lens[i] = static_cast<int32_t>(base + count);
    const int32_t* row = a.block_table + static_cast<int64_t>(i) * a.max_blocks;
    const int32_t* keep = a.keep + static_cast<int64_t>(i) * a.max_keep;
    const int end = static_cast<int>(min(static_cast<int64_t>(a.max_blocks) * c.page, static_cast<int64_t>(0x7FFFFFFF)));
    if (end == 0 || lane >= c.d) return;
    T* k = static_cast<T*>(c.k);
    T* v = static_cast<T*>(c.v);
    for (int j0 = 0; j0 < count; j0 += BATCH) {
        bool moves[BATCH];
        int64_t from[BATCH], to[BATCH];             // physical block
        int from_off[BATCH], to_off[BATCH];
        T kept_k[BATCH], kept_v[BATCH];
        uint8_t scale[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int j = min(j0 + u, count - 1), f = keep[j];
            moves[u] = j0 + u < count && f > j && f < drafts && base + j >= 0 && base + f < end;     // not in its place already, and a drafted token
            const int s = moves[u] ? static_cast<int>(base + f) : 0, t = moves[u] ? static_cast<int>(base + j) : 0, sp = a.by_page(s), tp = a.by_page(t);
            from[u] = block_of(c, row, sp);
            to[u] = block_of(c, row, tp);
            from_off[u] = s - sp * c.page;
            to_off[u] = t - tp * c.page;
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            kept_k[u] = k[k_index(c, from[u], from_off[u], h, lane)];
            kept_v[u] = v[v_index(c, from[u], from_off[u], h, lane)];
            scale[u] = c.f8 && lane < 2 ? c.scales[scale_index(c, from[u], from_off[u], h, lane)] : 0;
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (!moves[u]) continue;
            k[k_index(c, to[u], to_off[u], h, lane)] = kept_k[u];
            v[v_index(c, to[u], to_off[u], h, lane)] = kept_v[u];
            if (c.f8 && lane < 2) c.scales[scale_index(c, to[u], to_off[u], h, lane)] = scale[u];
        }
    }
}

template <int LPR, Mode MODE>
void launch_rows(const TokenRowsArgs& a, const dim3 grid, hipStream_t st) {
    const dim3 block(64 * kWaves);
    constexpr bool F32 = MODE != kWrite;            // (a write has no rows to put out)
    if (a.in_f32 && a.out_f32) hipLaunchKernelGGL((token_rows_kernel<LPR, true, F32, MODE>), grid, block, 0, st, a);
    else if (a.in_f32) hipLaunchKernelGGL((token_rows_kernel<LPR, true, false, MODE>), grid, block, 0, st, a);
    else if (a.out_f32) hipLaunchKernelGGL((token_rows_kernel<LPR, false, F32, MODE>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((token_rows_kernel<LPR, false, false, MODE>), grid, block, 0, st, a);
}

template <int D, bool F8>
void launch_read(const CacheReadArgs& a, const dim3 grid, hipStream_t st) {
    if (a.out_f32) hipLaunchKernelGGL((cache_read_kernel<D, F8, true>), grid, dim3(64 * kWaves), 0, st, a);
    else hipLaunchKernelGGL((cache_read_kernel<D, F8, false>), grid, dim3(64 * kWaves), 0, st, a);
}

}  // namespace

int launch_token_rows(TokenRowsArgs a, void* stream) {
    const int lanes = a.d <= 64 ? 8 : a.d <= 128 ? 16 : 32, tokens = lanes == 32 ? 2 : 4, heads = lanes == 8 ? 2 : 1;
    const int64_t groups = (a.tokens + tokens - 1) / tokens;
    const int steps = (a.Hq + heads - 1) / heads + (a.k_out.data ? 1 : 2) * ((a.Hkv + heads - 1) / heads);
    // waves for a group of tokens: steps of eight heads, fewer where that leaves compute units without work.  Three waves of a kernel that writes the cache run on a SIMD at
    // a time, and one round of them is enough (3000 tokens of 8 heads into a bf16 cache and back 16.7 us, with 8192 waves 19.7; without a cache 8192 are up to 0.3 us ahead).
    const int64_t most = a.k_out.data ? 8192 : 3072, wanted = most / (groups < most ? groups : most), eighths = (steps + 7) / 8;
    const int64_t splits = wanted > eighths ? wanted : eighths;
    a.splits = static_cast<int>(splits < steps ? splits : steps);
    a.by_splits = FastDiv::by(static_cast<uint32_t>(a.splits));
    a.by_d = 1. / a.d;
    a.axes_by_four = 1;
    for (int p = 0; p < a.pairs; ++p)
        if (a.pair_axis[p] != a.pair_axis[p & ~3]) a.axes_by_four = 0;
    const int64_t workgroups = (groups * a.splits + kWaves - 1) / kWaves;
    if (workgroups * kWaves > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const dim3 grid(static_cast<unsigned>(workgroups));
    hipStream_t st = static_cast<hipStream_t>(stream);
    // a cache has rows of 64 or 128 columns
    const Mode mode = a.k_out.data ? kRows : a.Hq == 0 && !a.table && !a.k_weight ? kWrite : kProjected;
    if (lanes == 8) mode == kRows ? launch_rows<8, kRows>(a, grid, st) : mode == kWrite ? launch_rows<8, kWrite>(a, grid, st) : launch_rows<8, kProjected>(a, grid, st);
    else if (lanes == 16) mode == kRows ? launch_rows<16, kRows>(a, grid, st) : mode == kWrite ? launch_rows<16, kWrite>(a, grid, st) : launch_rows<16, kProjected>(a, grid, st);
    else launch_rows<32, kRows>(a, grid, st);
    return static_cast<int>(hipGetLastError());
}

int launch_cache_read(CacheReadArgs a, void* stream) {
    const int64_t units = a.rows / 64 + a.n;        // at most: requests have rows of their own
    // the heads of a unit over several workgroups where there are few units
    const int64_t splits = 2048 / (units < 2048 ? units : 2048);
    a.splits = static_cast<int>(splits < a.cache.Hkv ? splits : a.cache.Hkv);
    a.by_splits = FastDiv::by(static_cast<uint32_t>(a.splits));
    if (units * a.splits > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const dim3 grid(static_cast<unsigned>(units * a.splits));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.cache.d == 128) { if (a.cache.f8) launch_read<128, true>(a, grid, st); else launch_read<128, false>(a, grid, st); }
    else { if (a.cache.f8) launch_read<64, true>(a, grid, st); else launch_read<64, false>(a, grid, st); }
    return static_cast<int>(hipGetLastError());
}

int launch_cache_keep(CacheKeepArgs a, void* stream) {
    a.by_page = FastDiv::by(static_cast<uint32_t>(a.cache.page));
    const dim3 grid(static_cast<unsigned>(a.n), static_cast<unsigned>(a.cache.Hkv));
    if (a.cache.f8) hipLaunchKernelGGL(cache_keep_kernel<uint8_t>, grid, dim3(128), 0, static_cast<hipStream_t>(stream), a);
    else hipLaunchKernelGGL(cache_keep_kernel<uint16_t>, grid, dim3(128), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace pk
