// The paged cache's formats (packinfer.h): addresses, E4M3 codes with a power-of-two scale for each row.
#pragma once
#include "cache.h"
#include "common.hip.h"

namespace pk {
namespace {

// E8M0 byte of a row whose largest finite magnitude has these float bits: the smallest 2^E with largest <= 448 * 2^E, so that
// the bits alone decide: 448 = 1.75 * 2^8.  At least 2^-126, so that factors made of it are normal numbers.
__device__ __forceinline__ uint32_t scale_byte(const uint32_t largest) {
    const int e = static_cast<int>(largest >> 23) - 8 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return static_cast<uint32_t>(max(e, 1));
}
__device__ __forceinline__ float scale_value(const uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float scale_inverse(const uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// magnitude bits of a finite number, 0 of any other
__device__ __forceinline__ uint32_t finite_bits(const float x) {
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}
// What is not finite becomes a NaN: the format has no infinities.
__device__ __forceinline__ float finite_or_nan(const float x) {
    return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : x;
}
// two codes in the low half; |x * inv| <= 448
__device__ __forceinline__ uint32_t pack_f8x2(const float a, const float b, const float inv) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(a) * inv, finite_or_nan(b) * inv, 0, false) & 0xFFFFu;
}

// Index of column `col` of slot (block, off), head h, in K and in V; of the row's scales
__device__ __forceinline__ int64_t k_index(const CacheView& c, const int64_t block, const int off, const int h, const int col) {
    return ((block * c.Hkv + h) * c.page + off) * c.d + col;
}
__device__ __forceinline__ int64_t v_index(const CacheView& c, const int64_t block, const int off, const int h, const int col) {
    return ((block * c.Hkv + h) * c.page + (off & ~3)) * c.d + 4 * col + (off & 3);
}
__device__ __forceinline__ int64_t scale_index(const CacheView& c, const int64_t block, const int off, const int h, const int of_v) {
    return ((block * c.Hkv + h) * 2 + of_v) * c.page + off;
}

// Physical block of a logical page; entries that no pool has are clamped into it, as the re-layout does
__device__ __forceinline__ int64_t block_of(const CacheView& c, const int32_t* row, const int page) {
    const int64_t b = row[page];
    return b < 0 ? 0 : (b >= c.num_blocks ? c.num_blocks - 1 : b);
}

}  // namespace
}  // namespace pk
