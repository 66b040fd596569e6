// Rows of a token: norm and rotation of queries and keys, and their way into the cache.
#include "cache_format.hip.h"

namespace pk {
namespace {

__device__ __forceinline__ float load_element(const void* p, const int64_t i, const int f32) {
    return f32 ? static_cast<const float*>(p)[i] : bf16_bits_to_float(static_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ void store_element(void* p, const int64_t i, const float x, const int f32) {
    if (f32) static_cast<float*>(p)[i] = x;
    else static_cast<uint16_t*>(p)[i] = float_to_bf16_bits(x);
}

// One wave for a row: y = x * rsqrt(mean(x^2) + eps) * w, then (a, b) -> (a cos - b sin, b cos + a sin) of every pair
__global__ __launch_bounds__(64) void token_rows_kernel(TokenRowsArgs a) {
    __shared__ float row[256];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x, d = a.d;
    int h = blockIdx.y;
    const int what = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;      // query, key, value
    h -= what == 0 ? 0 : what == 1 ? a.Hq : a.Hq + a.Hkv;
    const RowsView& in = what == 0 ? a.q : what == 1 ? a.k : a.v;
    const void* w = what == 0 ? a.q_weight : what == 1 ? a.k_weight : nullptr;
    float sum = 0.f;
    for (int c = lane; c < d; c += 64) {
        const float x = load_element(in.data, t * in.token_stride + h * in.head_stride + c, a.in_f32);
        row[c] = x;
        sum = fmaf(x, x, sum);
    }
    if (w) {
        const float inv = 1.f / sqrtf(wave_sum(sum) / d + a.eps);
        for (int c = lane; c < d; c += 64) row[c] = row[c] * inv * load_element(w, c, a.in_f32);
    }
    __syncthreads();
    if (what < 2 && a.table)
        for (int p = lane; p < a.pairs; p += 64) {
            int pos = a.positions[a.pair_axis[p] * a.axis_stride + t];
            pos = min(max(pos, 0), a.max_pos - 1);
            const float* cs = a.table + static_cast<int64_t>(pos) * 2 * a.pairs + p;
            const int i = a.interleaved ? 2 * p : p, j = a.interleaved ? 2 * p + 1 : p + a.pairs;
            const float x = row[i], y = row[j];
            row[i] = x * cs[0] - y * cs[a.pairs];
            row[j] = y * cs[0] + x * cs[a.pairs];
        }
    __syncthreads();
    if (what == 0 || a.k_out.data) {
        const RowsView& out = what == 0 ? a.q_out : a.k_out;
        for (int c = lane; c < d; c += 64) store_element(out.data, t * out.token_stride + h * out.head_stride + c, row[c], a.out_f32);
        return;
    }
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.cache.num_blocks * a.cache.page) return;
    const int64_t block = slot / a.cache.page;
    const int off = static_cast<int>(slot % a.cache.page);
    uint32_t largest = 0;
    for (int c = lane; c < d; c += 64) largest = max(largest, finite_bits(row[c]));
    for (int o = 32; o > 0; o >>= 1) largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), o, 64)));
    const uint32_t byte = scale_byte(largest);
    for (int c = lane; c < d; c += 64) {
        const int64_t i = what == 1 ? k_index(a.cache, block, off, h, c) : v_index(a.cache, block, off, h, c);
        void* dst = what == 1 ? a.cache.k : a.cache.v;
        if (a.cache.f8) static_cast<uint8_t*>(dst)[i] = static_cast<uint8_t>(pack_f8x2(row[c], 0.f, scale_inverse(byte)));
        else static_cast<uint16_t*>(dst)[i] = float_to_bf16_bits(row[c]);
    }
    if (a.cache.f8 && lane == 0) a.cache.scales[scale_index(a.cache, block, off, h, what - 1)] = static_cast<uint8_t>(byte);
}

// One workgroup for a token of a request
__global__ __launch_bounds__(64) void cache_read_kernel(CacheReadArgs a) {
    const int i = blockIdx.y, lane = threadIdx.x;
    const int64_t len = min(static_cast<int64_t>(a.kv_lens[i]), static_cast<int64_t>(a.max_blocks) * a.cache.page);
    const CacheView& c = a.cache;
    for (int64_t t = blockIdx.x; t < len; t += gridDim.x) {
        const int64_t out_row = a.row_start[i] + t;
        if (out_row < 0 || out_row >= a.rows) continue;
        const int64_t block = block_of(c, a.block_table + static_cast<int64_t>(i) * a.max_blocks, static_cast<int>(t / c.page));
        const int off = static_cast<int>(t % c.page);
        for (int e = lane; e < c.Hkv * c.d; e += 64) {
            const int h = e / c.d, col = e % c.d;
            const int64_t ki = k_index(c, block, off, h, col), vi = v_index(c, block, off, h, col);
            float k, v;
            if (c.f8) {
                const auto value = [](const void* p, int64_t at) { return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[at], 0); };
                k = value(c.k, ki) * scale_value(c.scales[scale_index(c, block, off, h, 0)]);
                v = value(c.v, vi) * scale_value(c.scales[scale_index(c, block, off, h, 1)]);
            } else {
                k = load_element(c.k, ki, 0);
                v = load_element(c.v, vi, 0);
            }
            store_element(a.k_out.data, out_row * a.k_out.token_stride + h * a.k_out.head_stride + col, k, a.out_f32);
            store_element(a.v_out.data, out_row * a.v_out.token_stride + h * a.v_out.head_stride + col, v, a.out_f32);
        }
    }
}

// One workgroup for a (request, KV head).  A lane moves the same columns of every kept row, first to last: what it overwrites are rows that it
// has moved already or that nobody keeps, since keep[j] >= j, and no other lane touches them.
template <class T>
__global__ __launch_bounds__(128) void cache_keep_kernel(CacheKeepArgs a) {
    const int i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const CacheView& c = a.cache;
    const int drafts = a.q_start[i + 1] - a.q_start[i];
    const int base = a.kv_lens[i] - drafts;
    const int count = min(max(min(a.keep_count[i], a.max_keep), 0), max(drafts, 0));
    if (h == 0 && lane == 0) a.new_lens[i] = base + count;
    const int32_t* row = a.block_table + static_cast<int64_t>(i) * a.max_blocks;
    const int end = static_cast<int>(min(static_cast<int64_t>(a.max_blocks) * c.page, static_cast<int64_t>(0x7FFFFFFF)));
    for (int j = 0; j < count; ++j) {
        const int from = a.keep[static_cast<int64_t>(i) * a.max_keep + j];
        if (from <= j || from >= drafts || base + j < 0 || base + from >= end) continue;      // in its place already, or no drafted token
        const int s = base + from, t = base + j;
        const int64_t sb = block_of(c, row, s / c.page), tb = block_of(c, row, t / c.page);
        if (lane < c.d) {
            static_cast<T*>(c.k)[k_index(c, tb, t % c.page, h, lane)] = static_cast<const T*>(c.k)[k_index(c, sb, s % c.page, h, lane)];
            static_cast<T*>(c.v)[v_index(c, tb, t % c.page, h, lane)] = static_cast<const T*>(c.v)[v_index(c, sb, s % c.page, h, lane)];
        }
        if (c.f8 && lane < 2) c.scales[scale_index(c, tb, t % c.page, h, lane)] = c.scales[scale_index(c, sb, s % c.page, h, lane)];
    }
}

}  // namespace

int launch_token_rows(const TokenRowsArgs& a, void* stream) {
    const unsigned heads = static_cast<unsigned>(a.Hq + (a.k_out.data ? 1 : 2) * a.Hkv);
    hipLaunchKernelGGL(token_rows_kernel, dim3(static_cast<unsigned>(a.tokens), heads), dim3(64), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

int launch_cache_read(const CacheReadArgs& a, void* stream) {
    hipLaunchKernelGGL(cache_read_kernel, dim3(1024, static_cast<unsigned>(a.n)), dim3(64), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

int launch_cache_keep(const CacheKeepArgs& a, void* stream) {
    const dim3 grid(static_cast<unsigned>(a.n), static_cast<unsigned>(a.cache.Hkv));
    if (a.cache.f8) hipLaunchKernelGGL(cache_keep_kernel<uint8_t>, grid, dim3(128), 0, static_cast<hipStream_t>(stream), a);
    else hipLaunchKernelGGL(cache_keep_kernel<uint16_t>, grid, dim3(128), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace pk
