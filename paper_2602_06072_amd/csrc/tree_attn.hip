// Attention of drafted tokens over the paged cache.
#include "cache_format.hip.h"

namespace pk {
namespace {

// One wave for a (drafted token, query head): 64 keys at a time, one for each lane, with running maximum and sum.
__global__ __launch_bounds__(64) void tree_attn_kernel(TreeArgs a) {
    __shared__ float qs[128], ps[64];
    const int i = blockIdx.z, h = blockIdx.y, lane = threadIdx.x;
    const CacheView& c = a.cache;
    const int d = c.d, kvh = h / (a.Hq / c.Hkv);
    const int64_t q0 = a.q_start[i], q1 = a.q_start[i + 1];
    const int drafts = static_cast<int>(q1 - q0), t = blockIdx.x;
    if (t >= drafts || q0 < 0 || q1 > a.total_q) return;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(a.kv_lens[i], 0)), static_cast<int64_t>(a.max_blocks) * c.page));
    const int ctx = a.kv_lens[i] - drafts;
    const uint64_t bits = a.mask ? a.mask[q0 + t] : ~uint64_t{0} >> (63 - t);
    const int32_t* table = a.block_table + static_cast<int64_t>(i) * a.max_blocks;
    for (int col = lane; col < d; col += 64)
        qs[col] = bf16_bits_to_float(static_cast<const uint16_t*>(a.q)[((q0 + t) * a.Hq + h) * d + col]) * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
    const auto value = [&](const void* p, int64_t at) {
        return c.f8 ? __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[at], 0) : bf16_bits_to_float(static_cast<const uint16_t*>(p)[at]);
    };
    for (int j0 = 0; j0 < len; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < len && (j < ctx || (j - ctx < 64 && (bits >> (j - ctx) & 1)));
        float x = -INFINITY;
        if (seen) {
            const int64_t block = block_of(c, table, j / c.page);
            const int off = j % c.page;
            float s = 0.f;
            for (int col = 0; col < d; ++col) s = fmaf(qs[col], value(c.k, k_index(c, block, off, kvh, col)), s);
            x = c.f8 ? s * scale_value(c.scales[scale_index(c, block, off, kvh, 0)]) : s;
        }
        float top = fmaxf(m, wave_max(x));
        if (top == -INFINITY) top = 0.f;
        const float p = seen ? expf(x - top) : 0.f, keep = expf(m - top);
        l = l * keep + wave_sum(p);
        m = fmaxf(m, wave_max(x));
        ps[lane] = p;
        __syncthreads();
        const uint64_t any = __ballot(seen);
        for (int u = 0; u < 2; ++u) {
            const int col = lane + 64 * u;
            o[u] *= keep;
            if (col >= d) continue;
            for (int y = 0; y < 64; ++y) {
                if (!(any >> y & 1)) continue;
                const int64_t block = block_of(c, table, (j0 + y) / c.page);
                const int off = (j0 + y) % c.page;
                const float v = value(c.v, v_index(c, block, off, kvh, col));
                o[u] = fmaf(ps[y], c.f8 ? v * scale_value(c.scales[scale_index(c, block, off, kvh, 1)]) : v, o[u]);
            }
        }
        __syncthreads();
    }
    for (int u = 0; u < 2; ++u) {
        const int col = lane + 64 * u;
        if (col >= d) continue;
        const float x = l > 0.f || l != l ? o[u] / l : 0.f;
        const int64_t at = ((q0 + t) * a.Hq + h) * d + col;
        if (a.out_f32) static_cast<float*>(a.out)[at] = x;
        else static_cast<uint16_t*>(a.out)[at] = float_to_bf16_bits(x);
    }
}

}  // namespace

int launch_tree_attn(const TreeArgs& a, void* stream) {
    const dim3 grid(static_cast<unsigned>(a.max_q), static_cast<unsigned>(a.Hq), static_cast<unsigned>(a.n));
    hipLaunchKernelGGL(tree_attn_kernel, grid, dim3(64), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace pk
