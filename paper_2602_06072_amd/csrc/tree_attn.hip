// Attention of drafted tokens over the paged cache: launches of the kernels in tree_body.hip.h.
#include "tree_body.hip.h"

namespace pk {
namespace {

// Puts the pieces of a request together: one workgroup for (request, KV head, chunk, slice of its rows); nothing to do where there is one piece.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a) {
    int rest = blockIdx.x;
    const auto take = [&](const int of) { const int x = rest % of; rest /= of; return x; };
    const int slice = take(a.slices), kvh = take(a.cache.Hkv), chunk = take(a.chunks), i = rest;
    const int asked = a.q_start[i + 1] - a.q_start[i];
    const int64_t q0 = min(max(static_cast<int64_t>(a.q_start[i]), int64_t{0}), a.total_q);
    const int rows = static_cast<int>(min(static_cast<int64_t>(min(asked, a.max_q)), a.total_q - q0)) * a.heads_per_kv;
    const int here = min(rows - chunk * (1 << a.chunk_shift), (1 << a.chunk_shift));
    if (here <= 0) return;
    const int2 p = a.pieces_of[i];
    if (p.x == 1) return;
    const int chunks = (rows + (1 << a.chunk_shift) - 1) / (1 << a.chunk_shift);
    const auto part_row = [&](const int piece) { return (static_cast<int64_t>(p.y + piece * chunks + chunk) * a.cache.Hkv + kvh) * (1 << a.chunk_shift); };
    for (int x = slice * 256 + threadIdx.x; x < here * (D / 4); x += a.slices * 256) {
        const int local = x / (D / 4), col = 4 * (x % (D / 4)), row = chunk * (1 << a.chunk_shift) + local, t = a.by_r(row);
        store4(a, ((q0 + t) * a.Hq + kvh * a.heads_per_kv + row - t * a.heads_per_kv) * D + col, merged(p.x, [&](const int piece, float& lse, floatx4& o) {
            const int64_t at = part_row(piece) + local;
            lse = a.part_lse[at];
            o = *reinterpret_cast<const floatx4*>(a.part_o + at * D + col);
        }));
    }
}

template <int D, bool F8>
int launch(TreeArgs a, const TreeShape& s, hipStream_t st) {
    const dim3 block(64 * kWaves);
    const int row_blocks = s.rows / 16, keys = 16 * (row_blocks == 1 ? kSubTiles1<D, F8> : row_blocks == 2 ? kSubTiles2<D, F8> : 4);
    a.least_per_share = static_cast<float>(keys) / kLeastKeys;
    const int64_t loads = static_cast<int64_t>(a.n) * a.chunks, most_keys = static_cast<int64_t>(a.max_blocks) * a.cache.page;
    a.whole = most_keys <= kLeastKeys;              // no request can have two pieces: nothing to be found out, nothing to be put together
    a.least_per_many = a.least_per_share / (s.rows == 128 ? 4 : 1);        // (cut into more, the partial results of 128 rows are more bytes than the keys)
    // Short requests, and more of them than workgroups run at once: a wave for every request and 32 rows (300 requests of up to 17 tokens behind 60, 64 and 8 heads of 128
    // columns, 73 us and 142 by 128 rows; of up to 60, 272 and 344).  More than 32 rows of 64 columns in 8 bits stay with workgroups, which convert a tile once and not for
    // every 32 rows: over 71 launches (70 or 300 requests behind up to 4, 60 or 180 tokens, four head shapes) they take 0.99 of the waves' time in the mean, 0.79 where the
    // last 128 rows are more than 96, 1.09 where they are up to 32.  From bf16 nothing is converted, and they would take 1.25 of it.
    if (const int64_t units = static_cast<int64_t>(a.n) * a.cache.Hkv * s.alone_chunks; a.whole && (s.rows <= 32 || D == 128 || !F8) && loads > a.items && units <= 0x7FFFFFFF) {
        a.chunks = s.alone_chunks;
        a.chunk_shift = s.rows == 16 ? 4 : 5;
        a.by_chunks = FastDiv::by(static_cast<uint32_t>(a.chunks));
        const dim3 grid(static_cast<unsigned>((units + kWaves - 1) / kWaves));
        if (row_blocks == 1) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 1, kSubTiles1<D, F8>, 2, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, kSubTiles2<D, F8>, kWavesOf2<D, F8>, true>), grid, block, 0, st, a);
        return static_cast<int>(hipGetLastError());
    }
    // (workgroups without a piece take 3 us, two at a time on a unit: there are no more of them than half a round)
    const int64_t workgroups = (a.whole ? loads : loads <= a.items / 2 ? a.items : loads + a.items / 2) * a.cache.Hkv;
    if (workgroups > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const dim3 grid(static_cast<unsigned>(workgroups));
    if (row_blocks == 1) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 1, kSubTiles1<D, F8>, 2>), grid, block, 0, st, a);
    else if (row_blocks == 2) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, kSubTiles2<D, F8>, kWavesOf2<D, F8>>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tree_attn_wide_kernel<D, F8>), grid, block, 0, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || row_blocks == 1 || a.whole) return static_cast<int>(e);
    // the merge: up to 2048 workgroups, of 8 rows and more each
    const int64_t groups = loads * a.cache.Hkv, slices = 2048 / (groups < 2048 ? groups : 2048);
    a.slices = static_cast<int>(slices < s.rows / 8 ? slices : s.rows / 8);
    if (groups * a.slices > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    hipLaunchKernelGGL((tree_merge_kernel<D>), dim3(static_cast<unsigned>(groups * a.slices)), dim3(256), 0, st, a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

int launch_tree_attn(TreeArgs a, const TreeShape& s, void* stream) {
    set_tree_sizes(a, s);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.cache.d == 128) return a.cache.f8 ? launch<128, true>(a, s, st) : launch<128, false>(a, s, st);
    return a.cache.f8 ? launch<64, true>(a, s, st) : launch<64, false>(a, s, st);
}

}  // namespace pk
