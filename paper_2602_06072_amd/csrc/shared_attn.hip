// Attention of drafted tokens over the paged cache where requests have their leading pages in common.
//
// softmax(q K^T) V over the keys of a request is put together from two parts: the keys that its family shares, for the rows of all members at once, and its own ones behind
// them.  With o = sum p v / sum p and lse = log sum p of each part, the whole is sum exp(lse) o over sum exp(lse).
//
// Three launches.  The first finds what a family shares: the pages in which the members' rows of the block table are the same from the front on, less what is not wholly in
// front of every member's drafted tokens, in whole tiles of 64 keys.  So the result does not depend on what the families are, nothing is masked in the shared part, and
// there are no lengths to be handed over.  The second runs the kernels of pk_tree_attn, for a family's rows as one request's and, by workgroups of their own, for each
// request's keys from there on; the third joins their partial results.
//
// Shared keys are bound by the matrix pipe and the exponentials, as prefill is: they are read once for all members, 4 d operations a row and key.  Own keys are bound by
// memory, (2 d + 2) bytes each.  Measured, cache in 8 bits: 128 requests of one token behind 8200 shared ones, 16 .. 1024 of their own, 32 / 8 heads of 128 columns, 6 + 53 + 8 us
// (pk_tree_attn 303; one request with less in common takes the rest from all: 71 -> 273, and 79 with it in a family of its own); 16 families of 4 .. 12 trees, 64 / 8 heads, 6 + 256 + 26, where the operations
// take 143; bf16, two documents of 40000 .. 66000 tokens for 9 .. 16 requests of 64 columns 6 + 172 + 9, of 84 (what a score's exponential, maximum and rounding take does not halve with d, as its products do).
#include "shared_attn.h"
#include "tree_body.hip.h"

namespace pk {
namespace {

constexpr int kSharedTile = 64;                     // keys

__device__ __forceinline__ int load_there(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_there(int32_t* p, const int x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A wave for each request finds its family and how many tokens it has in common with the family's first request; one more workgroup finds where families begin, and the last
// one to finish what each of them shares.  Families are [M[g], M[g + 1]) with M the largest of family_start up to g, within [0, n]: disjoint whatever the array holds.
// Bound by loads one behind the other, of 0.6 us and more each: those that need not wait for others are asked for in front of them (128 requests 8.1 us when the last workgroup
// found where families begin, too).
__global__ __launch_bounds__(256) void shared_find_kernel(SharedArgs s) {
    constexpr int kNear = 1024;                     // families whose lengths the last workgroup has in LDS
    __shared__ int last, lds[4], len_near[kNear];
    const TreeArgs& a = s.tree;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = blockIdx.x * 4 + wave;
    if (blockIdx.x == gridDim.x - 1) {
        int carried = 0, carried_q = 0;             // M, and the largest row of q, so far
        for (int g0 = 0; g0 <= s.families; g0 += 256) {
            const int g = g0 + tid;
            const auto prefix_max = [&](int x, const int carried) {
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int y = __shfl_up(x, o, 64);
                    x = lane >= o ? max(x, y) : x;
                }
                __syncthreads();
                if (lane == 63) lds[wave] = x;
                __syncthreads();
                x = max(x, carried);
                for (int w = 0; w < wave; ++w) x = max(x, lds[w]);
                return x;
            };
            const int first = prefix_max(g <= s.families ? min(s.family_start[g], a.n) : 0, carried);
            carried = max(max(max(lds[0], lds[1]), max(lds[2], lds[3])), carried);
            const int q0 = prefix_max(g <= s.families ? static_cast<int>(min(static_cast<int64_t>(a.q_start[first]), a.total_q)) : 0, carried_q);
            carried_q = max(max(max(lds[0], lds[1]), max(lds[2], lds[3])), carried_q);
            if (g <= s.families) store_there(s.q_start_of + g, q0);
            if (g < s.families) s.first_of[g] = min(first, a.n - 1);
        }
    } else if (i < a.n) {
        const int asked = a.q_start[i + 1] - a.q_start[i], kv_len = a.kv_lens[i], len = min(max(kv_len, 0), a.most_keys);
        int first = 0, end = 0, family = -1, before = 0;
        for (int g0 = 0; g0 <= s.families; g0 += 64) {
            const int start = g0 + lane <= s.families ? s.family_start[g0 + lane] : -1;
            const uint64_t behind = __ballot(start > i);
            const int upto = behind ? __builtin_ctzll(behind) : 64;
            int most = lane < upto ? start : 0;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
            before = max(before, most);
            if (behind) {
                family = g0 + upto - 1;
                first = before;
                end = min(__shfl(start, upto, 64), a.n);
                break;
            }
        }
        const bool member = family >= 0 && end - first > 1;
        if (member && min(asked, a.max_q) > 0) {
            const int context = max(min(kv_len - asked, len), 0), pages = a.by_subs((context + 15) / 16 + a.subs - 1);
            const int32_t* mine = a.block_table + static_cast<int64_t>(i) * a.max_blocks;
            const int32_t* firsts = a.block_table + static_cast<int64_t>(first) * a.max_blocks;
            int same = i == first ? pages : 0;
            constexpr int AT_ONCE = 8;              // times 64 pages
            while (same < pages) {
                int32_t a_page[AT_ONCE], b_page[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int p = min(same + 64 * u + lane, pages - 1);
                    a_page[u] = mine[p];
                    b_page[u] = firsts[p];
                }
                int more = 64 * AT_ONCE;
#pragma unroll
                for (int u = AT_ONCE - 1; u >= 0; --u) {
                    const uint64_t differs = __ballot(same + 64 * u + lane < pages && a_page[u] != b_page[u]);
                    more = differs ? 64 * u + __builtin_ctzll(differs) : more;
                }
                same += more;
                if (more < 64 * AT_ONCE) break;
            }
            const int common = min(context, static_cast<int>(min(static_cast<int64_t>(same) * a.cache.page, static_cast<int64_t>(a.most_keys))));
            if (lane == 0) atomicMax(s.missing + family, a.most_keys - common + 1);
        }
        if (lane == 0) store_there(s.family_of + i, member ? family : -1);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): what this wave has found is in memory (decode_body.hip.h)
    __syncthreads();
    if (tid == 0) last = arrives_last(TreeCount{s.arrived}, gridDim.x);
    __syncthreads();
    if (last == 0) return;
    const int near_family = tid < a.n ? load_there(s.family_of + tid) : -1, near_len = tid < a.n ? a.kv_lens[tid] : 0;            // (asked for beside the families)
    float own = 0.f, shared = 0.f;                  // tiles of 64 keys, for every 128 rows of the shared ones
    for (int g = tid; g < s.families; g += 256) {
        const int missing = load_there(s.missing + g), rows = (load_there(s.q_start_of + g + 1) - load_there(s.q_start_of + g)) * a.heads_per_kv;
        const int tiles = missing == 0 ? 0 : (a.most_keys + 1 - missing) / kSharedTile;
        if (g < kNear) len_near[g] = tiles * kSharedTile;
        store_there(s.len_of + g, tiles * kSharedTile);
        if (missing != 0) store_there(s.missing + g, 0);
        shared += static_cast<float>(tiles) * static_cast<float>((rows + kWideRows - 1) / kWideRows);
    }
    if (s.families > kNear) __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    for (int r = tid; r < a.n; r += 256) {
        const int g = r < 256 ? near_family : load_there(s.family_of + r), len = min(max(r < 256 ? near_len : a.kv_lens[r], 0), a.most_keys);
        const int of_family = g < 0 ? 0 : g < kNear ? len_near[g] : load_there(s.len_of + g);
        s.shared_of[r] = of_family;
        own += static_cast<float>(len - min(of_family, len)) / kSharedTile;
    }
    const auto sum = [&](const float x) {
        const float y = last_lane(wave_prefix(x));
        __syncthreads();
        if (lane == 0) lds[wave] = __float_as_int(y);
        __syncthreads();
        return __int_as_float(lds[0]) + __int_as_float(lds[1]) + __int_as_float(lds[2]) + __int_as_float(lds[3]);
    };
    own = sum(own);
    shared = sum(shared);
    // Where there is much to be done for own keys, by workgroups that wait for memory, the shared ones are cut for half of the workgroups that run at once: both kinds
    // are on every unit then, and there are half as many partial results to be put together.
    if (tid == 0) *s.places = s.few_rows && own > 0.7f * shared ? max(s.at_once / 2, 1) : s.at_once;
}

// Shared keys and own ones in one launch, the shared ones, which take longer, first.  (A unit of the one kind and one of the other in turns: 429 us instead of 313 for
// families of drafted trees.)
struct BothArgs { TreeArgs own, shared; int own_units, shared_units; };
// WAVES: own keys by single waves, each with pieces of its own, for batches of many short requests: what a workgroup takes to find its piece, to begin and to put its four waves'
// results together is half of its time there (128 requests of 16 .. 1024 own tokens: 43 us by workgroups).
template <int D, bool F8, int ROW_BLOCKS, bool WAVES = false>
__global__ __launch_bounds__(64 * kWaves, D == 64 && ROW_BLOCKS == 3 ? 3 : 2) void shared_both_kernel(BothArgs b) {
    __shared__ __align__(16) unsigned char lds[kWideBytes<D>];
    __shared__ int last;
    const int Hkv = b.own.cache.Hkv, unit = b.own.by_hkv(blockIdx.x), head = static_cast<int>(blockIdx.x) - unit * Hkv;
    const bool of_shared = unit < b.shared_units;
    const int number = (of_shared ? unit : unit - b.shared_units) * Hkv + head;
    if (of_shared) many_rows<D, F8, kShared, 1>(lds, last, number, b.shared_units * Hkv);
    else if constexpr (ROW_BLOCKS == 1) few_rows<D, F8, 1, kSubTiles1<D, F8>, WAVES, kOwn, 0>(lds, last, number, b.own_units * Hkv);
    else if constexpr (ROW_BLOCKS == 2) few_rows<D, F8, 2, kSubTiles2<D, F8>, WAVES, kOwn, 0>(lds, last, number, b.own_units * Hkv);
    else many_rows<D, F8, kOwn, 0>(lds, last, number, b.own_units * Hkv);
}

// Puts the parts together: a workgroup for (request, chunk of its rows, slice of that, KV head).  KV heads go round-robin over the XCDs, as they do in the launches that
// write the parts.
template <int D>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs s) {
    const TreeArgs& a = s.tree;
    int rest = blockIdx.x;
    const auto take = [&](const int of) { const int x = rest % of; rest /= of; return x; };
    const int kvh = take(a.cache.Hkv), slice = take(a.slices), chunk = take(a.chunks), i = rest;
    // (asked for at once, also what is not needed)
    const int start = a.q_start[i], asked = a.q_start[i + 1] - start, of_family = a.shared_of[i], family = max(s.family_of[i], 0);
    const int2 p = a.pieces_of[i];
    const int2 pieces_of_family = s.pieces_of_family[family];
    const int family_start = s.q_start_of[family], family_end = s.q_start_of[family + 1];
    const int64_t q0 = min(max(static_cast<int64_t>(start), int64_t{0}), a.total_q);
    const int rows = static_cast<int>(min(static_cast<int64_t>(min(asked, a.max_q)), a.total_q - q0)) * a.heads_per_kv;
    const int chunk_rows = 1 << a.chunk_shift, here = min(rows - chunk * chunk_rows, chunk_rows);
    if (here <= 0) return;
    const bool shares = of_family > 0;
    if (!shares && p.x == 1) return;
    const int chunks = (rows + chunk_rows - 1) / chunk_rows;
    const int2 f = shares ? pieces_of_family : int2{0, 0};
    const int64_t family_q0 = shares ? family_start : 0;
    const int family_rows = shares ? (family_end - family_start) * a.heads_per_kv : 1;
    const int family_chunks = (family_rows + kWideRows - 1) / kWideRows;
    for (int x = slice * 256 + threadIdx.x; x < here * (D / 4); x += a.slices * 256) {
        const int local = x / (D / 4), col = 4 * (x % (D / 4)), row = chunk * chunk_rows + local, t = a.by_r(row);
        const int row_of_family = static_cast<int>(min(max((q0 - family_q0) * a.heads_per_kv + row, int64_t{0}), static_cast<int64_t>(family_rows - 1)));
        const auto part = [&](const int piece, float& lse, floatx4& o) {
            const bool own = piece < p.x;
            const int64_t at_own = (static_cast<int64_t>(p.y + piece * chunks + chunk) * a.cache.Hkv + kvh) * chunk_rows + local;
            const int64_t at_shared = (static_cast<int64_t>(f.y + (piece - p.x) * family_chunks + row_of_family / kWideRows) * a.cache.Hkv + kvh) * kWideRows + row_of_family % kWideRows;
            lse = own ? a.part_lse[at_own] : s.family_lse[at_shared];
            o = *reinterpret_cast<const floatx4*>(own ? a.part_o + at_own * D + col : s.family_o + at_shared * D + col);
        };
        const int pieces = p.x + f.x;               // (nearly always few, where there are many rows)
        store4(a, ((q0 + t) * a.Hq + kvh * a.heads_per_kv + row - t * a.heads_per_kv) * D + col,
               pieces <= 2 ? merged<2>(pieces, part) : pieces <= 4 ? merged<4>(pieces, part) : merged<8>(pieces, part));
    }
}

template <int D, bool F8>
int launch(SharedArgs s, const TreeShape& shape, hipStream_t st) {
    TreeArgs& a = s.tree;
    const dim3 block(64 * kWaves);
    s.few_rows = shape.rows <= 32;
    s.at_once = D == 64 && shape.rows > 32 ? a.items * 3 / 2 : a.items;            // (three workgroups on a unit)
    hipLaunchKernelGGL(shared_find_kernel, dim3(static_cast<unsigned>((a.n + 3) / 4 + 1)), dim3(256), 0, st, s);

    TreeArgs f = a;                                 // families as requests
    f.q_start = s.q_start_of; f.kv_lens = s.len_of; f.first_of = s.first_of; f.n = s.families;
    f.max_q = static_cast<int32_t>(a.total_q); f.mask = nullptr; f.places = s.places;
    f.chunk_shift = 7;
    f.rounds = 5 / 4.f;
    f.least_per_share = 64.f / kLeastKeys; f.least_per_many = f.least_per_share / 4;
    f.pieces_of = s.pieces_of_family; f.part_o = s.family_o; f.part_lse = s.family_lse;
    const int64_t family_loads = a.total_q * a.heads_per_kv / kWideRows + s.families;
    const int row_blocks = shape.rows / 16, keys = 16 * (row_blocks == 1 ? kSubTiles1<D, F8> : row_blocks == 2 ? kSubTiles2<D, F8> : 4);
    a.least_per_share = static_cast<float>(keys) / kLeastKeys;
    a.least_per_many = a.least_per_share / (shape.rows == 128 ? 4 : 1);
    a.shared_of = s.shared_of;
    const int64_t loads = static_cast<int64_t>(a.n) * a.chunks;
    const auto units_of = [](const int64_t loads, const int64_t items) { return loads <= items / 2 ? items : loads + items / 2; };
    const bool waves = row_blocks < 3 && kWavesOf2<D, F8> == 2 && loads > a.items * 3 / 4;         // (more requests than one round of workgroups holds)
    const int64_t shared_units = units_of(family_loads, s.at_once);
    if (waves) a.items *= kWaves;
    const int64_t own_units = waves ? (units_of(loads, a.items) + kWaves - 1) / kWaves : units_of(loads, a.items);
    if ((own_units + shared_units) * a.cache.Hkv > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const auto workgroups = [&](const int64_t units) { return dim3(static_cast<unsigned>(units * a.cache.Hkv)); };
    const BothArgs both{a, f, static_cast<int>(own_units), static_cast<int>(shared_units)};
    const dim3 grid = workgroups(own_units + shared_units);
    if (row_blocks == 1) {
        if (waves) hipLaunchKernelGGL((shared_both_kernel<D, F8, 1, true>), grid, block, 0, st, both);
        else hipLaunchKernelGGL((shared_both_kernel<D, F8, 1>), grid, block, 0, st, both);
    } else if (row_blocks > 2) {
        hipLaunchKernelGGL((shared_both_kernel<D, F8, 3>), grid, block, 0, st, both);
    } else if constexpr (kWavesOf2<D, F8> == 2) {
        if (waves) hipLaunchKernelGGL((shared_both_kernel<D, F8, 2, true>), grid, block, 0, st, both);
        else hipLaunchKernelGGL((shared_both_kernel<D, F8, 2>), grid, block, 0, st, both);
    } else {                                        // (32 rows of 128 columns in bf16 have twice the registers to a wave)
        hipLaunchKernelGGL((tree_attn_wide_kernel<D, F8, kShared>), workgroups(shared_units), block, 0, st, f);
        hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, kSubTiles2<D, F8>, kWavesOf2<D, F8>, false, kOwn>), workgroups(own_units), block, 0, st, a);
    }

    // the merge: up to 2048 workgroups, of 8 rows and more each
    const int64_t merges = loads * a.cache.Hkv, slices = 2048 / (merges < 2048 ? merges : 2048);
    a.slices = static_cast<int>(slices < shape.rows / 8 ? slices : shape.rows / 8);
    if (merges * a.slices > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    hipLaunchKernelGGL((shared_merge_kernel<D>), dim3(static_cast<unsigned>(merges * a.slices)), dim3(256), 0, st, s);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

int launch_shared_tree_attn(SharedArgs s, const TreeShape& shape, void* stream) {
    set_tree_sizes(s.tree, shape);
    s.tree.whole = 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (s.tree.cache.d == 128) return s.tree.cache.f8 ? launch<128, true>(s, shape, st) : launch<128, false>(s, shape, st);
    return s.tree.cache.f8 ? launch<64, true>(s, shape, st) : launch<64, false>(s, shape, st);
}

}  // namespace pk
