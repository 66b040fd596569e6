// Attention of drafted tokens over the paged cache.
//
// A request's rows for a KV head are its drafted tokens times the query heads of that KV head (token-major).  The kernel works on the
// transposed problem with v_mfma_f32_16x16x32_bf16: S^T = K Q^T (A: 16 keys, B: 16 rows), O^T += V^T P^T (A: 16 columns, B: 16 rows), so
// that the scores of a row sit in four lanes and P^T leaves the first product as the operand of the second.  The cache is laid out for it:
// a lane's bytes of a K row are one token's (its scale goes in with the conversion to bf16, which is exact), and a dword of V is a column of
// the four keys whose scores the lane holds, so nothing goes through LDS on its way from memory to the matrix pipe.
#include "arrival.h"
#include "cache_format.hip.h"

#include <type_traits>

namespace pk {
namespace {

constexpr int kWaves = 4;
constexpr int kNonTemporalLoad = 2;                 // cache policy of a buffer load

__device__ __forceinline__ float max_of_lane_groups(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// What a workgroup works on: a piece of the tiles of a request.
struct Piece {
    int request, piece, pieces, slot;               // slot: of the request's first partial result
};

// Tiles of TOKENS keys that a request's rows have to visit (0: it has no rows), and pieces they are cut into.  A request with rows and no key
// has one piece, which writes zeros.
template <int TOKENS>
__device__ __forceinline__ int tiles_of(const TreeArgs& a, const int i) {
    const int64_t most = static_cast<int64_t>(a.max_blocks) * a.cache.page;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(a.kv_lens[i], 0)), most));
    return a.q_start[i + 1] > a.q_start[i] ? (len + TOKENS - 1) / TOKENS : -1;
}
__device__ __forceinline__ int pieces_of(const int tiles, const int share) { return tiles < 0 ? 0 : max(1, (tiles + share - 1) / share); }

// The piece number `item` of the launch, found from the lengths by every workgroup itself (no table to be made on the host, none to be
// copied when lengths change): tiles of all requests, the share of a piece that follows from them, prefix sums of pieces and slots.
template <int TOKENS>
__device__ __forceinline__ bool find_piece(const TreeArgs& a, const int item, Piece& out) {
    __shared__ int sums[3][kWaves];
    __shared__ Piece found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.n + 64 * kWaves - 1) / (64 * kWaves), i0 = min(a.n, tid * each), i1 = min(a.n, i0 + each);
    int total = 0;
    for (int i = i0; i < i1; ++i) total += max(0, tiles_of<TOKENS>(a, i));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    if (lane == 0) sums[0][wave] = total;
    if (tid == 0) found.pieces = 0;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sums[0][w];
    const int share = max(a.least_share, (total + a.items - 1) / a.items);
    int mine = 0, slots = 0;
    for (int i = i0; i < i1; ++i) {
        const int k = pieces_of(tiles_of<TOKENS>(a, i), share);
        mine += k;
        slots += k > 1 ? k : 0;
    }
    int before = mine, slots_before = slots;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(before, o, 64), y = __shfl_up(slots_before, o, 64);
        if (lane >= o) { before += x; slots_before += y; }
    }
    if (lane == 63) { sums[1][wave] = before; sums[2][wave] = slots_before; }
    __syncthreads();
    before -= mine;
    slots_before -= slots;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) { before += sums[1][w]; slots_before += sums[2][w]; }
    if (item >= before && item < before + mine) {
        for (int i = i0; i < i1; ++i) {
            const int k = pieces_of(tiles_of<TOKENS>(a, i), share);
            if (item < before + k) { found = {i, item - before, k, slots_before}; break; }
            before += k;
            slots_before += k > 1 ? k : 0;
        }
    }
    __syncthreads();
    out.request = __builtin_amdgcn_readfirstlane(found.request);
    out.piece = __builtin_amdgcn_readfirstlane(found.piece);
    out.pieces = __builtin_amdgcn_readfirstlane(found.pieces);
    out.slot = __builtin_amdgcn_readfirstlane(found.slot);
    return out.pieces > 0;
}

// K and V of a tile of N sub-tiles (16 keys each) as they are in memory
template <int D, bool F8, int N>
struct TileRegs {
    static constexpr int CH = F8 ? D / 64 : D / 32;  // 16-byte chunks of a lane in a sub-tile
    u32x4 k[N][CH], v[N][CH];
    uint32_t ks[N], vs[N];                          // scale byte of key 16u + lane % 16; of keys 16u + 4 (lane / 16) + 0..3
};

// 4 codes -> 4 bf16 values times `scale`
__device__ __forceinline__ uint2 widen(const uint32_t x, const float scale) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true)));
}
__device__ __forceinline__ bf16x8 operand(const uint2 a, const uint2 b) { return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y}); }

// Operands of the products.  K: columns of step s and lane group g; V: column of A row m in block t.
template <int D, bool F8> __device__ __forceinline__ constexpr int k_column(const int s, const int g) { return F8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g; }
template <int D, bool F8, int N>
__device__ __forceinline__ bf16x8 k_operand(const TileRegs<D, F8, N>& r, const int u, const int s) {
    if constexpr (F8) {
        const u32x4 x = r.k[u][s / 2];
        const float scale = scale_value(r.ks[u]);
        return s % 2 == 0 ? operand(widen(x[0], scale), widen(x[1], scale)) : operand(widen(x[2], scale), widen(x[3], scale));
    } else {
        return __builtin_bit_cast(bf16x8, r.k[u][s]);
    }
}
template <int D, bool F8, int N>
__device__ __forceinline__ bf16x8 v_operand(const TileRegs<D, F8, N>& r, const int b, const int t) {
    if constexpr (F8) {
        return operand(widen(r.v[2 * b][t / 4][t % 4], 1.f), widen(r.v[2 * b + 1][t / 4][t % 4], 1.f));
    } else {
        const u32x4 x = r.v[2 * b][t / 2], y = r.v[2 * b + 1][t / 2];
        return t % 2 == 0 ? __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]}) : __builtin_bit_cast(bf16x8, u32x4{x[2], x[3], y[2], y[3]});
    }
}

__device__ __forceinline__ void publish4(float* p, const floatx4 x) {
    uint64_t* q = reinterpret_cast<uint64_t*>(p);
    __hip_atomic_store(q, __builtin_bit_cast(uint64_t, floatx2{x[0], x[1]}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(q + 1, __builtin_bit_cast(uint64_t, floatx2{x[2], x[3]}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ floatx4 read_published4(const float* p) {
    const uint64_t* q = reinterpret_cast<const uint64_t*>(p);
    const floatx2 a = __builtin_bit_cast(floatx2, __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    const floatx2 b = __builtin_bit_cast(floatx2, __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    return floatx4{a[0], a[1], b[0], b[1]};
}
struct TreeCount {
    uint32_t* x;
    __device__ __forceinline__ uint32_t next(const uint32_t limit) const { return __builtin_amdgcn_atomic_inc32(x, limit, __ATOMIC_RELAXED, "agent"); }
};

__device__ __forceinline__ void store4(const TreeArgs& a, const int64_t at, const floatx4 x) {
    if (a.out_f32) *reinterpret_cast<floatx4*>(static_cast<float*>(a.out) + at) = x;
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}
// 1 / l; a row that saw nothing is zero, one whose sum is no number stays one
__device__ __forceinline__ float inverse_sum(const float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }

// What is no finite number in a word of V (four codes, or two bf16 numbers): all ones in its place
template <bool F8>
__device__ __forceinline__ uint32_t not_finite(const uint32_t x) {
    if constexpr (F8) return ((((x & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u) * 0xFFu;
    else return ((x & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

// Which of the keys key .. key + 3 a row sees, bit by bit: those of the context, of the drafted tokens those in its mask word, none from len on.
// Selects alone: with && and || this was a branch for each key.
__device__ __forceinline__ uint32_t seen_of_four(const uint64_t bits, const int key, const int ctx, const int len) {
    const int d = min(max(key - ctx, -4), 64);      // number of the first one among the drafted tokens
    const uint32_t context = (1u << max(-d, 0)) - 1, before = static_cast<uint32_t>(bits) << (-d & 31), behind = static_cast<uint32_t>(bits >> (d & 63));
    const uint32_t drafted = d < 0 ? before : d < 64 ? behind : 0u;
    return (context | drafted) & ((1u << min(max(len - key, 0), 4)) - 1);
}

// One workgroup for (piece, KV head, rows): ROWGROUPS of its four waves take 16 NB rows each, the waves of a row group take tiles of N sub-tiles
// in turns, two in flight for each.
template <int D, bool F8, int NB, int ROWGROUPS, int N, int WAVES_PER_SIMD>
__global__ __launch_bounds__(64 * kWaves, WAVES_PER_SIMD) void tree_attn_kernel(TreeArgs a) {
    using Regs = TileRegs<D, F8, N>;
    constexpr int CH = Regs::CH, TOKENS = 16 * N, KS = D / 32, VT = D / 16, SIZE = F8 ? 1 : 2;
    constexpr int SHARERS = kWaves / ROWGROUPS, ROWS = 16 * NB * ROWGROUPS, PITCH = D + 4;
    __shared__ __align__(16) float po[kWaves][16][PITCH];
    __shared__ float pm[kWaves][16], pl[kWaves][16];
    __shared__ int last;

    const CacheView& c = a.cache;
    const int kvh = blockIdx.x % c.Hkv, rest = blockIdx.x / c.Hkv, chunk = rest % a.chunks;
    Piece w;
    if (!find_piece<TOKENS>(a, rest / a.chunks, w)) return;
    const int i = w.request;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int rowgroup = wave / SHARERS, sharer = wave % SHARERS;

    const int64_t q0 = min(max(static_cast<int64_t>(a.q_start[i]), int64_t{0}), a.total_q);
    const int asked = a.q_start[i + 1] - a.q_start[i];
    const int rows = static_cast<int>(min(static_cast<int64_t>(min(asked, a.max_q)), a.total_q - q0)) * a.heads_per_kv, row0 = chunk * ROWS;
    if (row0 >= rows) return;                       // (all pieces of the request alike)
    const int len = static_cast<int>(min(static_cast<int64_t>(max(a.kv_lens[i], 0)), static_cast<int64_t>(a.max_blocks) * c.page));
    const int ctx = a.kv_lens[i] - asked;           // (negative: some drafted tokens have no place)
    const int tiles = (len + TOKENS - 1) / TOKENS;
    const int t0 = static_cast<int>(static_cast<int64_t>(tiles) * w.piece / w.pieces), t1 = static_cast<int>(static_cast<int64_t>(tiles) * (w.piece + 1) / w.pieces);
    const auto* table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(a.block_table + static_cast<int64_t>(i) * a.max_blocks));

    floatx4 o[NB][VT], l[NB];                       // sum of p v, relative to m; sum of p in every element
    float m[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        m[b] = -INFINITY; l[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < VT; ++t) o[b][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    const int first_row = row0 + rowgroup * 16 * NB;
    if (first_row < rows && t0 + sharer < t1) {
        const int last_sub = (len - 1) / 16;
        auto load = [&](Regs& r, const int tile) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int sub = min(tile * N + u, last_sub);
                const bool there = tile < t1 && tile * N + u <= last_sub;
                const int page = a.by_subs(sub), off = (sub - page * a.subs) * 16;
                const int block = min(max(static_cast<int>(table[page]), 0), static_cast<int>(c.num_blocks - 1));
                const int64_t at = (static_cast<int64_t>(block) * c.Hkv + kvh) * c.page;
                const auto resource = [&](const void* base, const int64_t byte, const int bytes) {
                    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(static_cast<const unsigned char*>(base) + byte), 0, there ? bytes : 0, 0x00020000);
                };
                const auto rk = resource(c.k, (at + off) * D * SIZE, 16 * D * SIZE), rv = resource(c.v, (at + off) * D * SIZE, 16 * D * SIZE);
#pragma unroll
                for (int x = 0; x < CH; ++x) r.k[u][x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, n * D * SIZE + 16 * g, 64 * x, kNonTemporalLoad));
#pragma unroll
                for (int x = 0; x < CH; ++x) r.v[u][x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, g * 4 * D * SIZE + 16 * n, 256 * x, kNonTemporalLoad));
                if constexpr (F8) {
                    const auto rs = resource(c.scales, 2 * at + off, c.page + 16);
                    r.ks[u] = __builtin_amdgcn_raw_buffer_load_b8(rs, n, 0, 0);
                    r.vs[u] = __builtin_amdgcn_raw_buffer_load_b32(rs, 4 * g, c.page, 0);
                }
            }
        };
        Regs r0, r1;
        load(r0, t0 + sharer);
        load(r1, t0 + sharer + SHARERS);

        // rows of this lane's columns; rows beyond the last repeat it and are not stored
        bf16x8 qf[NB][KS];
        uint64_t bits[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int row = min(first_row + 16 * b + n, rows - 1), t = a.by_r(row), h = row - t * a.heads_per_kv;
            const uint16_t* q = static_cast<const uint16_t*>(a.q) + ((q0 + t) * a.Hq + kvh * a.heads_per_kv + h) * D;
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[b][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + k_column<D, F8>(s, g)));
            bits[b] = a.mask ? a.mask[q0 + t] : ~uint64_t{0} >> (63 - t);
        }
        const float sl2 = a.scale * kLog2e;

        // `edge`: some key of the tile is not seen by some row
        auto step = [&](Regs& r, const int tile, auto edge) {
            constexpr bool EDGE = decltype(edge)::value;
            floatx4 s[NB][N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
#pragma unroll
                for (int b = 0; b < NB; ++b) s[b][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const bf16x8 x = k_operand<D, F8, N>(r, u, k);
#pragma unroll
                    for (int b = 0; b < NB; ++b) s[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, qf[b][k], s[b][u], 0, 0, 0);
                }
                if constexpr (F8) __builtin_amdgcn_sched_barrier(0);       // (bf16 copies of a sub-tile at a time: they are twice its size)
            }
            // lane (n, g) holds scores of its rows against keys TOKENS * tile + 16 u + 4 g + e
            const int key0 = tile * TOKENS + 4 * g;
            uint32_t hidden[NB];                                   // keys that this lane's row does not see, bit 4 u + e
            bool strange = false;                                  // V has something that is no finite number
            if constexpr (EDGE) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    uint32_t seen = 0;
#pragma unroll
                    for (int u = 0; u < N; ++u) seen |= seen_of_four(bits[b], key0 + 16 * u, ctx, len) << 4 * u;
                    hidden[b] = ~seen;
                }
                // A probability of zero does not hide what is no number: such values leave V here and come back below for the rows that see them.
                uint32_t any = 0;
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    if constexpr (F8) {                            // a scale where there is no key may be anything
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (key0 + 16 * u + e >= len) r.vs[u] = (r.vs[u] & ~(0xFFu << 8 * e)) | 127u << 8 * e;
                    }
#pragma unroll
                    for (int x = 0; x < CH; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const uint32_t odd = not_finite<F8>(r.v[u][x][y]);
                            r.v[u][x][y] &= ~odd;
                            any |= odd;
                        }
                }
                strange = __any(any != 0);
            }
            float factor[F8 ? N : 1][4];
            if constexpr (F8) {
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) factor[u][e] = scale_value(r.vs[u] >> 8 * e & 0xFF);
            }
            bf16x8 pf[NB][N / 2];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float raw[4 * N];
#pragma unroll
                for (int x = 0; x < 4 * N; ++x) raw[x] = !EDGE || !(hidden[b] >> x & 1) ? s[b][x / 4][x % 4] : -INFINITY;
                float mx = raw[0];
#pragma unroll
                for (int x = 1; x < 4 * N; ++x) mx = fmaxf(mx, raw[x]);
                const float m_new = fmaxf(m[b], max_of_lane_groups(mx) * sl2);
                const float m_use = m_new == -INFINITY ? 0.f : m_new;
                if (__any(m_new != m[b])) {
                    const float alpha = __builtin_amdgcn_exp2f(m[b] - m_use);
                    l[b] *= alpha;
#pragma unroll
                    for (int t = 0; t < VT; ++t) o[b][t] *= alpha;
                    m[b] = m_new;
                }
                uint32_t pw[2 * N];
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = __builtin_amdgcn_exp2f(fmaf(raw[4 * u + e], sl2, -m_use));
                        if constexpr (F8) p[e] *= factor[u][e];    // the scale of V, a power of two: it rounds nothing
                    }
                    pw[2 * u] = pack_bf16x2(p[0], p[1]);
                    pw[2 * u + 1] = pack_bf16x2(p[2], p[3]);
                }
#pragma unroll
                for (int x = 0; x < N / 2; ++x) pf[b][x] = __builtin_bit_cast(bf16x8, u32x4{pw[4 * x], pw[4 * x + 1], pw[4 * x + 2], pw[4 * x + 3]});
            }
#pragma unroll
            for (int x = 0; x < N / 2; ++x) {
                // sums of the ROUNDED probabilities (their error cancels in part) from the matrix pipe: every row of A holds the inverse scales
                u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
                if constexpr (F8) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t two = r.vs[2 * x + e / 2] >> 16 * (e % 2);
                        ones[e] = (254u - (two & 0xFF)) << 7 | (254u - (two >> 8 & 0xFF)) << 23;
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), pf[b][x], l[b], 0, 0, 0);
#pragma unroll
                for (int t = 0; t < VT; ++t) {
                    const bf16x8 v = v_operand<D, F8, N>(r, x, t);
#pragma unroll
                    for (int b = 0; b < NB; ++b) o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[b][x], o[b][t], 0, 0, 0);
                    if (F8 && t % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (EDGE) {
                if (strange) {                                     // how many such values of each kind a row sees in a column
                    load(r, tile);                                 // (it is gone from the registers)
                    Regs of_kind;
                    for (int kind = 0; kind < (F8 ? 1 : 3); ++kind) {
#pragma unroll
                        for (int u = 0; u < N; ++u)
#pragma unroll
                            for (int x = 0; x < CH; ++x)
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    const uint32_t v = r.v[u][x][y];
                                    if constexpr (F8) {
                                        of_kind.v[u][x][y] = ((((v & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u) * 0x38u;       // 0x38: one
                                    } else {
                                        const auto is = [&](const uint32_t half) { return kind == 0 ? (half & 0x7FFFu) > 0x7F80u : half == (kind == 1 ? 0x7F80u : 0xFF80u); };
                                        of_kind.v[u][x][y] = (is(v & 0xFFFFu) ? 0x3F80u : 0u) | (is(v >> 16) ? 0x3F800000u : 0u);
                                    }
                                }
                        const float value = kind == 0 ? __uint_as_float(0x7FC00000u) : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            bf16x8 seen[N / 2];
#pragma unroll
                            for (int x = 0; x < N / 2; ++x) {
                                u32x4 one;
#pragma unroll
                                for (int e = 0; e < 4; ++e) one[e] = (hidden[b] >> (8 * x + 2 * e) & 1 ? 0u : 0x3F80u) | (hidden[b] >> (8 * x + 2 * e + 1) & 1 ? 0u : 0x3F800000u);
                                seen[x] = __builtin_bit_cast(bf16x8, one);
                            }
#pragma unroll
                            for (int t = 0; t < VT; ++t) {
                                floatx4 count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int x = 0; x < N / 2; ++x) count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand<D, F8, N>(of_kind, x, t), seen[x], count, 0, 0, 0);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[b][t][e] += count[e] > 0.f ? value : 0.f;
                            }
                        }
                    }
                }
            }
        };
        // Tiles that every row sees whole, then the others (a tile or two of a request: the drafted tokens, the end), whose code needs the
        // registers of the second set.  Requests past the last tile have empty descriptors: behind a condition the compiler would wait for all of them.
        const int whole = min(max(min(ctx, len), 0) / TOKENS, t1);
        int tile = t0 + sharer;
        while (tile < whole) {
            step(r0, tile, std::false_type{});
            load(r0, tile + 2 * SHARERS);
            tile += SHARERS;
            if (tile >= whole) { r0 = r1; break; }
            step(r1, tile, std::false_type{});
            load(r1, tile + 2 * SHARERS);
            tile += SHARERS;
        }
        while (tile < t1) {
            step(r0, tile, std::true_type{});
            tile += SHARERS;
            load(r0, tile);
        }
    }

    const int64_t group = (static_cast<int64_t>(i) * c.Hkv + kvh) * a.chunks + chunk;
    const auto part_row = [&](const int piece) { return (static_cast<int64_t>(w.slot + piece) * c.Hkv + kvh) * a.chunks * ROWS + static_cast<int64_t>(chunk) * ROWS; };
    const auto out_at = [&](const int row, const int col) {
        const int t = a.by_r(row);
        return ((q0 + t) * a.Hq + kvh * a.heads_per_kv + row - t * a.heads_per_kv) * D + col;
    };
    const int rows_here = min(rows - row0, ROWS);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (b > 0) __syncthreads();
#pragma unroll
        for (int x = 0; x < CH; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (F8) *reinterpret_cast<floatx4*>(&po[wave][n][64 * x + 16 * g + 4 * e]) = floatx4{o[b][4 * x][e], o[b][4 * x + 1][e], o[b][4 * x + 2][e], o[b][4 * x + 3][e]};
                else *reinterpret_cast<floatx2*>(&po[wave][n][32 * x + 8 * g + 2 * e]) = floatx2{o[b][2 * x][e], o[b][2 * x + 1][e]};
            }
        if (g == 0) { pm[wave][n] = m[b]; pl[wave][n] = l[b][0]; }
        __syncthreads();
        for (int x = threadIdx.x; x < ROWGROUPS * 16 * (D / 4); x += 64 * kWaves) {
            const int of = x / (16 * (D / 4)), rn = x / (D / 4) % 16, col = 4 * (x % (D / 4)), local = (of * NB + b) * 16 + rn;
            if (local >= rows_here) continue;
            float top = pm[of * SHARERS][rn];
#pragma unroll
            for (int y = 1; y < SHARERS; ++y) top = fmaxf(top, pm[of * SHARERS + y][rn]);
            const float use = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < SHARERS; ++y) {
                const int from = of * SHARERS + y;
                const float f = __builtin_amdgcn_exp2f(pm[from][rn] - use);
                const floatx4 v = *reinterpret_cast<const floatx4*>(&po[from][rn][col]);
                sum = fmaf(f, pl[from][rn], sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, v[e], acc[e]);
            }
            acc *= inverse_sum(sum);
            if (w.pieces == 1) {
                store4(a, out_at(row0 + local, col), acc);
            } else {
                const int64_t at = part_row(w.piece) + local;
                publish4(a.part_o + at * D + col, acc);
                if (col == 0) __hip_atomic_store(a.part_lse + at, sum > 0.f || sum != sum ? top + __builtin_amdgcn_logf(sum) : -INFINITY, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
    }
    if (w.pieces == 1) return;
    // The workgroup that finishes last puts the pieces together, in their order whichever it is (decode_body.hip.h on the order of stores and counts).
    __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): this wave's partial results are in memory
    __syncthreads();
    if (threadIdx.x == 0) last = arrives_last(TreeCount{a.arrived + group}, static_cast<uint32_t>(w.pieces));
    __syncthreads();
    if (last == 0) return;
    constexpr int BATCH = 4;
    for (int x = threadIdx.x; x < rows_here * (D / 4); x += 64 * kWaves) {
        const int local = x / (D / 4), col = 4 * (x % (D / 4));
        float top = -INFINITY, sum = 0.f;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < w.pieces; p += BATCH) {
            float lse[BATCH];
            floatx4 v[BATCH];
#pragma unroll
            for (int y = 0; y < BATCH; ++y) {
                const int64_t at = part_row(min(p + y, w.pieces - 1)) + local;
                lse[y] = __hip_atomic_load(a.part_lse + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                v[y] = read_published4(a.part_o + at * D + col);
            }
            float top_new = top;
#pragma unroll
            for (int y = 0; y < BATCH; ++y) {
                if (p + y >= w.pieces) { lse[y] = -INFINITY; v[y] = floatx4{0.f, 0.f, 0.f, 0.f}; }
                top_new = fmaxf(top_new, lse[y]);
            }
            const float use = top_new == -INFINITY ? 0.f : top_new;
            const float alpha = __builtin_amdgcn_exp2f(top - use);
            sum *= alpha;
            acc *= alpha;
#pragma unroll
            for (int y = 0; y < BATCH; ++y) {
                const float f = __builtin_amdgcn_exp2f(lse[y] - use);
                sum += f;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, v[y][e], acc[e]);
            }
            top = top_new;
        }
        store4(a, out_at(row0 + local, col), acc * inverse_sum(sum));
    }
}

template <int D, bool F8>
int launch(const TreeArgs& a, const TreeShape& s, const dim3 grid, hipStream_t st) {
    const dim3 block(64 * kWaves);
    // sub-tiles in a tile: two tiles in flight, and with the accumulators of 16 or 32 rows within 256 registers (512 for 32 rows and d = 128 in bf16)
    constexpr int N1 = F8 ? 4 : 256 / D, N2 = F8 && D == 64 ? 4 : 2, W2 = F8 || D == 64 ? 2 : 1;
    if (s.row_blocks == 1) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 1, 1, N1, 2>), grid, block, 0, st, a);
    else if (s.row_groups == 1) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, 1, N2, W2>), grid, block, 0, st, a);
    else if (s.row_groups == 2) hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, 2, N2, W2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tree_attn_kernel<D, F8, 2, 4, N2, W2>), grid, block, 0, st, a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace

int launch_tree_attn(TreeArgs a, const TreeShape& s, void* stream) {
    a.heads_per_kv = a.Hq / a.cache.Hkv;
    a.by_r = FastDiv::by(static_cast<uint32_t>(a.heads_per_kv));
    a.subs = a.cache.page / 16;
    a.by_subs = FastDiv::by(static_cast<uint32_t>(a.subs));
    a.chunks = s.chunks;
    a.items = s.items;
    a.least_share = 4;
    const int64_t workgroups = (static_cast<int64_t>(a.items) + a.n) * a.chunks * a.cache.Hkv;
    if (workgroups > 0x7FFFFFFF) return static_cast<int>(hipErrorInvalidConfiguration);
    const dim3 grid(static_cast<unsigned>(workgroups));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.cache.d == 128) return a.cache.f8 ? launch<128, true>(a, s, grid, st) : launch<128, false>(a, s, grid, st);
    return a.cache.f8 ? launch<64, true>(a, s, grid, st) : launch<64, false>(a, s, grid, st);
}

}  // namespace pk
