// Attention of drafted tokens over the paged cache.
//
// A request's rows for a KV head are its drafted tokens times the query heads of that KV head (token-major).  The kernel works on the
// transposed problem with v_mfma_f32_16x16x32_bf16: S^T = K Q^T (A: 16 keys, B: 16 rows), O^T += V^T P^T (A: 16 columns, B: 16 rows), so
// that the scores of a row sit in four lanes and P^T leaves the first product as the operand of the second.  The cache is laid out for it:
// a lane's bytes of a K row are one token's (its scale goes in with the conversion to bf16, which is exact), and a dword of V is a column of
// the four keys whose scores the lane holds, so that with few rows nothing goes through LDS on its way from memory to the matrix pipe.
//
// With u = rows and L = keys of a request a launch reads (2 d + 2) L bytes a KV head (4 d L from bf16) and computes 4 d u L operations: memory bounds it up to some
// 100 rows, the matrix pipe beyond.  Measured (MI355X, cache in 8 bits, 8 KV heads of 128 columns): 256 single tokens behind 32 .. 16384 tokens with 32 heads 353 us,
// 6.1 TB/s; 128 trees of 4 .. 12 tokens with 32 heads 145 to 153 us and 8 for the merge, where the bytes take 94; 64 trees of up to 64 tokens with 64 heads 630 to 674
// us, 0.70 to 0.75 PFLOP/s of the pairs that are seen (a product of large matrices reaches 1.34); from a bf16 cache 228 us with the merge, of 184, and 779.
//
// Roundings: K and V to bf16 are exact (4 bits of fraction and a power of two; below 2^-126 multiples of 2^-133); probabilities are rounded to bf16 for the matrix
// pipe, half a unit of 2^-8, whatever the type of the output, and their sum is that of the rounded ones; scores, sums, accumulators and partial results have 32 bits.
// The scales of V stay out of the probabilities: times 2^-126 a probability would be a denormal of a bit or none, and a row of zeros would lose its weight.
#pragma once
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

// Sums of the lanes up to each one; the last lane's in all of them
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T from_before(const T x) {      // of a lane before this one, or 0
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, ROWS == 0xF));
}
template <class T>
__device__ __forceinline__ T wave_prefix(T x) {
    x += from_before<0x111, 0xF>(x);                // row_shr 1, 2, 4, 8
    x += from_before<0x112, 0xF>(x);
    x += from_before<0x114, 0xF>(x);
    x += from_before<0x118, 0xF>(x);
    x += from_before<0x142, 0xA>(x);                // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    x += from_before<0x143, 0xC>(x);
    return x;
}
template <class T>
__device__ __forceinline__ T last_lane(const T x) { return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63)); }

// What a workgroup works on: a piece of the tiles of a request, for some of its rows (a chunk).
struct Piece {
    int request, piece, pieces, chunk, slot;        // slot: of the piece's partial result; those of a chunk's pieces are `chunks` apart
    int chunks;
    bool partial = false;                           // of one piece, and yet not the whole result
};

// The pieces of a launch follow from the lengths, and every wave finds its own from them: no table to be made on the host, none to be copied when lengths
// change.  All of it is on the way to the first load, and its instructions come from memory in every launch: no division by a variable, and few instructions
// (with integer divisions and eight candidates for the share 4.5 to 9 us, half of a short launch).
//
// Tiles of TOKENS keys that a request has, and chunks of rows that visit them (0: no rows).  A request with rows and no key has one piece, which writes zeros.
//
// A launch takes all keys of the requests (kAll), or, where some share pages, those behind the shared ones (kOwn) or those that a family shares, for the rows of
// all its members (kShared: a "request" is a family then; whole tiles, which all rows see).  Results of the latter two are partial.
enum Keys { kAll, kOwn, kShared };
template <Keys KEYS> struct Load {
    int tiles, chunks;
    __device__ __forceinline__ bool partial() const { return KEYS == kShared; }
};
template <> struct Load<kOwn> {
    int tiles, chunks, shared;
    __device__ __forceinline__ bool partial() const { return shared > 0; }
};
template <int TOKENS, Keys KEYS>
__device__ __forceinline__ Load<KEYS> load_of(const TreeArgs& a, const int i) {
    const int in = min(i, a.n - 1), q0 = a.q_start[in], q1 = a.q_start[in + 1], len = min(max(a.kv_lens[in], 0), a.most_keys);
    const int rows = i < a.n ? max(min(q1 - q0, a.max_q), 0) * a.heads_per_kv : 0;
    const int tiles = (len + TOKENS - 1) / TOKENS, chunks = (rows + (1 << a.chunk_shift) - 1) >> a.chunk_shift;
    if constexpr (KEYS == kOwn) return {max(tiles - a.shared_of[in] / TOKENS, 0), chunks, a.shared_of[in]};
    else if constexpr (KEYS == kShared) return {tiles, tiles > 0 ? chunks : 0};
    else return {tiles, chunks};
}
// Pieces of a request, of `share` tiles and fewer.  Which side a division falls to that just comes out does not matter: every wave of every launch has the same.
struct Shares {
    float per_share;                                // 1 / share
    int middle, last;                               // number of the first piece of the second and third kind; middle < 0: pieces in the order of requests
};
__device__ __forceinline__ int pieces_of(const int tiles, const float per_share) { return max(1, static_cast<int>(ceilf(static_cast<float>(tiles) * per_share))); }

// Where one round of workgroups may hold all pieces, the share is the smallest of three with which it does (a second, partly filled round takes as long as the
// first): a cut request has half a piece more than its tiles make, on average, and one more at most.  Otherwise a piece is a part of what a workgroup's place gets to
// do, and long pieces come first (of more than half of the share, of more than a quarter, the others), so that the launch ends with short ones.
__device__ __forceinline__ int kind_of(const int tiles, const float per_share) { return (2.f * tiles * per_share > 1.f ? 0 : 1) + (4.f * tiles * per_share > 1.f ? 0 : 1); }
// The first 64 KEPT requests are read once, all at a time, and kept; beside streaming workgroups every further read takes 2 us and more.
template <int KEPT, Keys KEYS> struct Loads { Load<KEYS> of[KEPT]; };
template <int TOKENS, int KEPT, Keys KEYS>
__device__ __forceinline__ Loads<KEPT, KEYS> read_loads(const TreeArgs& a) {
    Loads<KEPT, KEYS> l{};
#pragma unroll
    for (int u = 0; u < KEPT; ++u)
        if (64 * u < a.n) l.of[u] = load_of<TOKENS, KEYS>(a, 64 * u + static_cast<int>(threadIdx.x & 63));
    return l;
}
// each(first number, load of this lane's request) for 64 requests at a time, until it says that it is enough
template <int TOKENS, int KEPT, Keys KEYS, class Each>
__device__ __forceinline__ void for_loads(const TreeArgs& a, const Loads<KEPT, KEYS>& l, Each each) {
#pragma unroll
    for (int u = 0; u < KEPT; ++u)
        if (64 * u >= a.n || each(64 * u, l.of[u])) return;
    for (int i0 = 64 * KEPT; i0 < a.n; i0 += 64)
        if (each(i0, load_of<TOKENS, KEYS>(a, i0 + static_cast<int>(threadIdx.x & 63)))) return;
}
template <int TOKENS, int KEPT, Keys KEYS>
__device__ __forceinline__ Shares share_of(const TreeArgs& a, const Loads<KEPT, KEYS>& l) {
    float tiles = 0.f;                              // (of requests that share their pages there may be more than 2^31)
    int loads = 0;
    for_loads<TOKENS>(a, l, [&](int, const Load<KEYS> w) {
        tiles = fmaf(static_cast<float>(w.tiles), static_cast<float>(w.chunks), tiles);
        loads += w.chunks;
        return false;
    });
    tiles = fmaxf(last_lane(wave_prefix(tiles)), 1.f);
    loads = last_lane(wave_prefix(loads));
    const int at_once = KEYS == kShared ? *a.places : a.items;
    const float least = a.least_per_share, places = static_cast<float>(at_once), taken = static_cast<float>(loads);
    Shares s{0.f, -1, 0};
    const bool one_round = taken <= 0.75f * places;
    // the two shares to be looked at, or how many pieces are long and half as long
    s.per_share = one_round ? min(least, (places - 0.5f * taken) / tiles) : min(a.least_per_many, places * a.rounds / tiles);
    const float more = min(least, (places - 0.7f * taken) / tiles);
    int first = 0, second = 0;
    for_loads<TOKENS>(a, l, [&](int, const Load<KEYS> w) {
        const int k = w.chunks * pieces_of(w.tiles, s.per_share), kind = kind_of(w.tiles, s.per_share);
        first += one_round || kind == 0 ? k : 0;
        second += one_round ? w.chunks * pieces_of(w.tiles, more) : kind == 1 ? k : 0;
        return false;
    });
    first = last_lane(wave_prefix(first));
    second = last_lane(wave_prefix(second));
    if (one_round) {
        if (first > at_once) s.per_share = second <= at_once ? more : min(least, (places - taken) / tiles);
    } else {
        s.middle = first;
        s.last = first + second;
    }
    return s;
}
// Piece number `item` of a KV head; false: there are fewer
template <int TOKENS, int KEPT, Keys KEYS>
__device__ __forceinline__ bool find_piece(const TreeArgs& a, const Loads<KEPT, KEYS>& l, const int item, const Shares& s, Piece& out) {
    const int kind = s.middle < 0 ? -1 : item < s.middle ? 0 : item < s.last ? 1 : 2;
    int before = kind < 1 ? 0 : kind == 1 ? s.middle : s.last, slots = 0;          // (only requests of the first kind are cut)
    bool found = false;
    for_loads<TOKENS>(a, l, [&](const int i0, const Load<KEYS> w) {
        const int k = pieces_of(w.tiles, s.per_share), mine = kind >= 0 && kind_of(w.tiles, s.per_share) != kind ? 0 : k * w.chunks;
        const int upto = wave_prefix(mine), slots_upto = wave_prefix(k > 1 ? mine : 0);
        const uint64_t here = __ballot(item >= before + upto - mine && item < before + upto);
        if (here != 0) {
            const int from = __builtin_ctzll(here);
            const auto of = [&](const int x) { return __builtin_amdgcn_readlane(x, from); };
            const int local = item - before - of(upto - mine);
            out.request = i0 + from;
            out.pieces = of(k);
            out.chunks = of(w.chunks);
            out.piece = static_cast<int>((static_cast<float>(local) + 0.5f) / static_cast<float>(out.chunks));       // (the chunks of a piece one after the other)
            out.chunk = local - out.piece * out.chunks;
            out.slot = KEYS == kAll ? slots + of(slots_upto - (k > 1 ? mine : 0)) + local : item;      // (uncut requests have partial results too there)
            if constexpr (KEYS == kOwn) out.partial = of(w.shared) > 0;
            return found = true;
        }
        before += last_lane(upto);
        slots += last_lane(slots_upto);
        return false;
    });
    return found;
}

// The kernel's arguments, to be read anew: kept in registers over the loop of pieces they would leave too few scalar ones for the loop of tiles inside (trees of 64
// requests 674 -> 756 us)
// AT: which of several (a launch with the arguments of two kinds of work, each with workgroups of its own).
template <int AT = 0>
__device__ __forceinline__ const TreeArgs& kernel_args() {
    auto p = (const __attribute__((address_space(4))) TreeArgs*)__builtin_amdgcn_kernarg_segment_ptr() + AT;
    asm volatile("" : "+s"(p));
    return *(const TreeArgs*)p;
}

// Runs `work(arguments, piece, KV head)` for the workgroup's pieces: the one of its number and, where there are more pieces than workgroups, those as many numbers on.
// Workgroups go round-robin over the XCDs: with eight KV heads an XCD keeps to one, and the chunks of its rows find its keys in the L2.
// (`first`, `step`: the workgroup's first number and the distance to the next one)
// OF_WAVE: they are a wave's.
template <int TOKENS, int KEPT, Keys KEYS, int AT = 0, bool OF_WAVE = false, class Work>
__device__ __forceinline__ void run_pieces(Work work, const int first, const int step) {
    if (const TreeArgs& a = kernel_args<AT>(); KEYS == kAll && a.whole) {              // no request can have two pieces
        const int rest = a.by_hkv(blockIdx.x), i = a.by_chunks(rest);
        work(a, Piece{i, 0, 1, rest - i * a.chunks, 0, a.chunks}, static_cast<int>(blockIdx.x) - rest * a.cache.Hkv);
        return;
    }
    const Loads<KEPT, KEYS> loads = read_loads<TOKENS, KEPT, KEYS>(kernel_args<AT>());
    const Shares shares = share_of<TOKENS>(kernel_args<AT>(), loads);
    for (int item = first;; item += step) {
        const TreeArgs& a = kernel_args<AT>();
        Piece w;
        const int rest = a.by_hkv(item), kvh = item - rest * a.cache.Hkv;
        if (!find_piece<TOKENS>(a, loads, rest, shares, w)) return;
        work(a, w, kvh);
        if (shares.middle < 0) return;
        if constexpr (OF_WAVE) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        else __syncthreads();
    }
}

// K and V of a tile of N sub-tiles (16 keys each) as they are in memory
template <int D, bool F8, int N>
struct TileRegs {
    static constexpr int CH = F8 ? D / 64 : D / 32;  // 16-byte chunks of a lane in a sub-tile
    u32x4 k[N][CH], v[N][CH];
    uint32_t ks[N], vs[N];                          // scale bytes of keys 16u + n..n + 3, n = lane % 16 & 12 (a byte would be widened, and waited for, where it is loaded); 16u + 4 (lane / 16)..
};

// 4 codes -> 4 bf16 values times `scale`
__device__ __forceinline__ uint2 widen(const uint32_t x, const float scale) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true)));
}
// 4 codes of four tokens -> bf16 values times each one's scale
__device__ __forceinline__ uint2 widen_each(const uint32_t x, const float (&s)[4]) {
    const auto two = [&](auto high, const float p, const float q) {
        constexpr bool HIGH = decltype(high)::value;
        return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, q, HIGH)),
                                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, p, HIGH)), 0x07060100u);
    };
    return make_uint2(two(std::false_type{}, s[0], s[1]), two(std::true_type{}, s[2], s[3]));
}
__device__ __forceinline__ bf16x8 operand(const uint2 a, const uint2 b) { return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y}); }

// Operands of the products.  K: columns of step s and lane group g; V: column of A row m in block t.
template <int D, bool F8> __device__ __forceinline__ constexpr int k_column(const int s, const int g) { return F8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g; }
template <int D, bool F8, int N>
__device__ __forceinline__ bf16x8 k_operand(const TileRegs<D, F8, N>& r, const int u, const int s) {
    if constexpr (F8) {
        const u32x4 x = r.k[u][s / 2];
        const float scale = scale_value(r.ks[u] >> 8 * (threadIdx.x & 3) & 0xFF);
        return s % 2 == 0 ? operand(widen(x[0], scale), widen(x[1], scale)) : operand(widen(x[2], scale), widen(x[3], scale));
    } else {
        return __builtin_bit_cast(bf16x8, r.k[u][s]);
    }
}
// scales of the keys of V that a lane has
template <bool F8, int N> struct ValueScales { float of[F8 ? N : 1][4]; };
template <bool F8, int N>
__device__ __forceinline__ ValueScales<F8, N> value_scales(const uint32_t (&bytes)[N]) {
    ValueScales<F8, N> s;
    if constexpr (F8) {
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s.of[u][e] = scale_value(bytes[u] >> 8 * e & 0xFF);
    }
    return s;
}
template <int D, bool F8, int N>
__device__ __forceinline__ bf16x8 v_operand(const TileRegs<D, F8, N>& r, const ValueScales<F8, N>& s, const int b, const int t) {
    if constexpr (F8) {
        return operand(widen_each(r.v[2 * b][t / 4][t % 4], s.of[2 * b]), widen_each(r.v[2 * b + 1][t / 4][t % 4], s.of[2 * b + 1]));
    } else {
        const u32x4 x = r.v[2 * b][t / 2], y = r.v[2 * b + 1][t / 2];
        return t % 2 == 0 ? __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]}) : __builtin_bit_cast(bf16x8, u32x4{x[2], x[3], y[2], y[3]});
    }
}

// Partial results that another workgroup of the same launch reads are written through to memory, and read past what an L2 has of an earlier launch
// (decode_body.hip.h on the order of such stores and the count)
constexpr int kDeviceScope = 16;                    // cache policy of a buffer load: the scope bit that a relaxed atomic load at device scope has
__device__ __forceinline__ void store4(const TreeArgs& a, const int64_t at, const floatx4 x) {
    if (a.out_f32) *reinterpret_cast<floatx4*>(static_cast<float*>(a.out) + at) = x;
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}
// 1 / l; a row that saw nothing is zero, one whose sum is no number stays one
__device__ __forceinline__ float inverse_sum(const float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }

struct TreeCount {
    uint32_t* x;
    __device__ __forceinline__ uint32_t next(const uint32_t limit) const { return __builtin_amdgcn_atomic_inc32(x, limit, __ATOMIC_RELAXED, "agent"); }
};

// All ones in the place of the bf16 numbers of a word that are not finite: an exponent of ones and one more is the sign of a half, and that is spread
__device__ __forceinline__ uint32_t not_finite(const uint32_t x) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    const i16x2 y = __builtin_bit_cast(i16x2, (x & 0x7F807F80u) + 0x00800080u);
    return __builtin_bit_cast(uint32_t, y >> 15);
}

// Which of the keys key .. key + 3 a row sees, bit by bit: those of the context, of the drafted tokens those in its mask word, none from len on.
// Selects alone: with && and || this was a branch for each key.
__device__ __forceinline__ uint32_t seen_of_four(const uint64_t bits, const int key, const int ctx, const int len) {
    const int d = min(max(key - ctx, -4), 64);      // number of the first one among the drafted tokens
    const uint32_t context = (1u << max(-d, 0)) - 1, before = static_cast<uint32_t>(bits) << (-d & 31), behind = static_cast<uint32_t>(bits >> (d & 63));
    const uint32_t drafted = d < 0 ? before : d < 64 ? behind : 0u;
    return (context | drafted) & ((1u << min(max(len - key, 0), 4)) - 1);
}

// Where a workgroup's rows and keys are
struct Bounds {
    int64_t q0;                                     // first drafted token's row of q
    int rows, row0, rows_here;                      // rows of the request for a KV head; first one of the chunk, and how many
    int len, ctx, tiles, t0, t1;                    // keys; those in front of the drafted tokens (negative: some have no place); tiles, the piece's
    const int32_t* table;
};
template <int TOKENS, Keys KEYS = kAll>
__device__ __forceinline__ Bounds bounds_of(const TreeArgs& a, const Piece& w) {
    Bounds b;
    const int i = w.request, asked = a.q_start[i + 1] - a.q_start[i];
    b.q0 = min(max(static_cast<int64_t>(a.q_start[i]), int64_t{0}), a.total_q);
    b.rows = static_cast<int>(min(static_cast<int64_t>(min(asked, a.max_q)), a.total_q - b.q0)) * a.heads_per_kv;
    b.row0 = w.chunk << a.chunk_shift;
    b.rows_here = min(b.rows - b.row0, 1 << a.chunk_shift);
    b.len = min(max(a.kv_lens[i], 0), a.most_keys);
    b.ctx = KEYS == kShared ? b.len : a.kv_lens[i] - asked;
    b.tiles = (b.len + TOKENS - 1) / TOKENS;
    int first = 0;
    if constexpr (KEYS == kOwn) {                   // (pieces of the tiles behind the shared ones)
        first = min(a.shared_of[i] / TOKENS, b.tiles);
        b.tiles -= first;
    }
    // pieces of as many tiles but the last, which may have fewer (or none): the smallest number of which `pieces` are enough
    int each = b.tiles;
    if (w.pieces > 1) {
        each = static_cast<int>(static_cast<float>(b.tiles) / static_cast<float>(w.pieces));
        each += each * w.pieces < b.tiles ? 1 : 0;
        each += each * w.pieces < b.tiles ? 1 : 0;
    }
    b.t0 = min(w.piece * each, b.tiles);
    b.t1 = min(b.t0 + each, b.tiles);
    if constexpr (KEYS == kOwn) { b.t0 += first; b.t1 += first; b.tiles += first; }
    b.table = a.block_table + static_cast<int64_t>(KEYS == kShared ? a.first_of[i] : i) * a.max_blocks;
    return b;
}

// Where the sub-tiles of 16 keys (each in one page) of a tile are, a lane for each: first row of K and V, first byte of the scales.  Asked for a turn of
// the loop before the tile's own requests, and before those of a tile that is used earlier, so that nothing waits for it.
template <int N>
__device__ __forceinline__ int ask_places(const TreeArgs& a, const Bounds& b, const int tile, const int first) {
    const int sub = tile * N + first + static_cast<int>(threadIdx.x & 15);
    return b.table[a.by_subs(min(sub, (b.len - 1) / 16))];         // (the entry as it is)
}
struct SubTile {
    __amdgpu_buffer_rsrc_t k, v, s;                 // buffers of K, V and scales; empty past the end of the piece (zeros, no traffic)
};
// In lane u: row of K and V where sub-tile `first + u` of the tile begins (-1: past the end of the piece), and byte of its scales
struct Rows { int row; uint32_t scale; };
template <int N>
__device__ __forceinline__ Rows rows_of(const TreeArgs& a, const Bounds& b, const int kvh, const int tile, const int first, const int entry) {
    const CacheView& c = a.cache;
    const int sub = tile * N + first + static_cast<int>(threadIdx.x & 15), last = (b.len - 1) / 16, in = min(sub, last);
    const int block = min(max(entry, 0), static_cast<int>(c.num_blocks - 1)), off = (in - a.by_subs(in) * a.subs) * 16;
    const int row = (block * c.Hkv + kvh) * c.page + off;          // (a cache has fewer than 2^31 rows)
    return {tile < b.t1 && sub <= last ? row : -1, 2 * static_cast<uint32_t>(row) - static_cast<uint32_t>(off)};
}
template <int D, bool F8>
__device__ __forceinline__ SubTile sub_tile(const TreeArgs& a, const Rows& r, const int u) {
    constexpr int SIZE = F8 ? 1 : 2;
    const CacheView& c = a.cache;
    const int row = __builtin_amdgcn_readlane(r.row, u);
    const bool there = row >= 0;
    const auto resource = [&](const void* base, const uint64_t byte, const int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(static_cast<const unsigned char*>(base) + byte), 0, there ? bytes : 0, 0x00020000);
    };
    const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(there ? row : 0)) * (D * SIZE);
    SubTile t;
    t.k = resource(c.k, at, 16 * D * SIZE);
    t.v = resource(c.v, at, 16 * D * SIZE);
    if constexpr (F8) t.s = resource(c.scales, there ? static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(r.scale), u)) : 0u, c.page + 16);
    return t;
}
__device__ __forceinline__ u32x4 load16(const __amdgpu_buffer_rsrc_t r, const int lane, const int at) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane, at, kNonTemporalLoad));
}

// What a wave has of 16 NB rows: lane (n, g) holds columns of row 16 b + n
template <int D, int NB>
struct Sums {
    floatx4 o[NB][D / 16], l[NB];                   // sum of p v, relative to m; sum of p in every element
    float m[NB];                                    // maximum of the scores (exponents of two)
    __device__ __forceinline__ Sums() {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = -INFINITY; l[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < D / 16; ++t) o[b][t] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
    }
};
template <int D, int NB>
struct Queries {
    bf16x8 q[NB][D / 32];
    uint64_t bits[NB];
};
template <int D, bool F8, int NB, Keys KEYS = kAll>
__device__ __forceinline__ void load_queries(const TreeArgs& a, const Bounds& w, const int kvh, const int first_row, Queries<D, NB>& y) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < NB; ++b) {                  // rows beyond the last repeat it and are not stored
        const int row = min(first_row + 16 * b + n, w.rows - 1), t = a.by_r(row), h = row - t * a.heads_per_kv;
        const uint16_t* q = static_cast<const uint16_t*>(a.q) + ((w.q0 + t) * a.Hq + kvh * a.heads_per_kv + h) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) y.q[b][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + k_column<D, F8>(s, g)));
        if constexpr (KEYS != kShared) y.bits[b] = a.mask ? a.mask[w.q0 + t] : ~uint64_t{0} >> (63 - t);
    }
}

// Probabilities of 16 N keys against a row, from their raw scores.  `hidden`: bit x for key x that the row does not see (looked at with EDGE).
// LAZY: they are relative to m, which need not be the maximum: bf16 and fp32 hold 2^8 as well as 1, so what is summed up so far is brought to a new
// maximum only when a probability reaches that, and as long as m is -inf (a wave's first tile, scores of -inf).  A maximum across the lanes for
// every tile costs as much as the exponents' arithmetic.
constexpr float kMostProbability = 256.f;
template <int D, int N, bool EDGE, bool LAZY>
__device__ __forceinline__ void probabilities(const floatx4 (&s)[N], const uint32_t hidden, const float sl2, floatx4 (&o)[D / 16], floatx4& l, float& m, float (&p)[4 * N]) {
    const auto raw = [&](const int x) { return !EDGE || !(hidden >> x & 1) ? s[x / 4][x % 4] : -INFINITY; };
    if constexpr (LAZY && !EDGE) {
        float top = 0.f;
#pragma unroll
        for (int x = 0; x < 4 * N; ++x) {
            p[x] = __builtin_amdgcn_exp2f(fmaf(raw(x), sl2, -m));
            top = fmaxf(top, p[x]);
        }
        if (!__any(!(top < kMostProbability) || m == -INFINITY)) return;
    }
    float mx = raw(0);
#pragma unroll
    for (int x = 1; x < 4 * N; ++x) mx = fmaxf(mx, raw(x));
    const float m_new = fmaxf(m, max_of_lane_groups(mx) * sl2);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    if (LAZY || __any(m_new != m)) {
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        l *= alpha;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[t] *= alpha;
        m = m_new;
    }
#pragma unroll
    for (int x = 0; x < 4 * N; ++x) p[x] = __builtin_amdgcn_exp2f(fmaf(raw(x), sl2, -m_use));
}

// The product of a block of V columns with the probabilities of 32 keys, of which some rows do not see some: a probability of zero does not hide what is no
// finite number in V, so such values leave the operand and come back for the rows that see them (how many of each kind).
template <int NB, int D, int XN>
__device__ __forceinline__ void product_with_hidden(const bf16x8 v, const uint32_t (&hidden)[NB], const int x, const bf16x8 (&pf)[NB][XN], Sums<D, NB>& y, const int t) {
    const u32x4 words = __builtin_bit_cast(u32x4, v);
    u32x4 clean;
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t odd = not_finite(words[e]);
        clean[e] = words[e] & ~odd;
        any |= odd;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) y.o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, clean), pf[b][x], y.o[b][t], 0, 0, 0);
    if (!__any(any != 0)) return;
    for (int kind = 0; kind < 3; ++kind) {
        const auto is = [&](const uint32_t half) { return kind == 0 ? (half & 0x7FFFu) > 0x7F80u : half == (kind == 1 ? 0x7F80u : 0xFF80u); };
        u32x4 of_kind;
#pragma unroll
        for (int e = 0; e < 4; ++e) of_kind[e] = (is(words[e] & 0xFFFFu) ? 0x3F80u : 0u) | (is(words[e] >> 16) ? 0x3F800000u : 0u);
        const float value = kind == 0 ? __uint_as_float(0x7FC00000u) : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            u32x4 seen;
#pragma unroll
            for (int e = 0; e < 4; ++e) seen[e] = (hidden[b] >> (8 * x + 2 * e) & 1 ? 0u : 0x3F80u) | (hidden[b] >> (8 * x + 2 * e + 1) & 1 ? 0u : 0x3F800000u);
            const floatx4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, of_kind), __builtin_bit_cast(bf16x8, seen), floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) y.o[b][t][e] += count[e] > 0.f ? value : 0.f;
        }
    }
}

// Four columns of a row from the partial results of its pieces: sum of exp(lse) o over sum of exp(lse), eight pieces (BATCH) on their way at a time
template <int BATCH = 8, class Read>
__device__ __forceinline__ floatx4 merged(const int pieces, Read read) {
    float top = -INFINITY, sum = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; p += BATCH) {
        float lse[BATCH];
        floatx4 o[BATCH];
#pragma unroll
        for (int z = 0; z < BATCH; ++z) read(min(p + z, pieces - 1), lse[z], o[z]);
        float top_new = top;
#pragma unroll
        for (int z = 0; z < BATCH; ++z) {
            if (p + z >= pieces) { lse[z] = -INFINITY; o[z] = floatx4{0.f, 0.f, 0.f, 0.f}; }
            top_new = fmaxf(top_new, lse[z]);
        }
        const float use = top_new == -INFINITY ? 0.f : top_new;
        const float alpha = __builtin_amdgcn_exp2f(top - use);
        sum *= alpha;
        acc *= alpha;
#pragma unroll
        for (int z = 0; z < BATCH; ++z) {
            const float f = __builtin_amdgcn_exp2f(lse[z] - use);
            sum += f;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, o[z][e], acc[e]);
        }
        top = top_new;
    }
    return acc * inverse_sum(sum);
}

// Results of a workgroup: those of the `sharers` waves of a row group are put together in LDS and written; where the request has other pieces they are
// partial results.  HERE (few rows): the workgroup that finishes last puts those together, in their order whichever it is; otherwise a second launch does
// (tree_merge_kernel): reads past the caches take 2 us each, and one workgroup's worth of them 6 to 16 us for 32 to 128 rows.
template <int D> constexpr int kPitch = D + 4;
template <int D> constexpr int kJoinBytes = kWaves * 16 * (kPitch<D> + 2) * 4;
template <int D, bool F8, int NB, bool HERE, bool ALONE = false, Keys KEYS = kAll>
__device__ __forceinline__ void finish(const TreeArgs& a, const Piece& w, const Bounds& bounds, const int kvh, const int row_groups, const int sharers, const Sums<D, NB>& y, unsigned char* lds, int* last) {
    constexpr int CH = F8 ? D / 64 : D / 32, PITCH = kPitch<D>;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    float* po = reinterpret_cast<float*>(lds);      // [wave][16][PITCH]
    float* pm = po + kWaves * 16 * PITCH;           // [wave][16]
    float* pl = pm + kWaves * 16;
    const auto part_row = [&](const int piece) { return (static_cast<int64_t>(w.slot + (piece - w.piece) * w.chunks) * a.cache.Hkv + kvh) * (1 << a.chunk_shift); };
    const auto out_at = [&](const int local, const int col) {
        const int row = bounds.row0 + local, t = a.by_r(row);
        return ((bounds.q0 + t) * a.Hq + kvh * a.heads_per_kv + row - t * a.heads_per_kv) * D + col;
    };
    // (a wave alone: LDS works through the accesses of a wave in their order, the compiler alone must leave them in it)
    const auto sync = [] { if constexpr (ALONE) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); else __syncthreads(); };
    const int thread = ALONE ? lane : threadIdx.x, threads = ALONE ? 64 : 64 * kWaves, first_wave = ALONE ? wave : 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        sync();
        float* mine = po + (wave * 16 + n) * PITCH;
#pragma unroll
        for (int x = 0; x < CH; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (F8) *reinterpret_cast<floatx4*>(mine + 64 * x + 16 * g + 4 * e) = floatx4{y.o[b][4 * x][e], y.o[b][4 * x + 1][e], y.o[b][4 * x + 2][e], y.o[b][4 * x + 3][e]};
                else *reinterpret_cast<floatx2*>(mine + 32 * x + 8 * g + 2 * e) = floatx2{y.o[b][2 * x][e], y.o[b][2 * x + 1][e]};
            }
        if (g == 0) { pm[wave * 16 + n] = y.m[b]; pl[wave * 16 + n] = y.l[b][0]; }
        sync();
        for (int x = thread; x < row_groups * 16 * (D / 4); x += threads) {
            const int of = x / (16 * (D / 4)), rn = x / (D / 4) % 16, col = 4 * (x % (D / 4)), local = (of * NB + b) * 16 + rn;
            if (local >= bounds.rows_here) continue;
            const int from = (first_wave + of * sharers) * 16 + rn;
            float top = -INFINITY;
            for (int z = 0; z < sharers; ++z) top = fmaxf(top, pm[from + 16 * z]);
            const float use = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
            for (int z = 0; z < sharers; ++z) {
                const float f = __builtin_amdgcn_exp2f(pm[from + 16 * z] - use);
                const floatx4 v = *reinterpret_cast<const floatx4*>(po + (from + 16 * z) * PITCH + col);
                sum = fmaf(f, pl[from + 16 * z], sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, v[e], acc[e]);
            }
            acc *= inverse_sum(sum);
            if (KEYS == kAll ? w.pieces == 1 : KEYS == kOwn && w.pieces == 1 && !w.partial) {
                store4(a, out_at(local, col), acc);
            } else {
                const int64_t at = part_row(w.piece) + local;
                const float lse = sum > 0.f || sum != sum ? top + __builtin_amdgcn_logf(sum) : -INFINITY;
                if constexpr (HERE) {
                    write_through(a.part_o + at * D + col, __builtin_bit_cast(u32x4, acc));
                    if (col == 0) __hip_atomic_store(a.part_lse + at, lse, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                } else {
                    *reinterpret_cast<floatx4*>(a.part_o + at * D + col) = acc;
                    if (col == 0) a.part_lse[at] = lse;
                }
            }
        }
    }
    if constexpr (ALONE && KEYS == kAll) return;
    if constexpr (!HERE) {
        if (w.piece == 0 && w.chunk == 0 && kvh == 0 && thread == 0) a.pieces_of[w.request] = make_int2(w.pieces, w.slot);
        return;
    }
    if (w.pieces == 1) return;
    // (decode_body.hip.h on the order of the stores and the count)
    __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): this wave's partial results are in memory
    __syncthreads();
    if (threadIdx.x == 0) {
        const int64_t group = static_cast<int64_t>(w.slot - w.piece * w.chunks) * a.cache.Hkv + kvh;
        *last = arrives_last(TreeCount{a.arrived + group}, static_cast<uint32_t>(w.pieces));
    }
    __syncthreads();
    if (*last == 0) return;
    const int apart = w.chunks * a.cache.Hkv * (1 << a.chunk_shift);    // rows from a piece to the next
    const auto o_rows = __builtin_amdgcn_make_buffer_rsrc(a.part_o + part_row(0) * D, 0, 0x7FFFFFFF, 0x00020000);
    const auto lse_rows = __builtin_amdgcn_make_buffer_rsrc(a.part_lse + part_row(0), 0, 0x7FFFFFFF, 0x00020000);
    for (int x = threadIdx.x; x < bounds.rows_here * (D / 4); x += 64 * kWaves) {
        const int local = x / (D / 4), col = 4 * (x % (D / 4));
        store4(a, out_at(local, col), merged(w.pieces, [&](const int p, float& lse, floatx4& o) {
            const int at = p * apart + local;
            lse = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lse_rows, at * 4, 0, kDeviceScope));
            o = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(o_rows, (at * D + col) * 4, 0, kDeviceScope));
        }));
    }
}

// Up to 16 NB rows: bound by memory, in short launches by latency (four single tokens behind 300 .. 3000 tokens 11 us: the pieces found 2 to 3, first tile 1 to 3,
// tiles 2, last one 2, results and merge 2 to 4).  The four waves of a workgroup take tiles of N sub-tiles in turns, SETS tiles in flight in each, from memory into
// registers and from there into the products.  ALONE: every wave has a request (and rows) of its own, all of whose tiles it takes.
template <int D, bool F8, int NB, int N, bool ALONE, Keys KEYS, int AT>
__device__ __forceinline__ void few_rows(unsigned char* lds, int& last, const int first, const int step_of_items) {
    using Regs = TileRegs<D, F8, N>;
    constexpr int SETS = 2, CH = Regs::CH, TOKENS = 16 * N, KS = D / 32, VT = D / 16, SIZE = F8 ? 1 : 2, STRIDE = ALONE ? 1 : kWaves;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const auto work = [&](const TreeArgs& a, const Piece& w, const int kvh) {
        const Bounds bounds = bounds_of<TOKENS, KEYS>(a, w);
        if (bounds.rows_here <= 0) return;              // (no rows, or total_q says so; all pieces of the request alike)
        const int len = bounds.len, ctx = bounds.ctx, t1 = bounds.t1;

        Sums<D, NB> y;
        int tile = bounds.t0 + (ALONE ? 0 : wave);
        if (tile < t1) {
            // requests a tile, whose places are known, and the places of the set's tile after that
            auto load = [&](Regs& r, int& places, const int tile) {
                const Rows rows = rows_of<N>(a, bounds, kvh, tile, 0, places);
                places = ask_places<N>(a, bounds, tile + SETS * STRIDE, 0);
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const SubTile t = sub_tile<D, F8>(a, rows, u);
#pragma unroll
                    for (int x = 0; x < CH; ++x) r.k[u][x] = load16(t.k, n * D * SIZE + 16 * g, 64 * x);
#pragma unroll
                    for (int x = 0; x < CH; ++x) r.v[u][x] = load16(t.v, g * 4 * D * SIZE + 16 * n, 256 * x);
                    if constexpr (F8) {
                        r.ks[u] = __builtin_amdgcn_raw_buffer_load_b32(t.s, n & 12, 0, 0);
                        r.vs[u] = __builtin_amdgcn_raw_buffer_load_b32(t.s, 4 * g, a.cache.page, 0);
                    }
                }
            };
            Regs r[SETS];
            int places[SETS];
#pragma unroll
            for (int s = 0; s < SETS; ++s) places[s] = ask_places<N>(a, bounds, tile + s * STRIDE, 0);
            load(r[0], places[0], tile);
            Queries<D, NB> q;
            load_queries<D, F8, NB>(a, bounds, kvh, bounds.row0, q);
            // The rows are waited for here, with the first tile; left to the loop, its first products wait for all tiles in flight in every turn.
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 1; s < SETS; ++s) load(r[s], places[s], tile + s * STRIDE);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int OTHERS = (SETS - 1) * (N * (2 * CH + (F8 ? 2 : 0)) + 1);
            static_assert(OTHERS < 64, "vmcnt");
            __builtin_amdgcn_s_waitcnt(0x0F70 | (OTHERS & 0xF) | (OTHERS >> 4 << 14));
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
                        for (int b = 0; b < NB; ++b) s[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q.q[b][k], s[b][u], 0, 0, 0);
                    }
                    if constexpr (F8) __builtin_amdgcn_sched_barrier(0);       // (bf16 copies of a sub-tile at a time: they are twice its size)
                }
                // lane (n, g) holds scores of its rows against keys TOKENS * tile + 16 u + 4 g + e
                const int key0 = tile * TOKENS + 4 * g;
                uint32_t hidden[NB] = {};                              // keys that this lane's row does not see, bit 4 u + e
                if constexpr (EDGE) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        uint32_t seen = 0;
#pragma unroll
                        for (int u = 0; u < N; ++u) seen |= seen_of_four(q.bits[b], key0 + 16 * u, ctx, len) << 4 * u;
                        hidden[b] = ~seen;
                    }
                }
                bf16x8 pf[NB][N / 2];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float p[4 * N];
                    probabilities<D, N, EDGE, false>(s[b], hidden[b], sl2, y.o[b], y.l[b], y.m[b], p);
                    uint32_t pw[2 * N];
#pragma unroll
                    for (int x = 0; x < 2 * N; ++x) pw[x] = pack_bf16x2(p[2 * x], p[2 * x + 1]);
#pragma unroll
                    for (int x = 0; x < N / 2; ++x) pf[b][x] = __builtin_bit_cast(bf16x8, u32x4{pw[4 * x], pw[4 * x + 1], pw[4 * x + 2], pw[4 * x + 3]});
                }
                const ValueScales<F8, N> scales = value_scales<F8>(r.vs);
#pragma unroll
                for (int x = 0; x < N / 2; ++x) {
                    // sums of the ROUNDED probabilities (their error cancels in part) from the matrix pipe
                    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
#pragma unroll
                    for (int b = 0; b < NB; ++b) y.l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[b][x], y.l[b], 0, 0, 0);
#pragma unroll
                    for (int t = 0; t < VT; ++t) {
                        const bf16x8 v = v_operand<D, F8, N>(r, scales, x, t);
                        if constexpr (EDGE) product_with_hidden<NB, D, N / 2>(v, hidden, x, pf, y, t);
                        else {
#pragma unroll
                            for (int b = 0; b < NB; ++b) y.o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[b][x], y.o[b][t], 0, 0, 0);
                        }
                        if (F8 && t % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            // Tiles that every row sees whole, then the others (a tile or two of a request: the drafted tokens, the end), whose code needs the
            // registers of the second set.  Requests past the last tile have empty descriptors: behind a condition the compiler would wait for all of them.
            const int whole = min(max(min(ctx, len), 0) / TOKENS, t1);
            const auto turn = [&](Regs& x, int& at) {
                step(x, tile, std::false_type{});
                load(x, at, tile + SETS * STRIDE);
                tile += STRIDE;
            };
            // (the loop has one way out: from another in the middle the compiler would take the younger set for the one that it has to wait for)
            while (tile + STRIDE < whole) {
                turn(r[0], places[0]);
                turn(r[1], places[1]);
            }
            if (tile < whole) {
                turn(r[0], places[0]);
                r[0] = r[1];
            }
            while (tile < t1) {
                step(r[0], tile, std::true_type{});
                tile += STRIDE;
                places[0] = ask_places<N>(a, bounds, tile, 0);
                load(r[0], places[0], tile);
            }
        }
        finish<D, F8, NB, NB == 1 && KEYS == kAll, ALONE, KEYS>(a, w, bounds, kvh, 1, ALONE ? 1 : kWaves, y, lds, &last);
    };
    if constexpr (ALONE && KEYS != kAll) {
        run_pieces<TOKENS, 4, KEYS, AT, true>(work, first * kWaves + wave, step_of_items * kWaves);
    } else if constexpr (ALONE) {
        const TreeArgs& a = kernel_args();
        const int item = blockIdx.x * kWaves + wave, rest = a.by_hkv(item), i = a.by_chunks(rest);
        if (i < a.n) work(a, Piece{i, 0, 1, rest - i * a.chunks, 0, a.chunks}, item - rest * a.cache.Hkv);
    } else {
        run_pieces<TOKENS, 4, KEYS, AT>(work, first, step_of_items);
    }
}
template <int D, bool F8, int NB, int N, int WAVES_PER_SIMD, bool ALONE = false, Keys KEYS = kAll>
__global__ __launch_bounds__(64 * kWaves, WAVES_PER_SIMD) void tree_attn_kernel(TreeArgs) {
    __shared__ __align__(16) unsigned char lds[kJoinBytes<D>];
    __shared__ int last;
    few_rows<D, F8, NB, N, ALONE, KEYS, 0>(lds, last, blockIdx.x, gridDim.x);
}

// More rows, 128 in a workgroup: bound by the matrix pipe and what surrounds it (for 32 keys and 32 rows 34 MFMAs of 16 cycles, 16 exponentials of 16, some 60 other
// instructions of 4 and 16 KiB out of LDS, 128 cycles of the unit).  Four waves: with eight (64 KiB shared by twice the rows) 736 instead of 691 us, and operands read
// two, six or eight steps ahead instead of four 641 to 647 instead of 640.  The workgroup's waves bring a tile of 64 keys into LDS together, a
// quarter each, as bf16 operands (the conversion is done once, not by every wave), two tiles at a time; every wave reads it for its 32 rows.  With 64 rows
// and fewer two waves share 32 rows, half of a tile's keys each.
constexpr int kWideRows = 128;
template <int D> constexpr int kWideStage = 2 * 4 * (D / 32) * 1024;           // K and V of 64 keys as operands
template <int D> constexpr int kWideBytes = 2 * kWideStage<D> > kJoinBytes<D> ? 2 * kWideStage<D> : kJoinBytes<D>;
template <int D, bool F8, Keys KEYS, int AT>
__device__ __forceinline__ void many_rows(unsigned char* lds, int& last, const int first_item, const int step_of_items) {
    constexpr int NB = 2, N = 4, TOKENS = 64, KS = D / 32, VT = D / 16, CH = F8 ? D / 64 : D / 32, SIZE = F8 ? 1 : 2;
    constexpr int K_BYTES = N * KS * 1024, STAGE = kWideStage<D>;

    run_pieces<TOKENS, 2, KEYS, AT>([&](const TreeArgs& a, const Piece& w, const int kvh) {
        const Bounds bounds = bounds_of<TOKENS, KEYS>(a, w);
        if (bounds.rows_here <= 0) return;
        const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
        const int len = bounds.len, ctx = bounds.ctx, t0 = bounds.t0, t1 = bounds.t1;
        const int sharers = bounds.rows_here <= 64 ? 2 : 1, row_group = wave / sharers, half = wave % sharers;
        const bool works = row_group * 32 < bounds.rows_here;

        Sums<D, NB> y;
        if (t0 < t1) {
            // this wave's quarter of a tile: K or V of two sub-tiles
            struct Quarter { u32x4 c[2][CH]; uint32_t s[2]; };
            const int of_v = wave & 1, pair = wave >> 1;
            const int lane_at = of_v ? g * 4 * D * SIZE + 16 * n : n * D * SIZE + 16 * g, chunk_at = of_v ? 256 : 64;
            const int scale_lane = of_v ? 4 * g : n & 12, scale_at = of_v ? a.cache.page : 0;
            auto load = [&](Quarter& r, int& places, const int tile) {
                const Rows rows = rows_of<N>(a, bounds, kvh, tile, 2 * pair, places);
                places = ask_places<N>(a, bounds, tile + 2, 2 * pair);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const SubTile t = sub_tile<D, F8>(a, rows, u);
#pragma unroll
                    for (int x = 0; x < CH; ++x) r.c[u][x] = load16(of_v ? t.v : t.k, lane_at, chunk_at * x);
                    if constexpr (F8) r.s[u] = __builtin_amdgcn_raw_buffer_load_b32(t.s, scale_lane, scale_at, 0);
                }
            };
            const int whole = min(max(min(ctx, len), 0) / TOKENS, t1);
            auto put = [&](const Quarter& r, const int stage) {
                unsigned char* to = lds + stage * STAGE + of_v * K_BYTES + 16 * lane;
                TileRegs<D, F8, 2> x;
                if (!of_v) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
#pragma unroll
                        for (int z = 0; z < CH; ++z) x.k[u][z] = r.c[u][z];
                        x.ks[u] = r.s[u];
#pragma unroll
                        for (int s = 0; s < KS; ++s) *reinterpret_cast<bf16x8*>(to + ((2 * pair + u) * KS + s) * 1024) = k_operand<D, F8, 2>(x, u, s);
                    }
                    return;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
#pragma unroll
                    for (int z = 0; z < CH; ++z) x.v[u][z] = r.c[u][z];
                }
                const ValueScales<F8, 2> scales = value_scales<F8>(r.s);
#pragma unroll
                for (int t = 0; t < VT; ++t) *reinterpret_cast<bf16x8*>(to + (pair * VT + t) * 1024) = v_operand<D, F8, 2>(x, scales, 0, t);
            };
            Quarter r0, r1;
            int p0 = ask_places<N>(a, bounds, t0, 2 * pair), p1 = ask_places<N>(a, bounds, t0 + 1, 2 * pair);
            load(r0, p0, t0);
            Queries<D, NB> q;
            load_queries<D, F8, NB, KEYS>(a, bounds, kvh, bounds.row0 + (works ? row_group * 32 : 0), q);
            __builtin_amdgcn_sched_barrier(0);
            load(r1, p1, t0 + 1);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int SECOND = 2 * (CH + (F8 ? 1 : 0)) + 1;
            __builtin_amdgcn_s_waitcnt(0x0F70 | (SECOND & 0xF) | (SECOND >> 4 << 14));     // (the rows too, tree_attn_kernel)
            const float sl2 = a.scale * kLog2e;

            // 32 keys of the tile, those of sub-tile pair x0
            auto step = [&](const int tile, const int stage, const int x0, auto edge) {
                constexpr int XN = 1, SN = 2 * XN;
                constexpr bool EDGE = decltype(edge)::value;
                const unsigned char* k = lds + stage * STAGE + 16 * lane + x0 * 2 * KS * 1024;
                const unsigned char* v = lds + stage * STAGE + K_BYTES + 16 * lane + x0 * VT * 1024;
                // operands are read RING steps ahead (all at once they would need the registers that there are)
                constexpr int RING = 4, KF = SN * KS, VF = XN * VT;
                bf16x8 ring[RING];
                floatx4 s[NB][SN];
#pragma unroll
                for (int f = 0; f < RING; ++f) ring[f] = *reinterpret_cast<const bf16x8*>(k + f * 1024);
#pragma unroll
                for (int f = 0; f < KF; ++f) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        s[b][f / KS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ring[f % RING], q.q[b][f % KS], f % KS == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : s[b][f / KS], 0, 0, 0);
                    ring[f % RING] = *reinterpret_cast<const bf16x8*>(f + RING < KF ? k + (f + RING) * 1024 : v + (f + RING - KF) * 1024);
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                uint32_t hidden[NB] = {};
                if constexpr (EDGE) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        uint32_t seen = 0;
#pragma unroll
                        for (int u = 0; u < SN; ++u) seen |= seen_of_four(q.bits[b], tile * TOKENS + 32 * x0 + 16 * u + 4 * g, ctx, len) << 4 * u;
                        hidden[b] = ~seen;
                    }
                }
                bf16x8 pf[NB][XN];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float p[4 * SN];
                    probabilities<D, SN, EDGE, true>(s[b], hidden[b], sl2, y.o[b], y.l[b], y.m[b], p);
#pragma unroll
                    for (int x = 0; x < XN; ++x)
                        pf[b][x] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[8 * x], p[8 * x + 1]), pack_bf16x2(p[8 * x + 2], p[8 * x + 3]),
                                                                    pack_bf16x2(p[8 * x + 4], p[8 * x + 5]), pack_bf16x2(p[8 * x + 6], p[8 * x + 7])});
                }
                __builtin_amdgcn_s_setprio(1);
                const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
#pragma unroll
                for (int f = 0; f < VF; ++f) {
                    const int x = f / VT, t = f % VT;
                    if (t == 0) {
#pragma unroll
                        for (int b = 0; b < NB; ++b) y.l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[b][x], y.l[b], 0, 0, 0);       // (of the rounded probabilities)
                    }
                    if constexpr (EDGE) product_with_hidden<NB, D, XN>(ring[f % RING], hidden, x, pf, y, t);
                    else {
#pragma unroll
                        for (int b = 0; b < NB; ++b) y.o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ring[f % RING], pf[b][x], y.o[b][t], 0, 0, 0);
                    }
                    if (f + RING < VF) ring[f % RING] = *reinterpret_cast<const bf16x8*>(v + (f + RING) * 1024);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            const int x0 = sharers == 1 ? 0 : half, x1 = sharers == 1 ? 2 : half + 1;
            // Whatever feeds the matrix pipe and the copies goes before the other wave's softmax (trees of 64 requests 648 -> 640 us)
            __builtin_amdgcn_s_setprio(1);
            // LDS alone is waited for: the quarters on their way stay so
            const auto all_here = [&] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
            put(r0, 0);
            load(r0, p0, t0 + 2);
            // Tiles that every row sees whole, then the others, as in tree_attn_kernel.  A tile is requested three turns before it is used: two of them in registers.
            int tile = t0;
            const auto turn = [&](Quarter& r, int& p, const int stage) {
                all_here();
                put(r, stage ^ 1);
                load(r, p, tile + 3);
                if (works) for (int x = x0; x < x1; ++x) step(tile, stage, x, std::false_type{});
                ++tile;
            };
            while (tile + 1 < whole) {                                 // (one way out, as there)
                turn(r1, p1, 0);
                turn(r0, p0, 1);
            }
            if (tile < whole) {
                turn(r1, p1, 0);
                r1 = r0;
            }
            while (KEYS != kShared && tile < t1) {
                const int stage = (tile - t0) & 1;
                all_here();
                put(r1, stage ^ 1);
                p1 = ask_places<N>(a, bounds, tile + 2, 2 * pair);
                load(r1, p1, tile + 2);
                if (works) for (int x = x0; x < x1; ++x) step(tile, stage, x, std::true_type{});
                ++tile;
            }
        }
        finish<D, F8, NB, false, false, KEYS>(a, w, bounds, kvh, kWaves / sharers, sharers, y, lds, &last);
    }, first_item, step_of_items);
}
template <int D, bool F8, Keys KEYS = kAll>
__global__ __launch_bounds__(64 * kWaves, D == 64 && F8 ? 3 : 2) void tree_attn_wide_kernel(TreeArgs) {
    __shared__ __align__(16) unsigned char lds[kWideBytes<D>];
    __shared__ int last;
    many_rows<D, F8, KEYS, 0>(lds, last, blockIdx.x, gridDim.x);
}

// sub-tiles in a tile: two tiles in flight, and with the accumulators of 16 or 32 rows within 256 registers (512 for 32 rows and d = 128 in bf16)
template <int D, bool F8> constexpr int kSubTiles1 = D == 64 ? 4 : 2;
template <int D, bool F8> constexpr int kSubTiles2 = F8 && D == 64 ? 4 : 2;
template <int D, bool F8> constexpr int kWavesOf2 = F8 || D == 64 ? 2 : 1;
constexpr int kLeastKeys = 256;                     // keys of a piece at least: when four users' tokens took 13.1 us, they took 15.6 with 128 and 13.4 with 512; 51-token trees of six requests 44, 55, 50

// Sizes that follow from those of the call
inline void set_tree_sizes(TreeArgs& a, const TreeShape& s) {
    a.heads_per_kv = a.Hq / a.cache.Hkv;
    a.by_r = FastDiv::by(static_cast<uint32_t>(a.heads_per_kv));
    a.subs = a.cache.page / 16;
    a.by_subs = FastDiv::by(static_cast<uint32_t>(a.subs));
    a.chunk_shift = s.rows == 16 ? 4 : s.rows == 32 ? 5 : 7;
    a.chunks = s.chunks;
    a.by_chunks = FastDiv::by(static_cast<uint32_t>(a.chunks));
    a.by_hkv = FastDiv::by(static_cast<uint32_t>(a.cache.Hkv));
    a.most_keys = a.max_blocks * a.cache.page;      // (fewer than 2^31)
    a.items = s.items;
    a.rounds = s.rounds / 4.f;
}

}  // namespace
}  // namespace pk
