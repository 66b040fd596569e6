// C ABI of the paged cache and of what runs on it: argument checks and launches.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <string>

#include "cache.h"
#include "plan.h"

using namespace pk;

namespace {

// why an argument is refused: a code and its message
struct Refusal { int code; std::string why; };

int refuse(const char* who, const Refusal& r) {
    set_error(std::string(who) + ": " + r.why);
    return r.code;
}
int launched(const char* who, const int e) {
    if (e == 0) return PK_OK;
    set_error(std::string(who) + ": " + hipGetErrorString(static_cast<hipError_t>(e)));
    return PK_EHIP;
}
bool aligned(const void* p, const size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr int64_t kMostTokens = 0x7FFFFFFF;
constexpr int64_t kMostExtent = int64_t{1} << 59;   // elements that one stride may lead to: two of them in bytes stay within 64 bits

Refusal check_rows(const pk_rows* r, const char* name, const int64_t tokens, const int heads, const int d, const int dtype, const bool output) {
    const std::string n = name;
    if (!r || (!r->data && tokens > 0)) return {PK_EINVAL, n + " is NULL"};
    if (r->dtype != PK_BF16 && r->dtype != PK_F32) return {PK_EINVAL, n + ": dtype must be PK_BF16 or PK_F32"};
    if (r->dtype != dtype) return {PK_EINVAL, n + " has another dtype than the rows beside it"};
    const int unit = r->dtype == PK_F32 ? 4 : 8;
    if (!aligned(r->data, 16) || r->token_stride % unit != 0 || r->head_stride % unit != 0)
        return {PK_EINVAL, n + ": address and strides must be multiples of 16 bytes"};
    if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride > kMostExtent / (tokens > 0 ? tokens : 1) || r->head_stride > kMostExtent / heads)
        return {PK_EINVAL, n + ": stride out of range"};
    if (output) {                                   // rows that lie apart one way or the other: heads inside tokens or tokens inside heads
        const bool heads_inside = (heads == 1 || r->head_stride >= d) && (tokens <= 1 || r->token_stride >= (heads - 1) * r->head_stride + d);
        const bool tokens_inside = (tokens <= 1 || r->token_stride >= d) && (heads == 1 || r->head_stride >= (tokens - 1) * r->token_stride + d);
        if (!heads_inside && !tokens_inside) return {PK_EINVAL, n + ": strides of an output must keep its rows apart"};
    }
    return {PK_OK, ""};
}

Refusal check_cache(const pk_cache* c) {
    if (!c) return {PK_EINVAL, "cache is NULL"};
    if (c->dtype != PK_F8 && c->dtype != PK_BF16) return {PK_EINVAL, "cache dtype must be PK_F8 or PK_BF16"};
    if (c->d != 64 && c->d != 128) return {PK_EUNSUPPORTED, "the cache is built for d in {64, 128}"};
    if (c->page_size <= 0 || c->page_size % 16 != 0) return {PK_EUNSUPPORTED, "page_size must be a multiple of 16"};
    if (c->Hkv <= 0 || c->Hkv > 65535 || c->num_blocks <= 0 || c->num_blocks > kMostTokens) return {PK_EINVAL, "need 0 < Hkv < 65536 and 0 < num_blocks < 2^31"};
    if (c->num_blocks * c->Hkv > kMostTokens / c->page_size) return {PK_EUNSUPPORTED, "a cache of 2^31 rows (num_blocks * Hkv * page_size) or more"};
    if (!c->k || !c->v || (c->dtype == PK_F8 && !c->scales)) return {PK_EINVAL, "k, v or scales of the cache is NULL"};
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 16)) return {PK_EINVAL, "k, v and scales of the cache must be 16-byte aligned"};
    return {PK_OK, ""};
}

Refusal check_rope(const pk_rope* r, const int64_t tokens, const int d) {
    if (!r) return {PK_OK, ""};
    if (!r->table || (!r->positions && tokens > 0)) return {PK_EINVAL, "table or positions of the rotation is NULL"};
    if (!aligned(r->table, 16)) return {PK_EINVAL, "the table of the rotation must be 16-byte aligned"};
    if (r->max_pos <= 0 || r->n_axes <= 0 || r->n_axes > 255 || r->axis_stride < 0) return {PK_EINVAL, "need max_pos > 0, 0 < n_axes < 256, axis_stride >= 0"};
    if (r->axis_stride > kMostExtent / r->n_axes) return {PK_EINVAL, "axis_stride out of range"};
    if (r->rot_dim <= 0 || r->rot_dim > d) return {PK_EINVAL, "need 0 < rot_dim <= d"};
    if (r->rot_dim % 16 != 0) return {PK_EUNSUPPORTED, "rot_dim must be a multiple of 16"};
    if (r->interleaved != 0 && r->interleaved != 1) return {PK_EINVAL, "interleaved must be 0 or 1"};
    for (int p = 0; r->pair_axis && p < r->rot_dim / 2; ++p)
        if (r->pair_axis[p] >= r->n_axes) return {PK_EINVAL, "pair_axis names an axis that there is not"};
    return {PK_OK, ""};
}

Refusal check_table(const int32_t* block_table, const int32_t max_blocks, const int32_t* kv_lens, const int32_t n, const pk_cache& c) {
    if (n < 0 || n > 65535) return {PK_EINVAL, "need 0 <= n < 65536"};
    if (n > 0 && (!block_table || !kv_lens)) return {PK_EINVAL, "block_table or kv_lens is NULL"};
    if (n > 0 && max_blocks <= 0) return {PK_EINVAL, "need max_blocks > 0"};
    if (max_blocks < 0 || static_cast<int64_t>(max_blocks) * c.page_size > kMostTokens) return {PK_EINVAL, "max_blocks is negative, or 2^31 tokens a request and more"};
    return {PK_OK, ""};
}

RowsView view(const pk_rows& r) { return {r.data, r.token_stride, r.head_stride}; }
CacheView view(const pk_cache& c) {
    return {c.k, c.v, static_cast<uint8_t*>(c.scales), c.num_blocks, c.page_size, c.Hkv, c.d, c.dtype == PK_F8};
}

void put_rope(const pk_rope* r, TokenRowsArgs& a) {
    if (!r) return;
    a.table = r->table; a.positions = r->positions; a.axis_stride = r->axis_stride;
    a.max_pos = r->max_pos; a.pairs = r->rot_dim / 2; a.interleaved = r->interleaved;
    for (int p = 0; p < a.pairs; ++p) a.pair_axis[p] = r->pair_axis ? r->pair_axis[p] : 0;
}

#define PK_CHECK(call) do { const Refusal refusal = call; if (refusal.code != PK_OK) return refuse(who, refusal); } while (0)

// norm and rotation of q and k: checks, and the part of the arguments that is theirs
int norm_rope_args(const char* who, const pk_rows* q, const pk_rows* k, const pk_rows* q_out, const void* q_weight, const void* k_weight, const float eps,
                   const pk_rope* rope, const int64_t tokens, const int Hq, const int Hkv, const int d, TokenRowsArgs& a) {
    if (tokens < 0 || tokens > kMostTokens) return refuse(who, {PK_EINVAL, "need 0 <= tokens < 2^31"});
    if (Hq <= 0 || Hkv <= 0 || Hq > 16384 || Hkv > 16384 || d <= 0) return refuse(who, {PK_EINVAL, "need 0 < Hq, Hkv <= 16384 and d > 0"});
    if (d % 8 != 0 || d > 256) return refuse(who, {PK_EUNSUPPORTED, "d must be a multiple of 8 and at most 256"});
    if (!q) return refuse(who, {PK_EINVAL, "q is NULL"});
    PK_CHECK(check_rows(q, "q", tokens, Hq, d, q->dtype, false));
    PK_CHECK(check_rows(k, "k", tokens, Hkv, d, q->dtype, false));
    if (!q_out) return refuse(who, {PK_EINVAL, "q_out is NULL"});
    PK_CHECK(check_rows(q_out, "q_out", tokens, Hq, d, q_out->dtype, true));
    if ((q_weight || k_weight) && !(std::isfinite(eps) && eps >= 0.f)) return refuse(who, {PK_EINVAL, "eps must be finite and not negative"});
    if (!aligned(q_weight, 16) || !aligned(k_weight, 16)) return refuse(who, {PK_EINVAL, "weights must be 16-byte aligned"});
    PK_CHECK(check_rope(rope, tokens, d));
    a.q = view(*q); a.k = view(*k); a.q_out = view(*q_out);
    a.q_weight = q_weight; a.k_weight = k_weight; a.eps = eps;
    a.tokens = tokens; a.Hq = Hq; a.Hkv = Hkv; a.d = d;
    a.in_f32 = q->dtype == PK_F32; a.out_f32 = q_out->dtype == PK_F32;
    put_rope(rope, a);
    return PK_OK;
}

int cache_write_args(const char* who, const pk_cache* cache, const pk_rows* v, const int v_dtype, const int64_t* slots, const int64_t tokens, TokenRowsArgs& a) {
    PK_CHECK(check_rows(v, "v", tokens, cache->Hkv, cache->d, v_dtype, false));
    if (!slots && tokens > 0) return refuse(who, {PK_EINVAL, "slots is NULL"});
    a.v = view(*v); a.cache = view(*cache); a.slots = slots;
    return PK_OK;
}

// Compute units of the current device; 256 when there is none to ask (sizes can be queried without one)
int compute_units() {
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
        (void)hipGetLastError();
        return 256;
    }
    return cus;
}

bool tree_sizes_ok(const int64_t n, const int64_t max_q, const int64_t Hq, const int64_t Hkv, const int64_t d) {
    return n >= 0 && n <= 65535 && max_q >= 0 && max_q <= PK_MAX_DRAFTS && Hkv > 0 && Hkv <= 65535 && Hq > 0 && Hq <= 16384 && Hq % Hkv == 0 && (d == 64 || d == 128);
}

}  // namespace

TreeShape TreeShape::of(const int max_q, const int Hq, const int Hkv, const int compute_units) {
    const int rows = max_q * (Hq / Hkv);
    TreeShape s{rows <= 16 ? 16 : rows <= 32 ? 32 : 128, 1, 0, rows <= 32 ? kRoundsOfFewRows : 5, (rows + 31) / 32};
    s.chunks = rows <= s.rows ? 1 : (rows + s.rows - 1) / s.rows;
    s.items = 2 * compute_units > Hkv ? 2 * compute_units / Hkv : 1;       // (two workgroups of a compute unit)
    return s;
}

extern "C" int pk_qk_norm_rope(const pk_rows* q, const pk_rows* k, const pk_rows* q_out, const pk_rows* k_out,
                               const void* q_weight, const void* k_weight, float eps, const pk_rope* rope,
                               int64_t tokens, int Hq, int Hkv, int d, void* stream) {
    const char* who = "pk_qk_norm_rope";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        TokenRowsArgs a{};
        if (const int rc = norm_rope_args(who, q, k, q_out, q_weight, k_weight, eps, rope, tokens, Hq, Hkv, d, a); rc != PK_OK) return rc;
        PK_CHECK(check_rows(k_out, "k_out", tokens, Hkv, d, q_out->dtype, true));
        if (tokens == 0) return PK_OK;
        a.k_out = view(*k_out);
        return launched(who, launch_token_rows(a, stream));
    });
}

extern "C" int pk_kv_cache_write(const pk_cache* cache, const pk_rows* k, const pk_rows* v, const int64_t* slots,
                                 int64_t tokens, void* stream) {
    const char* who = "pk_kv_cache_write";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(cache));
        if (tokens < 0 || tokens > kMostTokens) return refuse(who, {PK_EINVAL, "need 0 <= tokens < 2^31"});
        if (!k) return refuse(who, {PK_EINVAL, "k is NULL"});
        PK_CHECK(check_rows(k, "k", tokens, cache->Hkv, cache->d, k->dtype, false));
        TokenRowsArgs a{};
        if (const int rc = cache_write_args(who, cache, v, k->dtype, slots, tokens, a); rc != PK_OK) return rc;
        if (tokens == 0) return PK_OK;
        a.k = view(*k);
        a.tokens = tokens; a.Hkv = cache->Hkv; a.d = cache->d;
        a.in_f32 = k->dtype == PK_F32;
        return launched(who, launch_token_rows(a, stream));
    });
}

extern "C" int pk_qkv_cache_write(const pk_cache* cache, const pk_rows* q, const pk_rows* k, const pk_rows* v,
                                  const int64_t* slots, const pk_rows* q_out,
                                  const void* q_weight, const void* k_weight, float eps, const pk_rope* rope,
                                  int64_t tokens, int Hq, void* stream) {
    const char* who = "pk_qkv_cache_write";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(cache));
        TokenRowsArgs a{};
        if (const int rc = norm_rope_args(who, q, k, q_out, q_weight, k_weight, eps, rope, tokens, Hq, cache->Hkv, cache->d, a); rc != PK_OK) return rc;
        if (const int rc = cache_write_args(who, cache, v, q->dtype, slots, tokens, a); rc != PK_OK) return rc;
        if (tokens == 0) return PK_OK;
        return launched(who, launch_token_rows(a, stream));
    });
}

extern "C" int pk_kv_cache_read(const pk_cache* cache, const int32_t* block_table, int32_t max_blocks,
                                const int32_t* kv_lens, const int32_t* row_start, int32_t n,
                                const pk_rows* k_out, const pk_rows* v_out, int64_t rows, void* stream) {
    const char* who = "pk_kv_cache_read";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(cache));
        PK_CHECK(check_table(block_table, max_blocks, kv_lens, n, *cache));
        if (rows < 0 || rows > kMostTokens) return refuse(who, {PK_EINVAL, "need 0 <= rows < 2^31"});
        if (!row_start && n > 0) return refuse(who, {PK_EINVAL, "row_start is NULL"});
        if (!k_out) return refuse(who, {PK_EINVAL, "k_out is NULL"});
        PK_CHECK(check_rows(k_out, "k_out", rows, cache->Hkv, cache->d, k_out->dtype, true));
        PK_CHECK(check_rows(v_out, "v_out", rows, cache->Hkv, cache->d, k_out->dtype, true));
        if (n == 0 || rows == 0) return PK_OK;
        CacheReadArgs a{};
        a.cache = view(*cache); a.block_table = block_table; a.max_blocks = max_blocks;
        a.kv_lens = kv_lens; a.row_start = row_start; a.n = n;
        a.k_out = view(*k_out); a.v_out = view(*v_out); a.rows = rows;
        a.out_f32 = k_out->dtype == PK_F32;
        return launched(who, launch_cache_read(a, stream));
    });
}

extern "C" size_t pk_tree_attn_workspace_bytes(int32_t n, int32_t max_q, int Hq, int Hkv, int d) {
    return guarded<size_t>(size_t{0}, size_t{0}, "pk_tree_attn_workspace_bytes", [&]() -> size_t {
        if (!tree_sizes_ok(n, max_q, Hq, Hkv, d)) return 0;
        const int cus = compute_units();
        const TreeShape s = TreeShape::of(max_q, Hq, Hkv, cus);
        return TreeShape::count_bytes(Hkv, cus) + s.partial_bytes(Hkv, d, cus) + TreeShape::pieces_bytes(n);
    });
}

extern "C" int pk_tree_attn(const pk_cache* cache, const void* q, const int32_t* q_start, int64_t total_q, int32_t max_q,
                            const uint64_t* tree_mask, const int32_t* block_table, int32_t max_blocks,
                            const int32_t* kv_lens, int32_t n, void* out, float scale, int Hq, int out_dtype,
                            void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "pk_tree_attn";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(cache));
        PK_CHECK(check_table(block_table, max_blocks, kv_lens, n, *cache));
        if (Hq <= 0 || Hq % cache->Hkv != 0 || Hq > 16384) return refuse(who, {PK_EINVAL, "need 0 < Hq <= 16384 and Hq % Hkv == 0"});
        if (total_q < 0 || total_q > kMostTokens || max_q < 0) return refuse(who, {PK_EINVAL, "need 0 <= total_q < 2^31 and max_q >= 0"});
        if (max_q > PK_MAX_DRAFTS) return refuse(who, {PK_EUNSUPPORTED, "more than 64 drafted tokens of a request (pk_packed_prefill_attn takes chunks)"});
        if (out_dtype != PK_BF16 && out_dtype != PK_F32) return refuse(who, {PK_EINVAL, "out_dtype must be PK_BF16 or PK_F32"});
        if (!(std::isfinite(scale) && scale > 0.f)) return refuse(who, {PK_EINVAL, "scale must be finite and positive"});
        if (n == 0 || total_q == 0 || max_q == 0) return PK_OK;
        if (!q || !out || !q_start) return refuse(who, {PK_EINVAL, "q, out or q_start is NULL"});
        if (!aligned(q, 16) || !aligned(out, 16)) return refuse(who, {PK_EINVAL, "q and out must be 16-byte aligned"});
        if (!workspace || !aligned(workspace, 256)) return refuse(who, {PK_EINVAL, "workspace is NULL or not 256-byte aligned"});
        const int cus = compute_units();
        const TreeShape shape = TreeShape::of(max_q, Hq, cache->Hkv, cus);
        const size_t counts = TreeShape::count_bytes(cache->Hkv, cus), partial = shape.partial_bytes(cache->Hkv, cache->d, cus);
        if (workspace_bytes < counts + partial + TreeShape::pieces_bytes(n))
            return refuse(who, {PK_EINVAL, "workspace smaller than pk_tree_attn_workspace_bytes"});
        TreeArgs a{};
        a.cache = view(*cache); a.block_table = block_table; a.max_blocks = max_blocks;
        a.q = q; a.q_start = q_start; a.total_q = total_q; a.max_q = max_q; a.mask = tree_mask;
        a.kv_lens = kv_lens; a.n = n;
        a.out = out; a.out_f32 = out_dtype == PK_F32; a.scale = scale; a.Hq = Hq;
        char* at = static_cast<char*>(workspace);
        a.arrived = reinterpret_cast<uint32_t*>(at);
        a.part_o = reinterpret_cast<float*>(at + counts);
        a.part_lse = a.part_o + shape.rows_of_slots(cache->Hkv, cus) * cache->d;
        a.pieces_of = reinterpret_cast<int2*>(at + counts + partial);
        return launched(who, launch_tree_attn(a, shape, stream));
    });
}

extern "C" int pk_kv_cache_keep(const pk_cache* cache, const int32_t* block_table, int32_t max_blocks,
                                const int32_t* kv_lens, const int32_t* q_start, int32_t n,
                                const int32_t* keep, int32_t max_keep, const int32_t* keep_count,
                                int32_t* new_lens, void* stream) {
    const char* who = "pk_kv_cache_keep";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(cache));
        PK_CHECK(check_table(block_table, max_blocks, kv_lens, n, *cache));
        if (max_keep < 0) return refuse(who, {PK_EINVAL, "max_keep is negative"});
        if (n == 0) return PK_OK;
        if (!q_start || (!keep && max_keep > 0) || !keep_count || !new_lens) return refuse(who, {PK_EINVAL, "q_start, keep, keep_count or new_lens is NULL"});
        // (a workgroup writes a request's new length while those of its other heads still read)
        const auto meets = [&](const void* p, const int64_t words) {
            const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(new_lens);
            return x < y + static_cast<uintptr_t>(n) * 4 && y < x + static_cast<uintptr_t>(words) * 4;
        };
        if (meets(kv_lens, n) || meets(q_start, n + 1) || meets(keep_count, n) || meets(keep, static_cast<int64_t>(n) * max_keep) ||
            meets(block_table, static_cast<int64_t>(n) * max_blocks))
            return refuse(who, {PK_EINVAL, "new_lens must not be kv_lens itself nor lie in another of the arrays"});
        CacheKeepArgs a{};
        a.cache = view(*cache); a.block_table = block_table; a.max_blocks = max_blocks;
        a.kv_lens = kv_lens; a.q_start = q_start; a.n = n;
        a.keep = keep; a.max_keep = max_keep; a.keep_count = keep_count; a.new_lens = new_lens;
        return launched(who, launch_cache_keep(a, stream));
    });
}
