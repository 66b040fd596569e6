// Checks that the C entry points of the paged cache have in common, and how they refuse.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <string>

#include "cache.h"
#include "plan.h"

namespace pk {

// why an argument is refused: a code and its message
struct Refusal { int code; std::string why; };

inline int refuse(const char* who, const Refusal& r) {
    set_error(std::string(who) + ": " + r.why);
    return r.code;
}
inline int launched(const char* who, const int e) {
    if (e == 0) return PK_OK;
    set_error(std::string(who) + ": " + hipGetErrorString(static_cast<hipError_t>(e)));
    return PK_EHIP;
}
inline bool aligned(const void* p, const size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr int64_t kMostTokens = 0x7FFFFFFF;
constexpr int64_t kMostExtent = int64_t{1} << 59;   // elements that one stride may lead to: two of them in bytes stay within 64 bits

inline Refusal check_cache(const pk_cache* c) {
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

inline Refusal check_table(const int32_t* block_table, const int32_t max_blocks, const int32_t* kv_lens, const int32_t n, const pk_cache& c) {
    if (n < 0 || n > 65535) return {PK_EINVAL, "need 0 <= n < 65536"};
    if (n > 0 && (!block_table || !kv_lens)) return {PK_EINVAL, "block_table or kv_lens is NULL"};
    if (n > 0 && max_blocks <= 0) return {PK_EINVAL, "need max_blocks > 0"};
    if (max_blocks < 0 || static_cast<int64_t>(max_blocks) * c.page_size > kMostTokens) return {PK_EINVAL, "max_blocks is negative, or 2^31 tokens a request and more"};
    return {PK_OK, ""};
}

inline RowsView view(const pk_rows& r) { return {r.data, r.token_stride, r.head_stride}; }
inline CacheView view(const pk_cache& c) {
    return {c.k, c.v, static_cast<uint8_t*>(c.scales), c.num_blocks, c.page_size, c.Hkv, c.d, c.dtype == PK_F8};
}

// Compute units of the current device; 256 when there is none to ask (sizes can be queried without one)
inline int compute_units() {
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
        (void)hipGetLastError();
        return 256;
    }
    return cus;
}

#define PK_CHECK(call) do { const Refusal refusal = call; if (refusal.code != PK_OK) return refuse(who, refusal); } while (0)

inline bool tree_sizes_ok(const int64_t n, const int64_t max_q, const int64_t Hq, const int64_t Hkv, const int64_t d) {
    return n >= 0 && n <= 65535 && max_q >= 0 && max_q <= PK_MAX_DRAFTS && Hkv > 0 && Hkv <= 65535 && Hq > 0 && Hq <= 16384 && Hq % Hkv == 0 && (d == 64 || d == 128);
}

// Checks of pk_tree_attn, and the part of the arguments that is the caller's; `empty`: nothing to do
inline int tree_args(const char* who, const pk_cache* cache, const void* q, const int32_t* q_start, const int64_t total_q, const int32_t max_q, const uint64_t* tree_mask,
                     const int32_t* block_table, const int32_t max_blocks, const int32_t* kv_lens, const int32_t n, void* out, const float scale, const int Hq,
                     const int out_dtype, void* workspace, TreeArgs& a, bool& empty) {
    PK_CHECK(check_cache(cache));
    PK_CHECK(check_table(block_table, max_blocks, kv_lens, n, *cache));
    if (Hq <= 0 || Hq % cache->Hkv != 0 || Hq > 16384) return refuse(who, {PK_EINVAL, "need 0 < Hq <= 16384 and Hq % Hkv == 0"});
    if (total_q < 0 || total_q > kMostTokens || max_q < 0) return refuse(who, {PK_EINVAL, "need 0 <= total_q < 2^31 and max_q >= 0"});
    if (max_q > PK_MAX_DRAFTS) return refuse(who, {PK_EUNSUPPORTED, "more than 64 drafted tokens of a request (pk_packed_prefill_attn takes chunks)"});
    if (out_dtype != PK_BF16 && out_dtype != PK_F32) return refuse(who, {PK_EINVAL, "out_dtype must be PK_BF16 or PK_F32"});
    if (!(std::isfinite(scale) && scale > 0.f)) return refuse(who, {PK_EINVAL, "scale must be finite and positive"});
    empty = n == 0 || total_q == 0 || max_q == 0;
    if (empty) return PK_OK;
    if (!q || !out || !q_start) return refuse(who, {PK_EINVAL, "q, out or q_start is NULL"});
    if (!aligned(q, 16) || !aligned(out, 16)) return refuse(who, {PK_EINVAL, "q and out must be 16-byte aligned"});
    if (!workspace || !aligned(workspace, 256)) return refuse(who, {PK_EINVAL, "workspace is NULL or not 256-byte aligned"});
    a.cache = view(*cache); a.block_table = block_table; a.max_blocks = max_blocks;
    a.q = q; a.q_start = q_start; a.total_q = total_q; a.max_q = max_q; a.mask = tree_mask;
    a.kv_lens = kv_lens; a.n = n;
    a.out = out; a.out_f32 = out_dtype == PK_F32; a.scale = scale; a.Hq = Hq;
    return PK_OK;
}

}  // namespace pk
