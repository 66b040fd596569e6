// Checks that the C entry points of the paged cache have in common, and how they refuse.
#pragma once
#include <hip/hip_runtime_api.h>

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

}  // namespace pk
