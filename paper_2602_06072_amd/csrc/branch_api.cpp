// C ABI of the pages of the cache, of attention over shared pages and of the judging of drafted tokens: argument checks and launches.
#include <cmath>
#include <initializer_list>

#include "branch.h"
#include "cache_checks.h"
#include "shared_attn.h"

using namespace pk;

namespace {

// An array of 32-bit words, by the name that a message has for it
struct Words { const char* name; const void* at; int64_t count; };

bool overlap(const Words& x, const Words& y) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.at), b = reinterpret_cast<uintptr_t>(y.at);
    return x.count > 0 && y.count > 0 && a < b + static_cast<uintptr_t>(y.count) * 4 && b < a + static_cast<uintptr_t>(x.count) * 4;
}
Refusal check_words(const std::initializer_list<Words>& arrays) {
    for (const Words& x : arrays) {
        if (!x.at && x.count > 0) return {PK_EINVAL, std::string(x.name) + " is NULL"};
        if (!aligned(x.at, 4)) return {PK_EINVAL, std::string(x.name) + " must be 4-byte aligned"};
    }
    return {PK_OK, ""};
}
// outputs: apart from one another and from the inputs
Refusal check_apart(const std::initializer_list<Words>& outputs, const std::initializer_list<Words>& inputs) {
    for (const Words* x = outputs.begin(); x != outputs.end(); ++x) {
        for (const Words* y = outputs.begin(); y != x; ++y)
            if (overlap(*x, *y)) return {PK_EINVAL, std::string(x->name) + " overlaps " + y->name};
        for (const Words& y : inputs)
            if (overlap(*x, y)) return {PK_EINVAL, std::string(x->name) + " overlaps " + y.name};
    }
    return {PK_OK, ""};
}

// Rows of logits, in bytes: what is between them is not theirs
struct Rows { const char* name; const void* at; int64_t count, stride, length; };

bool overlap(const Words& x, const Rows& r) {
    if (x.count <= 0 || r.count <= 0) return false;
    const uintptr_t first = reinterpret_cast<uintptr_t>(r.at), begin = reinterpret_cast<uintptr_t>(x.at), end = begin + static_cast<uintptr_t>(x.count) * 4;
    if (end <= first) return false;
    const int64_t from = begin > first ? static_cast<int64_t>(begin - first) : 0, to = static_cast<int64_t>(end - first);
    const int64_t in = r.count > 1 ? from / r.stride : 0, row = in < r.count ? in : r.count - 1;      // the last row that begins at `from` or in front of it
    return from < row * r.stride + r.length || (row + 1 < r.count && to > (row + 1) * r.stride);
}

Refusal check_pages(const int32_t n, const int32_t max_blocks, const int64_t num_blocks, const int32_t page_size) {
    if (n < 0 || n > 65535) return {PK_EINVAL, "need 0 <= n < 65536"};
    if (num_blocks <= 0 || num_blocks > kMostTokens) return {PK_EINVAL, "need 0 < num_blocks < 2^31"};
    if (page_size <= 0) return {PK_EINVAL, "need page_size > 0"};
    if (max_blocks < 0 || (n > 0 && max_blocks == 0) || static_cast<int64_t>(max_blocks) * page_size > kMostTokens)
        return {PK_EINVAL, "max_blocks is 0 or negative, or 2^31 tokens a request and more"};
    return {PK_OK, ""};
}
Refusal check_workspace(const void* workspace, const size_t bytes, const size_t needed, const char* query) {
    if (!workspace || !aligned(workspace, 256)) return {PK_EINVAL, "workspace is NULL or not 256-byte aligned"};
    if (bytes < needed) return {PK_EINVAL, std::string("workspace smaller than ") + query};
    return {PK_OK, ""};
}

constexpr int32_t kMostVocab = 1 << 26;

// Whether shared pages are looked for, or every request is taken alone, by what the tables have room for (lengths are on the device).  Three dependent launches take 20 us, and
// reads of what is shared come from the caches: with requests that share nearly all, of 32 / 8 heads of 128 columns in 8 bits, one new token each, 31 us against 31 at 278 MB of keys and
// values (32 requests of 4100 tokens), 35 against 46 at 403 MB (16 of 12100), 26 against 20 at 139 MB; with six new tokens each 70 against 99 at 556 MB (64 of
// 4100), 54 against 62 at 226 MB (64 of 1600), 55 against 44 at 278 MB; in bf16 27 against 28 and 50 against 39 around 250 MB.
// What it costs where tables are wide and requests short: eight requests of one token behind 1200 to 1400, 11 us up to 512 pages of 16 tokens and 22 from 1024 on; eight of 60 to 300 18
// against 9.  A caller who knows such lengths says so with no families.
bool shared_pays(const TreeArgs& a, const int32_t families) {
    const CacheView& c = a.cache;
    const int64_t row = 2 * static_cast<int64_t>(c.Hkv) * (c.f8 ? c.d + 1 : 2 * c.d), tokens = static_cast<int64_t>(a.max_blocks) * c.page;       // (below 2^25 and 2^31)
    return families > 0 && families < a.n && tokens * a.n > (int64_t{1} << 28) / row && a.total_q * (a.Hq / c.Hkv) < (int64_t{1} << 30);
}

}  // namespace

extern "C" int pk_kv_pages_select(const int32_t* block_table, const int32_t* lens, const int32_t* pages, int32_t n, int32_t max_blocks,
                                  const int32_t* from, int32_t n_new, int32_t* new_table, int32_t* new_lens, int32_t* new_pages,
                                  int32_t* refs, int64_t num_blocks, int32_t page_size, void* stream) {
    const char* who = "pk_kv_pages_select";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        if (n_new < 0 || n_new > 65535) return refuse(who, {PK_EINVAL, "need 0 <= n_new < 65536"});
        PK_CHECK(check_pages(n > n_new ? n : n_new, max_blocks, num_blocks, page_size));
        if (n < 0) return refuse(who, {PK_EINVAL, "need 0 <= n < 65536"});
        if (n == 0 && n_new == 0) return PK_OK;
        const int64_t words = static_cast<int64_t>(n) * max_blocks, new_words = static_cast<int64_t>(n_new) * max_blocks;
        const Words table{"block_table", block_table, words}, ls{"lens", lens, n}, ps{"pages", pages, n}, fr{"from", from, n_new};
        const Words nt{"new_table", new_table, new_words}, nl{"new_lens", new_lens, n_new}, np{"new_pages", new_pages, n_new}, rf{"refs", refs, num_blocks};
        PK_CHECK(check_words({table, ls, ps, fr, nt, nl, np, rf}));
        PK_CHECK(check_apart({nt, nl, np, rf}, {table, ls, ps, fr}));
        PagesSelectArgs a{block_table, lens, pages, n, max_blocks, from, n_new, new_table, new_lens, new_pages, refs, static_cast<int32_t>(num_blocks), page_size};
        return launched(who, launch_pages_select(a, stream));
    });
}

extern "C" size_t pk_kv_pages_workspace_bytes(int64_t num_blocks) {
    return num_blocks > 0 && num_blocks <= kMostTokens ? PagesWorkspace::bytes(num_blocks) : 0;
}

extern "C" int pk_kv_pages_reserve(int32_t* block_table, const int32_t* lens, int32_t* pages, int32_t n, int32_t max_blocks,
                                   const int32_t* grow, int32_t* refs, int64_t num_blocks, int32_t page_size,
                                   int32_t* served, int32_t* copy_src, int32_t* copy_dst,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "pk_kv_pages_reserve";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_pages(n, max_blocks, num_blocks, page_size));
        if (n == 0) return PK_OK;
        const Words table{"block_table", block_table, static_cast<int64_t>(n) * max_blocks}, ls{"lens", lens, n}, ps{"pages", pages, n}, gr{"grow", grow, n};
        const Words rf{"refs", refs, num_blocks}, sv{"served", served, n}, cs{"copy_src", copy_src, n}, cd{"copy_dst", copy_dst, n};
        PK_CHECK(check_words({table, ls, ps, gr, rf, sv, cs, cd}));
        PK_CHECK(check_workspace(workspace, workspace_bytes, PagesWorkspace::bytes(num_blocks), "pk_kv_pages_workspace_bytes"));
        const Words ws{"workspace", workspace, static_cast<int64_t>(PagesWorkspace::bytes(num_blocks) / 4)};
        PK_CHECK(check_apart({table, ps, rf, sv, cs, cd, ws}, {ls, gr}));
        int32_t* at = static_cast<int32_t*>(workspace);
        PagesReserveArgs a{block_table, lens, pages, n, max_blocks, grow, refs, static_cast<int32_t>(num_blocks), page_size,
                           served, copy_src, copy_dst, at, at + PagesWorkspace::kWriters, at + PagesWorkspace::kNumbers};
        return launched(who, launch_pages_reserve(a, stream));
    });
}

extern "C" int pk_kv_pages_compact(const int32_t* block_table, const int32_t* pages, int32_t n, int32_t max_blocks,
                                   const int32_t* refs, int64_t num_blocks, int32_t* new_table, int32_t* new_refs,
                                   int32_t* copy_src, int32_t* copy_dst, int32_t max_moves,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "pk_kv_pages_compact";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_pages(n, max_blocks, num_blocks, 1));
        if (max_moves < 0) return refuse(who, {PK_EINVAL, "max_moves is negative"});
        const int64_t words = static_cast<int64_t>(n) * max_blocks;
        const Words table{"block_table", block_table, words}, ps{"pages", pages, n}, rf{"refs", refs, num_blocks};
        const Words nt{"new_table", new_table, words}, nr{"new_refs", new_refs, num_blocks}, cs{"copy_src", copy_src, max_moves}, cd{"copy_dst", copy_dst, max_moves};
        PK_CHECK(check_words({table, ps, rf, nt, nr, cs, cd}));
        PK_CHECK(check_workspace(workspace, workspace_bytes, PagesWorkspace::bytes(num_blocks), "pk_kv_pages_workspace_bytes"));
        const Words ws{"workspace", workspace, static_cast<int64_t>(PagesWorkspace::bytes(num_blocks) / 4)};
        PK_CHECK(check_apart({nr, cs, cd, ws}, {table, ps, rf}));
        PK_CHECK(check_apart({nt}, {ps, rf, nr, cs, cd, ws}));
        if (new_table != block_table) PK_CHECK(check_apart({nt}, {table}));
        int32_t* at = static_cast<int32_t*>(workspace);
        PagesCompactArgs a{block_table, pages, n, max_blocks, refs, static_cast<int32_t>(num_blocks), new_table, new_refs, copy_src, copy_dst, max_moves,
                           at + PagesWorkspace::kNumbers, at + PagesWorkspace::kUsed};
        return launched(who, launch_pages_compact(a, stream));
    });
}

extern "C" int pk_kv_cache_copy(const pk_cache* from, const pk_cache* to, const int32_t* copy_src, const int32_t* copy_dst,
                                int32_t count, void* stream) {
    const char* who = "pk_kv_cache_copy";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        PK_CHECK(check_cache(from));
        PK_CHECK(check_cache(to));
        if (from->page_size != to->page_size || from->Hkv != to->Hkv || from->d != to->d || from->dtype != to->dtype)
            return refuse(who, {PK_EINVAL, "the caches differ in dtype, page size or head shape"});
        if (count < 0) return refuse(who, {PK_EINVAL, "count is negative"});
        PK_CHECK(check_words({{"copy_src", copy_src, count}, {"copy_dst", copy_dst, count}}));
        const bool one = from->k == to->k;
        const auto parts = [](const pk_cache& c, const bool writes, Words (&w)[3]) {
            const int64_t values = c.num_blocks * c.Hkv * c.page_size * c.d * (c.dtype == PK_F8 ? 1 : 2) / 4, scales = c.num_blocks * c.Hkv * c.page_size * 2 / 4;
            w[0] = {writes ? "k of `to`" : "k of `from`", c.k, values};
            w[1] = {writes ? "v of `to`" : "v of `from`", c.v, values};
            w[2] = {writes ? "scales of `to`" : "scales of `from`", c.scales, c.dtype == PK_F8 ? scales : 0};
        };
        if (one && (from->v != to->v || (from->dtype == PK_F8 && from->scales != to->scales) || from->num_blocks != to->num_blocks))
            return refuse(who, {PK_EINVAL, "the caches overlap"});
        Words f[3], t[3];
        parts(*from, false, f);
        parts(*to, true, t);
        if (!one) PK_CHECK(check_apart({t[0], t[1], t[2]}, {f[0], f[1], f[2]}));
        PK_CHECK(check_apart({t[0], t[1], t[2]}, {{"copy_src", copy_src, count}, {"copy_dst", copy_dst, count}}));
        if (count == 0) return PK_OK;
        CacheCopyArgs a{};
        a.from = view(*from); a.to = view(*to);
        a.src = copy_src; a.dst = copy_dst; a.count = count;
        return launched(who, launch_cache_copy(a, stream));
    });
}

extern "C" size_t pk_shared_tree_attn_workspace_bytes(int32_t n, int32_t max_q, int64_t total_q, int Hq, int Hkv, int d) {
    if (!tree_sizes_ok(n, max_q, Hq, Hkv, d) || total_q < 0 || total_q > kMostTokens) return 0;
    const int cus = compute_units();
    return SharedWorkspace::of(n, total_q, TreeShape::of(max_q, Hq, Hkv, cus), Hq, Hkv, d, cus).bytes;
}

extern "C" int pk_shared_tree_attn(const pk_cache* cache, const void* q, const int32_t* q_start, int64_t total_q, int32_t max_q,
                                   const uint64_t* tree_mask, const int32_t* block_table, int32_t max_blocks,
                                   const int32_t* kv_lens, int32_t n, const int32_t* family_start, int32_t families,
                                   void* out, float scale, int Hq, int out_dtype,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "pk_shared_tree_attn";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        SharedArgs s{};
        TreeArgs& a = s.tree;
        bool empty = false;
        if (const int rc = tree_args(who, cache, q, q_start, total_q, max_q, tree_mask, block_table, max_blocks, kv_lens, n, out, scale, Hq, out_dtype, workspace, a, empty);
            rc != PK_OK) return rc;
        if (families < 0 || families > n) return refuse(who, {PK_EINVAL, "need 0 <= families <= n"});
        if (empty) return PK_OK;
        if (!family_start) return refuse(who, {PK_EINVAL, "family_start is NULL"});
        const int cus = compute_units();
        const TreeShape shape = TreeShape::of(max_q, Hq, cache->Hkv, cus);
        const SharedWorkspace w = SharedWorkspace::of(n, total_q, shape, Hq, cache->Hkv, cache->d, cus);
        if (workspace_bytes < w.bytes) return refuse(who, {PK_EINVAL, "workspace smaller than pk_shared_tree_attn_workspace_bytes"});
        char* at = static_cast<char*>(workspace);
        if (!shared_pays(a, families)) {
            a.arrived = reinterpret_cast<uint32_t*>(at + w.counts);
            a.part_o = reinterpret_cast<float*>(at + w.plain);
            a.part_lse = a.part_o + shape.rows_of_slots(cache->Hkv, cus) * cache->d;
            a.pieces_of = reinterpret_cast<int2*>(at + w.plain + shape.partial_bytes(cache->Hkv, cache->d, cus));
            return launched(who, launch_tree_attn(a, shape, stream));
        }
        s.family_start = family_start; s.families = families;
        s.arrived = reinterpret_cast<uint32_t*>(at);
        s.missing = reinterpret_cast<int32_t*>(at + 256);
        a.pieces_of = reinterpret_cast<int2*>(at + w.arrays);
        s.pieces_of_family = a.pieces_of + n;
        s.family_of = reinterpret_cast<int32_t*>(s.pieces_of_family + n);
        s.shared_of = s.family_of + n;
        s.first_of = s.shared_of + n;
        s.len_of = s.first_of + n;
        s.q_start_of = s.len_of + n;
        s.places = s.q_start_of + n + 1;
        a.part_o = reinterpret_cast<float*>(at + w.own);
        a.part_lse = a.part_o + w.own_slots * cache->Hkv * shape.rows * cache->d;
        s.family_o = reinterpret_cast<float*>(at + w.family);
        s.family_lse = s.family_o + w.family_slots * cache->Hkv * 128 * cache->d;
        return launched(who, launch_shared_tree_attn(s, shape, stream));
    });
}

extern "C" size_t pk_draft_verify_workspace_bytes(int32_t n, int64_t total_q, int32_t vocab) {
    if (n < 0 || n > 65535 || total_q < 0 || total_q > kMostTokens || vocab <= 0 || vocab > kMostVocab) return 0;
    return VerifyShape::bytes(n, total_q, vocab);
}

extern "C" int pk_draft_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int dtype,
                               int32_t vocab, const int32_t* tokens, const int32_t* q_start, int64_t total_q, int32_t max_q,
                               const uint64_t* tree_mask, int32_t n, const float* temperature,
                               const float* accept_u, const float* sample_u,
                               int32_t* keep, int32_t max_keep, int32_t* keep_count, int32_t* next_token,
                               void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "pk_draft_verify";
    return guarded<int>(PK_ENOMEM, PK_EINVAL, who, [&]() -> int {
        if (n < 0 || n > 65535) return refuse(who, {PK_EINVAL, "need 0 <= n < 65536"});
        if (total_q < 0 || total_q > kMostTokens || max_q < 0) return refuse(who, {PK_EINVAL, "need 0 <= total_q < 2^31 and max_q >= 0"});
        if (max_q > PK_MAX_DRAFTS) return refuse(who, {PK_EUNSUPPORTED, "more than 64 tokens of a request"});
        if (dtype != PK_BF16 && dtype != PK_F32) return refuse(who, {PK_EINVAL, "dtype must be PK_BF16 or PK_F32"});
        if (vocab <= 0) return refuse(who, {PK_EINVAL, "need vocab > 0"});
        if (vocab > kMostVocab) return refuse(who, {PK_EUNSUPPORTED, "a vocabulary of more than 2^26"});
        const int64_t most_stride = kMostExtent / (total_q > 0 ? total_q : 1);
        if ((total_q > 1 && target_stride < vocab) || target_stride < 0 || target_stride > most_stride) return refuse(who, {PK_EINVAL, "target_stride is less than vocab, or out of range"});
        if (draft && ((total_q > 1 && draft_stride < vocab) || draft_stride < 0 || draft_stride > most_stride)) return refuse(who, {PK_EINVAL, "draft_stride is less than vocab, or out of range"});
        if (n > 0 && max_keep < 1) return refuse(who, {PK_EINVAL, "need max_keep >= 1"});
        if (n == 0) return PK_OK;
        const size_t size = dtype == PK_F32 ? 4 : 2;
        if (total_q > 0 && !target) return refuse(who, {PK_EINVAL, "target is NULL"});
        if (!aligned(target, size) || !aligned(draft, size)) return refuse(who, {PK_EINVAL, "target and draft must be aligned to their type"});
        if (tree_mask && !aligned(tree_mask, 8)) return refuse(who, {PK_EINVAL, "tree_mask must be 8-byte aligned"});
        if (!aligned(temperature, 4)) return refuse(who, {PK_EINVAL, "temperature must be 4-byte aligned"});
        const Words kp{"keep", keep, static_cast<int64_t>(n) * max_keep}, kc{"keep_count", keep_count, n}, nt{"next_token", next_token, n};
        const Words tk{"tokens", tokens, total_q}, qs{"q_start", q_start, n + 1}, au{"accept_u", accept_u, total_q}, su{"sample_u", sample_u, n};
        PK_CHECK(check_words({kp, kc, nt, tk, qs, au, su}));
        const VerifyShape shape = VerifyShape::of(n, total_q, vocab);
        const size_t needed = VerifyShape::bytes(n, total_q, vocab);
        PK_CHECK(check_workspace(workspace, workspace_bytes, needed, "pk_draft_verify_workspace_bytes"));
        const Words ws{"workspace", workspace, static_cast<int64_t>(needed / 4)};
        const Words tm{"temperature", temperature, temperature ? n : 0}, mk{"tree_mask", tree_mask, tree_mask ? 2 * total_q : 0};
        PK_CHECK(check_apart({kp, kc, nt, ws}, {tk, qs, au, su, tm, mk}));
        const int64_t bytes = static_cast<int64_t>(size);
        for (const Words& x : {kp, kc, nt, ws})
            for (const Rows& r : {Rows{"target", target, total_q, target_stride * bytes, vocab * bytes}, Rows{"draft", draft, draft ? total_q : 0, draft_stride * bytes, vocab * bytes}})
                if (overlap(x, r)) return refuse(who, {PK_EINVAL, std::string(x.name) + " overlaps " + r.name});
        VerifyArgs a{target, target_stride, draft, draft_stride, dtype == PK_F32, vocab, tokens, q_start, total_q, max_q > 0 ? max_q : 1, tree_mask, n, temperature,
                     accept_u, sample_u, keep, max_keep, keep_count, next_token, shape, nullptr, nullptr, nullptr, nullptr, 1};
        if (max_q == 0) a.total_q = 0;              // no tokens: the outputs say so
        char* at = static_cast<char*>(workspace);
        a.arrived = reinterpret_cast<uint32_t*>(at);
        at += VerifyShape::kCountBytes;
        a.parts = reinterpret_cast<RowPart*>(at);
        a.last_parts = reinterpret_cast<RowPart*>(at + VerifyShape::part_bytes(total_q, vocab));
        a.choices = reinterpret_cast<VerifyChoice*>(at + VerifyShape::part_bytes(total_q, vocab) + VerifyShape::last_bytes(n, vocab));
        return launched(who, launch_draft_verify(a, stream));
    });
}
