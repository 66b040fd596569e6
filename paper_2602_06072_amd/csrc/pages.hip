// Pages of the paged cache: a new batch out of rows of the old one, pages for the next tokens, compaction, copies of blocks.
//
// All but the copies is whole numbers: 4 bytes an entry of a block table and a block of the pool.  Counts of holders change by atomic additions,
// whose order does not matter; whatever is handed out is found by prefix sums over requests and blocks in their order, so that results repeat.
#include "branch.h"
#include "common.hip.h"

namespace pk {
namespace {

constexpr int kWave = 64;

template <class T>
__device__ __forceinline__ T wave_prefix_sum(T x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(x, o, 64);
        x += lane >= o ? y : 0;
    }
    return x;
}
// Sum of x over the threads in front of this one, and over all of them.  `lds`: a word for every wave.
template <int THREADS, class T>
__device__ __forceinline__ T sum_in_front(const T x, T* lds, T& all) {
    const int wave = threadIdx.x >> 6;
    const T upto = wave_prefix_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[wave] = upto;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    return before + upto - x;
}

__device__ __forceinline__ int64_t place_of(const int64_t b) { return PagesWorkspace::at(static_cast<uint32_t>(b)); }
__device__ __forceinline__ bool is_block(const int b, const int num_blocks) { return b >= 0 && b < num_blocks; }

// Counts of four blocks; `none` for those that the pool does not have
__device__ __forceinline__ void load_refs(const int32_t* refs, const int64_t b, const int64_t num_blocks, const int none, int (&x)[4]) {
    if (b + 4 <= num_blocks) {
        __builtin_memcpy(x, refs + b, 16);          // (at any alignment)
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = b + e < num_blocks ? refs[b + e] : none;
    }
}

// ------------------------------------------------------------------ a new batch out of rows of the old one
// One wave for kOfRow entries of every new request (and as many again, gridDim.y times that further on), one for those of every old one.  Bound by the way there, three loads
// one behind the other and the additions: 2 to 8 forks of each of 64 requests of 200 to 6000 tokens 6.5 us, four requests forked twice 2.5 (a wave for a whole row 7.5 and 2.6, and 6 requests of 1000 pages renamed 20 us instead of 5).
constexpr int kAtOnce = 4, kOfRow = kAtOnce * kWave;
template <class Each>
__device__ __forceinline__ void for_entries(const int32_t* row, const int pages, Each each) {       // each(entry's number, block)
    for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * kOfRow + (threadIdx.x & 63); j0 < pages; j0 += static_cast<int64_t>(gridDim.y) * kOfRow) {
        int b[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) b[e] = row[min(j0 + e * kWave, static_cast<int64_t>(pages) - 1)];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) if (j0 + e * kWave < pages) each(j0 + e * kWave, b[e]);
    }
}
__global__ __launch_bounds__(256) void pages_select_kernel(PagesSelectArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t most = static_cast<int64_t>(a.max_blocks) * a.page;
    const auto held = [&](const int i) { return min(max(a.pages[i], 0), a.max_blocks); };
    if (unit < a.n_new) {
        const int i = static_cast<int>(unit), s = a.from[i];
        const bool there = s >= 0 && s < a.n;
        const int len = there ? static_cast<int>(min(static_cast<int64_t>(max(a.lens[s], 0)), most)) : 0;
        const int pages = there ? min(static_cast<int>((static_cast<int64_t>(len) + a.page - 1) / a.page), held(s)) : 0;
        int32_t* to = a.new_table + static_cast<int64_t>(i) * a.max_blocks;
        for_entries(a.table + static_cast<int64_t>(there ? s : 0) * a.max_blocks, pages, [&](const int64_t j, const int b) {
            to[j] = b;
            if (is_block(b, a.num_blocks)) atomicAdd(a.refs + b, 1);
        });
        if (lane == 0 && blockIdx.y == 0) { a.new_lens[i] = len; a.new_pages[i] = pages; }
    } else if (unit - a.n_new < a.n) {
        const int i = static_cast<int>(unit - a.n_new);
        for_entries(a.table + static_cast<int64_t>(i) * a.max_blocks, held(i), [&](int64_t, const int b) {
            if (is_block(b, a.num_blocks)) atomicAdd(a.refs + b, -1);
        });
    }
}

// ------------------------------------------------------------------ pages for the next tokens
// What a request asks for.  A page wholly behind its tokens that others hold too (it was cut to fewer tokens behind a fork) is not to be written either: the request gives it
// up, with the entries behind it, and takes free blocks instead.
struct Wish {
    int at, had, held, wanted, end;                 // page of its next token, pages it holds, those that it goes on holding, pages of all its tokens then, pages it holds then
    int block, holders;                             // block of the next token's page, how many hold it
    bool shared;                                    // that page holds tokens of its own and is held by others too: it is not to be written
};
__device__ __forceinline__ Wish wish_of(const PagesReserveArgs& a, const int i) {
    const int64_t most = static_cast<int64_t>(a.max_blocks) * a.page;
    const int64_t len = min(static_cast<int64_t>(max(a.lens[i], 0)), most);
    const int32_t* row = a.table + static_cast<int64_t>(i) * a.max_blocks;
    const int grow = max(a.grow[i], 0);
    Wish w;
    w.at = static_cast<int>(len / a.page);
    w.had = w.held = min(max(a.pages[i], 0), a.max_blocks);
    const bool part = len % a.page > 0;
    w.wanted = grow > 0 ? static_cast<int>(min((len + grow + a.page - 1) / a.page, static_cast<int64_t>(a.max_blocks))) : 0;
    const int behind = w.at + (part ? 1 : 0), upto = min(w.held, w.wanted);
    // (the next token's page and the one behind are asked for together, also where they are not needed; further ones hardly ever are)
    const int block = row[min(w.at, a.max_blocks - 1)], next = row[min(behind, a.max_blocks - 1)];
    const auto holders_of = [&](const int b) { const int x = a.refs[is_block(b, a.num_blocks) ? b : 0]; return is_block(b, a.num_blocks) ? x : 0; };
    const int holders = holders_of(block), holders_of_next = holders_of(next);
    const bool there = grow > 0 && part && w.at < w.held;
    w.block = there ? block : -1;
    w.holders = there ? holders : 0;
    w.shared = w.holders > 1;
    if (behind < upto) {
        int j = behind;
        if (holders_of_next <= 1) do ++j; while (j < upto && holders_of(row[j]) <= 1);
        w.held = j < upto ? j : w.held;
    }
    w.end = max(w.held, w.wanted);
    return w;
}
__device__ __forceinline__ int device_load(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// left in served[i] between two launches; copy_dst[i]: its first free block's number among those handed out; copy_src[i]: pages that it goes on holding
enum { kServed = 1, kCopies = 2, kWrites = 4 };

// One workgroup: who gets what.  (Requests are 4 to 12 bytes, blocks 4: the whole state of a batch is a few hundred KiB, and what takes time is the chain of loads: 9 us for
// 8 requests, 14 for 320 and 20000 blocks; 20 when what is known of a request was read in each of the three passes over them.)  HERE: the requests fit its threads, and it writes their entries too: a thread for each block
// that is handed out, which finds its request among the prefix sums.  (More requests: this workgroup reads each three times, and a second launch writes; 2000 on 140000 blocks 16 to 25 us, by how
// far the free ones are behind; 65535 on 2000000 blocks 590 to 690.)
constexpr int kPlanThreads = 1024;
template <bool HERE>
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(PagesReserveArgs a) {
    __shared__ int64_t lds[kPlanThreads / 64];
    __shared__ int begins[HERE ? kPlanThreads : 1];
    __shared__ int2 rows[HERE ? kPlanThreads : 1];  // page that the first block goes to (negative: -1 - the page that is copied), page of the others less their number
    const int tid = threadIdx.x;
    // four times four blocks of a thread, those of all threads side by side; counts of the four in 16 bits each
    constexpr int GROUPS = 4, OF_GROUP = 4 * kPlanThreads;
    int refs[GROUPS][4];
    const auto ask = [&](const int64_t b0) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) load_refs(a.refs, b0 + g * OF_GROUP + 4 * tid, a.num_blocks, 1, refs[g]);
    };
    ask(0);                                         // (beside the requests)
    Wish kept{};                                    // of request tid
    for (int i = tid; i < a.n; i += kPlanThreads) {
        const Wish w = wish_of(a, i);
        if (i == tid) kept = w;
        if (!w.shared) continue;
        atomicMax(a.last_writer + place_of(w.block), i + 1);
        atomicAdd(a.writers + place_of(w.block), 1);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): the sums are in the L2, where they are read
    __syncthreads();
    const auto wish = [&](const int i) { return i == tid ? kept : wish_of(a, i); };
    const auto needs = [&](const int i, const Wish& w, bool& keeps) {
        // of as many writers as there are holders the last one keeps the page
        keeps = w.shared && device_load(a.writers + place_of(w.block)) == w.holders && device_load(a.last_writer + place_of(w.block)) == i + 1;
        return static_cast<int64_t>(w.end - w.held + (w.shared && !keeps ? 1 : 0));
    };
    // the blocks that are wanted
    int64_t wanted = 0, begin = 0, need = 0;
    bool keeps = false;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        int64_t all;
        need = 0;
        keeps = false;
        if (i < a.n) need = needs(i, wish(i), keeps);
        begin = sum_in_front<kPlanThreads>(need, lds, all);
        wanted += all;
    }
    // as many free ones, by rising number
    int64_t found = 0;
    for (int64_t b0 = 0; b0 < a.num_blocks && found < wanted; b0 += GROUPS * OF_GROUP) {
        if (b0 > 0) ask(b0);
        int64_t mine = 0, all;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += static_cast<int64_t>(refs[g][e] == 0) << 16 * g;
        const int64_t front = sum_in_front<kPlanThreads>(mine, lds, all);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            int64_t at = found + (front >> 16 * g & 0xFFFF);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (refs[g][e] == 0 && at < a.num_blocks) a.free[place_of(at++)] = static_cast<int32_t>(b0 + g * OF_GROUP + 4 * tid + e);
            found += all >> 16 * g & 0xFFFF;
        }
    }
    if constexpr (HERE) {
        const int i = tid;
        const bool there = i < a.n, served = there && (begin + need <= found || (need == 0 && !keeps)), copies = served && kept.shared && !keeps;
        // (where blocks run out, requests that are not served want none, and no later one is)
        begins[tid] = static_cast<int>(begin < found ? begin : found);
        rows[tid] = {copies ? -1 - kept.at : kept.held, kept.held - (copies ? 1 : 0)};
        int64_t handed = served ? need : 0, all;
        sum_in_front<kPlanThreads>(handed, lds, all);
        if (there) {
            a.served[i] = served ? 1 : 0;
            a.copy_src[i] = copies ? kept.block : -1;
            if (!copies) a.copy_dst[i] = -1;
            if (served) a.pages[i] = kept.end;
            if (copies) atomicAdd(a.refs + kept.block, -1);
            if (kept.shared) { a.last_writer[place_of(kept.block)] = 0; a.writers[place_of(kept.block)] = 0; }
            for (int j = kept.held; served && j < kept.had; ++j)
                if (const int b = a.table[static_cast<int64_t>(i) * a.max_blocks + j]; is_block(b, a.num_blocks)) atomicAdd(a.refs + b, -1);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);        // (the free blocks: of this workgroup, through the L2)
        __syncthreads();
        for (int64_t k = tid; k < all; k += kPlanThreads) {
            int r = 0;                              // the last request that begins at k or in front of it (those behind it with no blocks begin there too, and are none of k's)
            for (int step = kPlanThreads / 2; step > 0; step >>= 1) r += r + step < a.n && begins[r + step] <= k ? step : 0;
            const int b = device_load(a.free + place_of(k)), number = static_cast<int>(k) - begins[r];
            const int2 at = rows[r];
            const bool copy = number == 0 && at.x < 0;
            a.table[static_cast<int64_t>(r) * a.max_blocks + (copy ? -1 - at.x : at.y + number)] = b;
            a.refs[b] = 1;
            if (copy) a.copy_dst[r] = b;
        }
        return;
    }
    // in the order of requests
    int64_t before = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        int64_t all;
        need = 0;
        keeps = false;
        Wish w{};
        if (i < a.n) { w = wish(i); need = needs(i, w, keeps); }
        begin = before + sum_in_front<kPlanThreads>(need, lds, all);
        if (i < a.n) {
            const bool served = begin + need <= found || (need == 0 && !keeps);
            a.served[i] = (served ? kServed : 0) | (w.shared && !keeps ? kCopies : 0) | (w.shared ? kWrites : 0);
            a.copy_dst[i] = served ? static_cast<int32_t>(begin) : -1;
            a.copy_src[i] = w.held;
        }
        before += all;
    }
}

// A wave for every request: its entries
__global__ __launch_bounds__(256) void pages_apply_kernel(PagesReserveArgs a) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= a.n) return;
    const int flags = a.served[i], begin = a.copy_dst[i];
    Wish w = wish_of(a, i);
    w.shared = flags & kWrites;                     // (counts change meanwhile: what was shared has been left here)
    w.held = a.copy_src[i];
    w.end = max(w.held, w.wanted);
    int32_t* row = a.table + static_cast<int64_t>(i) * a.max_blocks;
    const bool served = flags & kServed, copies = served && (flags & kCopies);
    if (lane == 0) {
        int dst = -1;
        if (copies) {
            dst = a.free[place_of(begin)];
            row[w.at] = dst;
            a.refs[dst] = 1;
            atomicAdd(a.refs + w.block, -1);
        }
        if (w.shared) { a.last_writer[place_of(w.block)] = 0; a.writers[place_of(w.block)] = 0; }
        a.copy_src[i] = copies ? w.block : -1;
        a.copy_dst[i] = dst;
        a.served[i] = served ? 1 : 0;
        if (served) a.pages[i] = w.end;
    }
    if (!served) return;
    for (int j = w.held + lane; j < max(w.had, w.end); j += kWave) {
        if (j < w.had && is_block(row[j], a.num_blocks)) atomicAdd(a.refs + row[j], -1);
        if (j >= w.end) continue;
        const int b = a.free[place_of(begin + (copies ? 1 : 0) + j - w.held)];
        row[j] = b;
        a.refs[b] = 1;
    }
}

// ------------------------------------------------------------------ compaction
constexpr int kSegment = PagesWorkspace::kSegment, kOfThread = kSegment / 256;
static_assert(kOfThread == 4, "load_refs");

__device__ __forceinline__ int used_in_segment(const int32_t* refs, const int64_t first, const int64_t end, int* lds) {
    int mine = 0, all;
    for (int64_t b = first + threadIdx.x; b < end; b += 256) mine += refs[b] > 0 ? 1 : 0;
    sum_in_front<256>(mine, lds, all);
    return all;
}
__global__ __launch_bounds__(256) void pages_count_kernel(PagesCompactArgs a) {
    __shared__ int lds[4];
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kSegment;
    const int used = used_in_segment(a.refs, first, min(first + kSegment, static_cast<int64_t>(a.num_blocks)), lds);
    if (threadIdx.x == 0) a.used_of[static_cast<int64_t>(blockIdx.x) * PagesWorkspace::kWords] = used;
}
// Three launches, bound by the ways to what the one in front has written: 300 requests on a pool of which 24000 blocks move 4.6, 5.1 and 5.4 us (the tables' 4 bytes an
// entry, one load behind the other, in the last), 6 requests 2.5, 3.9 and 2.8.
//
// Every workgroup has its segment's blocks, and finds from all segments' counts how many are in use, in front of it and in front of block U.
__global__ __launch_bounds__(256) void pages_move_kernel(PagesCompactArgs a) {
    __shared__ int lds[4];
    const int segments = gridDim.x, mine = blockIdx.x, tid = threadIdx.x;
    int of_all = 0, of_front = 0, used, front;
    for (int s = tid; s < segments; s += 256) {
        const int x = a.used_of[static_cast<int64_t>(s) * PagesWorkspace::kWords];
        of_all += x;
        of_front += s < mine ? x : 0;
    }
    sum_in_front<256>(of_all, lds, used);
    sum_in_front<256>(of_front, lds, front);
    const int cut = used / kSegment;                // segment of block U
    int of_cut = 0, low;
    for (int s = tid; s < min(cut, segments); s += 256) of_cut += a.used_of[static_cast<int64_t>(s) * PagesWorkspace::kWords];
    sum_in_front<256>(of_cut, lds, low);
    low += used_in_segment(a.refs, static_cast<int64_t>(cut) * kSegment, used, lds);           // in use below U
    const int moves = min(used - low, a.max_moves);
    for (int64_t k = moves + static_cast<int64_t>(mine) * 256 + tid; k < a.max_moves; k += static_cast<int64_t>(segments) * 256) {
        a.copy_src[k] = -1;
        a.copy_dst[k] = -1;
    }
    // The lists, block by block.  A block that moves does not know yet where to: its number in the list stands for the new number.
    const int64_t first = static_cast<int64_t>(mine) * kSegment + tid * kOfThread;
    int refs[kOfThread], count = 0, all;
    load_refs(a.refs, first, a.num_blocks, 0, refs);
#pragma unroll
    for (int e = 0; e < kOfThread; ++e) count += refs[e] > 0 ? 1 : 0;
    int before = front + sum_in_front<256>(count, lds, all);       // blocks in use in front of this one
#pragma unroll
    for (int e = 0; e < kOfThread; ++e) {
        const int64_t b = first + e;
        if (b >= a.num_blocks) break;
        const bool in_use = refs[e] > 0;
        const bool goes = b >= used && in_use && before - low < moves;
        if (goes) a.copy_src[before - low] = static_cast<int32_t>(b);
        if (b < used && !in_use && b - before < moves) a.copy_dst[b - before] = static_cast<int32_t>(b);
        a.to[place_of(b)] = goes ? -1 - (before - low) : static_cast<int32_t>(b);
        a.new_refs[b] = goes ? 0 : refs[e];
        before += in_use ? 1 : 0;
    }
}
// A wave for kOfRow entries of a request (as above), or for the counts of 64 blocks that moved
__global__ __launch_bounds__(256) void pages_rename_kernel(PagesCompactArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (unit >= a.n) {
        if (blockIdx.y > 0) return;
        const int64_t k = (unit - a.n) * kWave + lane;
        if (k < a.max_moves && a.copy_src[k] >= 0) a.new_refs[a.copy_dst[k]] = a.refs[a.copy_src[k]];
        return;
    }
    const int pages = min(max(a.pages[unit], 0), a.max_blocks);
    const int64_t row = unit * a.max_blocks;
    for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * kOfRow + lane; j0 < pages; j0 += static_cast<int64_t>(gridDim.y) * kOfRow) {
        int b[kAtOnce], to[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) b[e] = a.table[row + min(j0 + e * kWave, static_cast<int64_t>(pages) - 1)];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) to[e] = is_block(b[e], a.num_blocks) ? a.to[place_of(b[e])] : 0;
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) to[e] = !is_block(b[e], a.num_blocks) ? b[e] : to[e] < 0 ? a.copy_dst[-1 - to[e]] : to[e];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) if (j0 + e * kWave < pages) a.new_table[row + j0 + e * kWave] = to[e];
    }
}

// ------------------------------------------------------------------ copies of blocks
// A wave for (block, keys or values, part of them); the scales go with the first part of the values.  Bound by memory: 24000 blocks of 33 KB (16 tokens of 8 heads of 128 columns in 8 bits)
// 300 to 320 us, 5.0 to 5.3 TB/s read and written together (a copy of 2 GiB: 4.9).  By workgroups, a block or a part of it each: the same there, but 24000 blocks of 4 KB 37 us instead of 26
// and of 2 KB 34 instead of 17.5, 32 blocks of 1 MB 19 instead of 13.  With parts for 1024 waves 32 of these 15; for 16384 1024 blocks of 33 KB 14.6 instead of 13.9.
__global__ __launch_bounds__(256) void cache_copy_kernel(CacheCopyArgs a) {
    const CacheView &f = a.from, &t = a.to;
    const int lane = threadIdx.x & 63;
    const int64_t rows = static_cast<int64_t>(f.Hkv) * f.page, units = 2 * static_cast<int64_t>(a.count) * a.parts;
    const int64_t words = rows * f.d * (f.f8 ? 1 : 2) / 16, each = (words + a.parts - 1) / a.parts, scales = f.f8 ? rows * 2 / 16 : 0;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units; u += 4 * static_cast<int64_t>(gridDim.x)) {
        const int64_t pair = u / a.parts, i = pair >> 1, part = u - pair * a.parts;
        const bool values = pair & 1;
        const int src = a.src[i], dst = a.dst[i];
        if (src < 0 || src >= f.num_blocks || dst < 0 || dst >= t.num_blocks || (src == dst && f.k == t.k)) continue;
        const u32x4* x = static_cast<const u32x4*>(values ? f.v : f.k) + src * words;
        u32x4* y = static_cast<u32x4*>(values ? t.v : t.k) + dst * words;
        if (values && part == 0) {
            const u32x4* xs = reinterpret_cast<const u32x4*>(f.scales) + src * scales;
            u32x4* ys = reinterpret_cast<u32x4*>(t.scales) + dst * scales;
            for (int64_t w = lane; w < scales; w += 64) ys[w] = xs[w];
        }
        const int64_t end = min(words, (part + 1) * each);
        int64_t w = part * each + lane;
        constexpr int AT_ONCE = 4;
        for (; w + (AT_ONCE - 1) * 64 < end; w += AT_ONCE * 64) {
            u32x4 r[AT_ONCE];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) r[e] = x[w + e * 64];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) y[w + e * 64] = r[e];
        }
        u32x4 r[AT_ONCE - 1];
#pragma unroll
        for (int e = 0; e < AT_ONCE - 1; ++e) if (w + e * 64 < end) r[e] = x[w + e * 64];
#pragma unroll
        for (int e = 0; e < AT_ONCE - 1; ++e) if (w + e * 64 < end) y[w + e * 64] = r[e];
    }
}

unsigned groups_of(const int64_t units, const int64_t each) { return static_cast<unsigned>((units + each - 1) / each); }
unsigned parts_of_row(const int max_blocks) { return groups_of(max_blocks < 64 * kOfRow ? max_blocks : 64 * kOfRow, kOfRow); }

}  // namespace

int launch_pages_select(const PagesSelectArgs& a, void* stream) {
    hipLaunchKernelGGL(pages_select_kernel, dim3(groups_of(static_cast<int64_t>(a.n) + a.n_new, 4), parts_of_row(a.max_blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_reserve(const PagesReserveArgs& a, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.n <= kPlanThreads) {
        hipLaunchKernelGGL((pages_plan_kernel<true>), dim3(1), dim3(kPlanThreads), 0, st, a);
        return static_cast<int>(hipGetLastError());
    }
    hipLaunchKernelGGL((pages_plan_kernel<false>), dim3(1), dim3(kPlanThreads), 0, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return static_cast<int>(e);
    hipLaunchKernelGGL(pages_apply_kernel, dim3(groups_of(a.n, 4)), dim3(256), 0, st, a);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_compact(const PagesCompactArgs& a, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned segments = groups_of(a.num_blocks, kSegment);
    hipLaunchKernelGGL(pages_count_kernel, dim3(segments), dim3(256), 0, st, a);
    hipLaunchKernelGGL(pages_move_kernel, dim3(segments), dim3(256), 0, st, a);
    const int64_t waves = a.n + (static_cast<int64_t>(a.max_moves) + kWave - 1) / kWave;
    if (waves > 0) hipLaunchKernelGGL(pages_rename_kernel, dim3(groups_of(waves, 4), a.max_blocks > 0 ? parts_of_row(a.max_blocks) : 1), dim3(256), 0, st, a);
    return static_cast<int>(hipGetLastError());
}

int launch_cache_copy(CacheCopyArgs a, void* stream) {
    const int64_t words = static_cast<int64_t>(a.from.Hkv) * a.from.page * a.from.d * (a.from.f8 ? 1 : 2) / 16;
    // parts: waves for the machine, of 256 words and more each
    const int64_t pairs = 2 * static_cast<int64_t>(a.count), parts = (4096 + pairs - 1) / pairs, most = (words + 255) / 256;
    a.parts = static_cast<int>(parts < most ? parts : most);
    const int64_t groups = (pairs * a.parts + 3) / 4;
    hipLaunchKernelGGL(cache_copy_kernel, dim3(static_cast<unsigned>(groups < 65536 ? groups : 65536)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace pk
