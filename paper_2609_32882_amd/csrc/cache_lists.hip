// The page lists of the paged 8-bit cache: which pages every sequence's list holds,
// how often a page is held, and copies of tokens between lists.
//
// Assigning lists is index work, bound by the latency of launches and of steps that wait
// for one another, unless pages are copied.  Where lists move, one launch saves the old
// lists and gives up their pages, a second writes the new ones; a single workgroup then
// settles who copies a shared last page, numbers the requests for pages in order of the
// sequences, and hands out the free pages in order of their index; the last launch copies
// pages.  Counts are changed with whole-number atomics, whose order is of no
// consequence; every choice goes by indices.
#include <algorithm>

#include "common.hpp"

namespace vsa2 {

namespace {

constexpr int NT = 1024;                 // threads of the planning workgroup
constexpr int PER = 16;                  // pages a thread looks at in a step
constexpr int STEP = NT * PER;           // pages of a step
constexpr int LONE_STEPS = 4;            // steps that one workgroup takes alone
constexpr int LONE_ENTRIES = 8192;       // list entries that it trims by itself
constexpr int FINDERS = 4096;            // sequences whose request numbers it keeps in LDS

enum last_page { NONE, KEEPS, COPIES, STUCK };      // what a sequence does about its shared last page

// Per sequence: pages kept, requests before it, pages wanted behind the kept ones, last_page,
// its page, the copy's page.
struct seq_info {
    int kept, base, wanted, last, page, copy;
};

struct assign_args {
    cache_view c;
    int32_t* table;
    int32_t* refs;
    const int32_t *length, *source, *drop, *count;
    int32_t* room;
    int32_t* old;            // [batch][max_pages]
    seq_info* info;          // [batch]
    int32_t* free_pages;     // of each step
    int32_t* totals;         // requests, free pages
    bool trims, lone;        // the planning workgroup trims the lists; it hands out the pages
};

__device__ __forceinline__ bool is_page(const assign_args& a, int e) { return e >= 0 && e < a.c.pages; }
__device__ __forceinline__ int source_of(const assign_args& a, int b) { return a.source ? a.source[b] : b; }

// Tokens and pages that sequence b keeps.
__device__ __forceinline__ int64_t kept_tokens(const assign_args& a, int b) {
    const int src = source_of(a, b);
    if (src < 0 || src >= a.c.batch) return 0;
    const int64_t most = static_cast<int64_t>(a.c.max_pages) * CACHE_TOKENS, n = a.length[b];
    return n < 0 ? 0 : (n > most ? most : n);
}
__device__ __forceinline__ int pages_of(int64_t tokens) { return static_cast<int>((tokens + CACHE_TOKENS - 1) / CACHE_TOKENS); }

// Where entry s of sequence b's new list comes from, -1 for nowhere.
struct entry_source {
    int src, at;
    bool stays;          // the same place of the same list
};
__device__ __forceinline__ entry_source entry_of(const assign_args& a, int b, int s) {
    if (s >= pages_of(kept_tokens(a, b))) return {0, -1, false};
    const int src = source_of(a, b);
    int64_t at = s;
    if (a.drop && s >= a.drop[2 * b]) at += max(a.drop[2 * b + 1], 0);
    return {src, at < a.c.max_pages ? static_cast<int>(at) : -1, src == b && at == s};
}

__device__ __forceinline__ int held(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The old lists are saved and, where an entry does not stay, its page is given up.
__global__ __launch_bounds__(256) void lists_save_kernel(assign_args a) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < all; x += static_cast<int64_t>(gridDim.x) * 256) {
        const int b = static_cast<int>(x / a.c.max_pages), s = static_cast<int>(x - static_cast<int64_t>(b) * a.c.max_pages);
        const int e = a.table[x];
        a.old[x] = e;
        if (is_page(a, e) && !entry_of(a, b, s).stays) atomicAdd(a.refs + e, -1);
    }
}
__global__ __launch_bounds__(256) void lists_write_kernel(assign_args a) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < all; x += static_cast<int64_t>(gridDim.x) * 256) {
        const int b = static_cast<int>(x / a.c.max_pages), s = static_cast<int>(x - static_cast<int64_t>(b) * a.c.max_pages);
        const entry_source from = entry_of(a, b, s);
        int e = from.at < 0 ? -1 : a.old[static_cast<int64_t>(from.src) * a.c.max_pages + from.at];
        if (!is_page(a, e)) e = -1;
        a.table[x] = e;
        if (e >= 0 && !from.stays) atomicAdd(a.refs + e, 1);
    }
}

// Lists that all stay: pages behind the kept ones are given up.
__device__ __forceinline__ void trim(const assign_args& a, int64_t first, int64_t step) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = first; x < all; x += step) {
        const int b = static_cast<int>(x / a.c.max_pages), s = static_cast<int>(x - static_cast<int64_t>(b) * a.c.max_pages);
        const int e = a.table[x];
        const bool page = is_page(a, e);
        if (s < pages_of(kept_tokens(a, b))) {
            if (!page && e != -1) a.table[x] = -1;
            continue;
        }
        if (page) atomicAdd(a.refs + e, -1);
        if (e != -1) a.table[x] = -1;
    }
}
__global__ __launch_bounds__(256) void lists_trim_kernel(assign_args a) {
    trim(a, static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, static_cast<int64_t>(gridDim.x) * 256);
}

// Exclusive prefix over the workgroup's threads, and the total.
__device__ __forceinline__ int prefix(int x, int* sums, int& total) {
    const int lane = lane_id(), wave = wave_id();
    int y = x;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int z = __shfl_up(y, k, 64);
        if (lane >= k) y += z;
    }
    if (lane == 63) sums[wave] = y;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    __syncthreads();
    return before + y - x;
}

// Who copies its last page, and every sequence's first request.  A sequence that writes into
// a kept page takes itself off the page's count; where nobody else is left, the last of
// them (by index) keeps it, the others need copies.
__device__ void plan_requests(const assign_args& a, int* sums, int* bases) {
    const int tid = threadIdx.x, batch = a.c.batch;
    for (int b = tid; b < batch; b += NT) {
        const int64_t n = kept_tokens(a, b), count = a.count ? max(a.count[b], 0) : 0;
        seq_info w{pages_of(n), 0, 0, NONE, -1, -1};
        const int64_t end = (n + count + CACHE_TOKENS - 1) / CACHE_TOKENS;
        w.wanted = static_cast<int>(min(end, static_cast<int64_t>(a.c.max_pages))) - w.kept;
        if (count > 0 && n % CACHE_TOKENS) {
            w.page = a.table[static_cast<int64_t>(b) * a.c.max_pages + w.kept - 1];
            w.last = w.page < 0 ? STUCK : KEEPS;
            if (w.page >= 0) atomicAdd(a.refs + w.page, -1);
        }
        a.info[b] = w;
    }
    __syncthreads();
    for (int b = tid; b < batch; b += NT)
        if (a.info[b].last == KEEPS && held(a.refs + a.info[b].page) <= 0) atomicMin(a.refs + a.info[b].page, -(b + 1));
    __syncthreads();
    for (int b = tid; b < batch; b += NT)
        if (a.info[b].last == KEEPS && held(a.refs + a.info[b].page) != -(b + 1)) a.info[b].last = COPIES;
    __syncthreads();
    int all = 0;
    for (int b0 = 0; b0 < batch; b0 += NT) {
        const int b = b0 + tid;
        int need = 0;
        if (b < batch) {
            if (a.info[b].last == KEEPS) __hip_atomic_store(a.refs + a.info[b].page, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            need = a.info[b].wanted + (a.info[b].last == COPIES ? 1 : 0);
        }
        int total;
        const int base = all + prefix(need, sums, total);
        if (b < batch) {
            a.info[b].base = base;
            if (batch <= FINDERS) bases[b] = base;
        }
        all += total;
    }
    if (tid == 0) a.totals[0] = all;
    __syncthreads();
    __threadfence();         // the counts below are read past what this CU may hold of them
}

// Sixteen counts from page p0 on: a bit for each free page.
__device__ __forceinline__ uint32_t free_bits(const assign_args& a, int64_t p0) {
    uint32_t bits = 0;
    if (p0 + PER <= a.c.pages) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const int4 r = *reinterpret_cast<const int4*>(a.refs + p0 + i);
            bits |= (r.x == 0 ? 1u : 0u) << i | (r.y == 0 ? 2u : 0u) << i | (r.z == 0 ? 4u : 0u) << i | (r.w == 0 ? 8u : 0u) << i;
        }
    } else {
        for (int i = 0; i < PER; ++i)
            if (p0 + i < a.c.pages && a.refs[p0 + i] == 0) bits |= 1u << i;
    }
    return bits;
}

// Hands the free pages of `bits`, the first of which is number `rank`, to the requests.
__device__ __forceinline__ void hand_out(const assign_args& a, int64_t p0, uint32_t bits, int64_t rank, int requests,
                                         const int* bases) {
    for (; bits && rank < requests; ++rank) {
        const int i = __builtin_ctz(bits);
        bits &= bits - 1;
        const int page = static_cast<int>(p0 + i);
        int lo = 0, hi = a.c.batch - 1;           // the last sequence whose first request is not past it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((bases ? bases[mid] : a.info[mid].base) <= rank) lo = mid;
            else hi = mid - 1;
        }
        const seq_info w = a.info[lo];
        const int nth = static_cast<int>(rank) - w.base - (w.last == COPIES ? 1 : 0);
        if (nth < 0) a.info[lo].copy = page;
        else a.table[static_cast<int64_t>(lo) * a.c.max_pages + w.kept + nth] = page;
        a.refs[page] = 1;
    }
}

// What the requests got.  Sequences whose copy was refused are holders of the page again, and then
// nobody may write into it.
__device__ void finish(const assign_args& a, int64_t found) {
    const int tid = threadIdx.x, batch = a.c.batch;
    for (int b = tid; b < batch; b += NT) {
        const seq_info w = a.info[b];
        if (w.last != COPIES) continue;
        if (w.base < found) a.table[static_cast<int64_t>(b) * a.c.max_pages + w.kept - 1] = w.copy;
        else atomicAdd(a.refs + w.page, 1);
    }
    __syncthreads();
    for (int b = tid; a.room && b < batch; b += NT) {
        const seq_info w = a.info[b];
        const int64_t count = a.count ? max(a.count[b], 0) : 0, n = kept_tokens(a, b);
        const int copies = w.last == COPIES ? 1 : 0;
        const int64_t left = found - w.base - copies;
        const int64_t got = left < 0 ? 0 : (left < w.wanted ? left : w.wanted);
        int64_t room = (w.kept + got) * CACHE_TOKENS - n;
        room = room < count ? room : count;
        const bool alone = w.last == NONE || (w.last == KEEPS && held(a.refs + w.page) <= 1) || (copies && w.base < found);
        a.room[b] = alone && room > 0 ? static_cast<int>(room) : 0;
    }
}

__global__ __launch_bounds__(NT) void lists_plan_kernel(assign_args a) {
    __shared__ int sums[NT / 64], bases[FINDERS];
    if (a.trims) {
        trim(a, threadIdx.x, NT);
        __syncthreads();
    }
    plan_requests(a, sums, bases);
    if (!a.lone) return;
    const int requests = a.totals[0];
    int found = 0;
    for (int64_t p0 = 0; p0 < a.c.pages && found < requests; p0 += STEP) {
        const int64_t mine = p0 + threadIdx.x * PER;
        const uint32_t bits = free_bits(a, mine);
        int total;
        const int rank = found + prefix(__popc(bits), sums, total);
        hand_out(a, mine, bits, rank, requests, a.c.batch <= FINDERS ? bases : nullptr);
        found += total;
    }
    __syncthreads();
    finish(a, found);
}

// Large pools: a workgroup for every step, which counts its free pages first.
__global__ __launch_bounds__(NT) void lists_count_kernel(assign_args a) {
    __shared__ int sums[NT / 64];
    int total;
    prefix(__popc(free_bits(a, static_cast<int64_t>(blockIdx.x) * STEP + threadIdx.x * PER)), sums, total);
    if (threadIdx.x == 0) a.free_pages[blockIdx.x] = total;
}
__device__ __forceinline__ int64_t free_before(const assign_args& a, int steps, int* sums) {
    int mine = 0, total;             // pages are 31 bits, so is their sum
    for (int i = threadIdx.x; i < steps; i += NT) mine += a.free_pages[i];
    prefix(mine, sums, total);
    return total;
}
__global__ __launch_bounds__(NT) void lists_hand_kernel(assign_args a) {
    __shared__ int sums[NT / 64];
    const int64_t before = free_before(a, blockIdx.x, sums);
    const int requests = a.totals[0];
    if (before >= requests) return;
    const int64_t mine = static_cast<int64_t>(blockIdx.x) * STEP + threadIdx.x * PER;
    const uint32_t bits = free_bits(a, mine);
    int total;
    const int64_t rank = before + prefix(__popc(bits), sums, total);
    hand_out(a, mine, bits, rank, requests, nullptr);
}
__global__ __launch_bounds__(NT) void lists_finish_kernel(assign_args a, int steps) {
    __shared__ int sums[NT / 64];
    finish(a, free_before(a, steps, sums));
}

// Pages that got a copy: 16 KB a workgroup.
constexpr int COPY_BYTES = 16384;
__global__ __launch_bounds__(256) void lists_copy_kernel(assign_args a, int64_t page_bytes) {
    const seq_info w = a.info[blockIdx.x];
    if (w.last != COPIES || w.copy < 0) return;
    const int64_t at = static_cast<int64_t>(blockIdx.y) * COPY_BYTES;
    const int n = static_cast<int>(min(static_cast<int64_t>(COPY_BYTES), page_bytes - at) / 16);
    const uint4* from = reinterpret_cast<const uint4*>(a.c.pool + w.page * page_bytes + at);
    uint4* to = reinterpret_cast<uint4*>(a.c.pool + w.copy * page_bytes + at);
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) to[i] = from[i];
}

int64_t steps_of(int pages) { return (static_cast<int64_t>(pages) + STEP - 1) / STEP; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// ---------------------------------------------------------------------------
// Tokens from lists to lists.  A workgroup takes one page of one KV head of the
// written list; where each of its tokens comes from is worked out once.
// ---------------------------------------------------------------------------
struct move_args {
    cache_view from, to;
    const int32_t *index, *start, *count;
    int n, chunks;
};

constexpr uint32_t ZERO_POWER = 27;      // 2^-100, as a row of zeros is written

__device__ __forceinline__ const char* page_of(const cache_view& c, int b, int h, int64_t pos, int D) {
    if (pos < 0 || pos >= static_cast<int64_t>(c.max_pages) * CACHE_TOKENS) return nullptr;
    const int32_t* list = c.table + (static_cast<int64_t>(b) * c.table_heads + (c.table_heads > 1 ? h : 0)) * c.max_pages;
    const int e = list[pos / CACHE_TOKENS];
    return e >= 0 && e < c.pages ? c.pool + (static_cast<int64_t>(e) * c.heads + h) * cache_page_bytes(D) : nullptr;
}

template <int D>
__global__ __launch_bounds__(256) void cache_move_kernel(move_args a) {
    __shared__ const char* page[64];     // where each token is: its page, place in it; live: is it written
    __shared__ int place[64];
    const int64_t item = blockIdx.x;
    const int chunk = static_cast<int>(item % a.chunks);
    const int64_t bh = item / a.chunks;
    const int b = static_cast<int>(bh / a.to.heads), h = static_cast<int>(bh % a.to.heads);
    const int tid = threadIdx.x;
    const int cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const int64_t start = a.start[b];
    // the page's first position: pages from the one that holds position `start` on
    const int64_t first_page = start >= 0 ? start / CACHE_TOKENS : -((-start + CACHE_TOKENS - 1) / CACHE_TOKENS);
    const int64_t pos0 = (first_page + chunk) * CACHE_TOKENS;
    if (pos0 >= start + cnt) return;
    char* to = const_cast<char*>(page_of(a.to, b, h, pos0, D));
    if (!to) return;
    const int lo = static_cast<int>(max(start - pos0, static_cast<int64_t>(0)));
    const int hi = static_cast<int>(min(start + cnt - pos0, static_cast<int64_t>(64)));
    if (tid < 64) {
        const char* p = nullptr;
        int j = 0;
        if (tid >= lo && tid < hi) {
            const int from = a.index[static_cast<int64_t>(b) * a.n + (pos0 + tid - start)];
            p = page_of(a.from, b, h, from, D);
            j = from & 63;
        }
        page[tid] = p;
        place[tid] = j;
    }
    __syncthreads();
    // keys: 16 bytes are one token's
    for (int u = tid; u < 4 * D; u += 256) {
        const int r = u & 15, t = u / D, rest = u & (D - 1) & ~15, j = 16 * t + r;
        if (j < lo || j >= hi) continue;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (page[j]) w = reinterpret_cast<const uint4*>(page[j])[place[j] / 16 * D + rest + (place[j] & 15)];
        reinterpret_cast<uint4*>(to)[u] = w;
    }
    // values: a dword is four tokens' of one element
    for (int u = tid; u < 16 * D; u += 256) {
        const int t = u & 3, el = u >> 2 & 15, g = u >> 6 & 3, c = u >> 8, j0 = 16 * t + 4 * g;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const char* p = page[j0 + i];
            const int j = place[j0 + i];
            if (p) w |= static_cast<uint32_t>(static_cast<uint8_t>(p[64 * D + ((c * 4 + (j >> 2 & 3)) * 16 + el) * 16 + (j >> 4) * 4 + (j & 3)])) << (8 * i);
        }
        char* out = to + 64 * D + 4 * u;
        if (j0 >= lo && j0 + 4 <= hi) {
            *reinterpret_cast<uint32_t*>(out) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j0 + i >= lo && j0 + i < hi) out[i] = static_cast<char>(w >> (8 * i));
        }
    }
    // powers
    if (tid < 128) {
        const bool values = tid >= 64;
        const int x = tid & 63, j = values ? 16 * (x >> 2 & 3) + 4 * (x >> 4) + (x & 3) : 16 * (x & 3) + (x >> 2);
        if (j >= lo && j < hi) {
            const char* p = page[j];
            const int s = place[j], at = values ? 64 + (s >> 2 & 3) * 16 + (s >> 4) * 4 + (s & 3) : (s & 15) * 4 + (s >> 4);
            to[128 * D + tid] = p ? p[128 * D + at] : static_cast<char>(ZERO_POWER);
        }
    }
}

}  // namespace

size_t cache_assign_workspace_bytes(const cache_view& c) {
    return up256(static_cast<size_t>(c.batch) * c.max_pages * sizeof(int32_t)) + up256(static_cast<size_t>(c.batch) * sizeof(seq_info)) +
           up256(static_cast<size_t>(steps_of(c.pages)) * sizeof(int32_t)) + 256;
}

hipError_t launch_cache_assign(int D, const cache_view& c, int32_t* table, int32_t* refs, const int32_t* length,
                               const int32_t* source, const int32_t* drop, const int32_t* count, int32_t* room,
                               void* ws, hipStream_t s) {
    assign_args a{};
    a.c = c;
    a.table = table;
    a.refs = refs;
    a.length = length;
    a.source = source;
    a.drop = drop;
    a.count = count;
    a.room = room;
    char* w = static_cast<char*>(ws);
    a.old = reinterpret_cast<int32_t*>(w);
    w += up256(static_cast<size_t>(c.batch) * c.max_pages * sizeof(int32_t));
    a.info = reinterpret_cast<seq_info*>(w);
    w += up256(static_cast<size_t>(c.batch) * sizeof(seq_info));
    a.free_pages = reinterpret_cast<int32_t*>(w);
    w += up256(static_cast<size_t>(steps_of(c.pages)) * sizeof(int32_t));
    a.totals = reinterpret_cast<int32_t*>(w);
    const int64_t entries = static_cast<int64_t>(c.batch) * c.max_pages, steps = steps_of(c.pages);
    const dim3 wide(static_cast<unsigned>(std::min<int64_t>((entries + 255) / 256, 4096)));
    a.lone = steps <= LONE_STEPS;
    if (source || drop) {
        hipLaunchKernelGGL(lists_save_kernel, wide, dim3(256), 0, s, a);
        hipLaunchKernelGGL(lists_write_kernel, wide, dim3(256), 0, s, a);
    } else if (entries <= LONE_ENTRIES) {
        a.trims = true;
    } else {
        hipLaunchKernelGGL(lists_trim_kernel, wide, dim3(256), 0, s, a);
    }
    hipLaunchKernelGGL(lists_plan_kernel, dim3(1), dim3(NT), 0, s, a);
    if (!a.lone) {
        hipLaunchKernelGGL(lists_count_kernel, dim3(static_cast<unsigned>(steps)), dim3(NT), 0, s, a);
        hipLaunchKernelGGL(lists_hand_kernel, dim3(static_cast<unsigned>(steps)), dim3(NT), 0, s, a);
        hipLaunchKernelGGL(lists_finish_kernel, dim3(1), dim3(NT), 0, s, a, static_cast<int>(steps));
    }
    if (count) {
        const int64_t bytes = c.heads * cache_page_bytes(D);
        const dim3 grid(static_cast<unsigned>(c.batch), static_cast<unsigned>((bytes + COPY_BYTES - 1) / COPY_BYTES));
        hipLaunchKernelGGL(lists_copy_kernel, grid, dim3(256), 0, s, a, bytes);
    }
    return hipGetLastError();
}

hipError_t launch_cache_move(int D, const cache_view& from, const cache_view& to, int n, const int32_t* index,
                             const int32_t* start, const int32_t* count, hipStream_t s) {
    move_args a{from, to, index, start, count, n, static_cast<int>((static_cast<int64_t>(n) + 62) / 64 + 1)};
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(to.batch) * to.heads * a.chunks));
    if (D == 64) hipLaunchKernelGGL((cache_move_kernel<64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_move_kernel<128>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace vsa2
