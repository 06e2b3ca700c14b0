// The page lists of the paged 8-bit cache: which pages every sequence's list holds,
// how often a page is held, and copies of tokens between lists.
//
// Assigning lists is index work, bound by the latency of launches and of loads that wait
// for one another, unless pages are copied.  One workgroup does it where lists are short, in
// its LDS: it saves the old lists, gives up their pages, writes the new lists, settles who
// copies a shared last page, numbers the requests for pages in order of the sequences, and
// hands out the free pages in order of their index; a second launch copies pages.  Longer
// lists are moved by launches of their own, larger pools searched by a workgroup for every
// 16,384 pages.  Counts are changed with whole-number atomics, whose order is of no
// consequence; every choice goes by indices.  64 lists of up to 33 pages that get a token each:
// 9.3 us (14.4 in memory instead of LDS); 8 lists of 600 that lose and get 60: 11.3 (22.8);
// 32 lists of 280 pages forked from 8, 24 pages copied: 16.7.
#include <algorithm>

#include "common.hpp"

namespace vsa2 {

namespace {

constexpr int NT = 1024;                 // threads of the planning workgroup
constexpr int PER = 16;                  // pages a thread looks at in a step
constexpr int STEP = NT * PER;           // pages of a step
// One workgroup alone against several launches, us a call with a token for every list, in pools with
// room at their start: 64 lists of 32, 48, 64, 128 and 384 pages that stay 8.9 9.1 10.0 13.2 26.2
// against 9.6 9.3 9.7 10.7 15.2; that take others' lists, of 32, 64, 80, 96 and 128 pages 9.9 11.2 11.5
// 12.4 13.8 against 11.4 12.2 12.2 12.4 13.0; that lose pages, of 96 and 128 11.7 13.3 against 12.6 13.4;
// both, of 96 and 128 12.5 13.9 against 14.3 14.8.
constexpr int LONE_TRIMS = 3400;         // list entries of a workgroup alone where they stay in their places
constexpr int LONE_ENTRIES = 6144;       // and where lists take others' or lose pages
// Free pages at the end of pools of 4, 5, 8 and 16 steps: 17.2 19.6 26.7 45.4 by a workgroup alone, against
// 17.5 18.4 18.5 18.1 with a workgroup for every step.
constexpr int LONE_STEPS = 4;            // steps that one workgroup searches alone

enum last_page { NONE, KEEPS, COPIES, STUCK };      // what a sequence does about its shared last page

// Per sequence: pages kept, requests before it, pages wanted behind the kept ones, last_page,
// its page, the copy's page, places left in the kept pages, tokens to make room for.
struct seq_info {
    int kept, base, wanted, last, page, copy, slack, count;
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
    int32_t* totals;         // requests
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

// What becomes of a sequence's list.
struct list_move {
    int kept, src, first, num;
    // where new entry s comes from, -1 for nowhere
    __device__ __forceinline__ int from(int s, int max_pages) const {
        const int64_t at = s + (s >= first ? static_cast<int64_t>(num) : 0);
        return s < kept && at < max_pages ? static_cast<int>(at) : -1;
    }
    // does old entry s stay in the list (at any place)?
    __device__ __forceinline__ bool retains(int b, int s) const {
        if (src != b) return false;
        return s < first ? s < kept : s - static_cast<int64_t>(first) >= num && s - static_cast<int64_t>(num) < kept;
    }
};
__device__ __forceinline__ list_move move_of(const assign_args& a, int b) {
    list_move w{pages_of(kept_tokens(a, b)), source_of(a, b), 0, 0};
    if (a.drop) {
        w.first = max(a.drop[2 * b], 0);
        w.num = max(a.drop[2 * b + 1], 0);
    }
    return w;
}

__device__ __forceinline__ int held(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The old lists are saved, and the pages that leave them given up.
__global__ __launch_bounds__(256) void lists_save_kernel(assign_args a) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < all; x += static_cast<int64_t>(gridDim.x) * 256) {
        const int b = static_cast<int>(x / a.c.max_pages), s = static_cast<int>(x - static_cast<int64_t>(b) * a.c.max_pages);
        const int e = a.table[x];
        a.old[x] = e;
        if (is_page(a, e) && !move_of(a, b).retains(b, s)) atomicAdd(a.refs + e, -1);
    }
}
__global__ __launch_bounds__(256) void lists_write_kernel(assign_args a) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < all; x += static_cast<int64_t>(gridDim.x) * 256) {
        const int b = static_cast<int>(x / a.c.max_pages), s = static_cast<int>(x - static_cast<int64_t>(b) * a.c.max_pages);
        const list_move w = move_of(a, b);
        const int at = w.from(s, a.c.max_pages);
        int e = at < 0 ? -1 : a.old[static_cast<int64_t>(w.src) * a.c.max_pages + at];
        if (!is_page(a, e)) e = -1;
        a.table[x] = e;
        if (e >= 0 && w.src != b) atomicAdd(a.refs + e, 1);
    }
}

// Lists that go on from others' without losing pages: entries stay in their columns, so a workgroup
// that holds some columns of all lists saves and writes them in one launch.  With 128 workgroups at
// least, where there are as many columns, against saved and written lists (us): 64 lists of 100, 200
// and 512 pages 12.8 14.2 13.3 against 14.4 16.1 15.0, 32 of 2,000 14.2 against 15.1, 4 of 8,000 10.8
// against 13.6, but 500 of 40 18.3 against 17.4; 512 workgroups 12.8 15.9 18.4, 14.7, 11.2, 32 of them
// 11.8 14.7 16.9, 20.4, 14.2.
constexpr int COLUMN_ENTRIES = 8192;
__global__ __launch_bounds__(256) void lists_columns_kernel(assign_args a, int columns) {
    __shared__ int old[COLUMN_ENTRIES];
    const int s0 = blockIdx.x * columns, n = min(columns, a.c.max_pages - s0), all = a.c.batch * n;
    for (int x = threadIdx.x; x < all; x += 256) old[x] = a.table[static_cast<int64_t>(x / n) * a.c.max_pages + s0 + x % n];
    __syncthreads();
    for (int x = threadIdx.x; x < all; x += 256) {
        const int b = x / n, i = x - b * n, s = s0 + i, was = old[x];
        const list_move w = move_of(a, b);
        int e = s < w.kept ? old[w.src * n + i] : -1;
        if (!is_page(a, e)) e = -1;
        if (is_page(a, was) && !w.retains(b, s)) atomicAdd(a.refs + was, -1);
        if (e >= 0 && w.src != b) atomicAdd(a.refs + e, 1);
        if (e != was) a.table[static_cast<int64_t>(b) * a.c.max_pages + s] = e;
    }
}

// Lists that all stay: pages behind the kept ones are given up.
__global__ __launch_bounds__(256) void lists_trim_kernel(assign_args a) {
    const int64_t all = static_cast<int64_t>(a.c.batch) * a.c.max_pages;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < all; x += static_cast<int64_t>(gridDim.x) * 256) {
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

// Inclusive sum over a wave's lanes up to each lane.
__device__ __forceinline__ int wave_prefix(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // rows of 16 lanes: 1, 2, 4, 8 back
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // a row's last lane to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);       // the first half's to the second
    return x;
}

// Exclusive prefix over the workgroup's threads, and the total.  One barrier: calls that follow each
// other take turns with two arrays of sums.
struct wg_sums {
    int of[2][NT / 64];
};
__device__ __forceinline__ int prefix(int x, wg_sums& sums, int turn, int& total) {
    const int y = wave_prefix(x);
    int (&mine)[NT / 64] = sums.of[turn & 1];
    if (lane_id() == 63) mine[wave_id()] = y;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int z = mine[w];
        before += w < wave_id() ? z : 0;
        total += z;
    }
    return before + y - x;
}

// A sequence before its requests are numbered; its last page follows where it writes into one
// (`inside`).
__device__ __forceinline__ seq_info info_of(const assign_args& a, int b, bool& inside) {
    const int count = a.count ? max(a.count[b], 0) : 0;
    const int64_t n = kept_tokens(a, b), end = (n + count + CACHE_TOKENS - 1) / CACHE_TOKENS;
    seq_info w{pages_of(n), 0, 0, NONE, -1, -1, static_cast<int>(-n & (CACHE_TOKENS - 1)), count};
    w.wanted = static_cast<int>(min(end, static_cast<int64_t>(a.c.max_pages))) - w.kept;
    inside = count > 0 && w.slack > 0;
    if (inside) w.last = STUCK;
    return w;
}

// Who copies its last page, and every sequence's first request; returns all requests.  A sequence
// that writes into a kept page which others hold, too, takes itself off the page's count; where
// nobody else is left, the last of them (by index) keeps it, the others need copies.  No count
// becomes 0 or stops being 0 here.
__device__ __forceinline__ int plan_requests(const assign_args& a, seq_info* info, wg_sums& sums) {
    const int tid = threadIdx.x, batch = a.c.batch;
    bool shared = false;
    for (int b = tid; b < batch; b += NT) {
        const int page = info[b].page;
        if (page < 0) continue;
        const bool copies = held(a.refs + page) != 1;
        info[b].last = copies ? COPIES : KEEPS;
        shared |= copies;
    }
    if (__syncthreads_or(shared)) {
        for (int b = tid; b < batch; b += NT)
            if (info[b].last == COPIES) atomicAdd(a.refs + info[b].page, -1);
        __syncthreads();
        for (int b = tid; b < batch; b += NT)
            if (info[b].last == COPIES && held(a.refs + info[b].page) <= 0) atomicMin(a.refs + info[b].page, -(b + 1));
        __syncthreads();
        for (int b = tid; b < batch; b += NT)
            if (info[b].last == COPIES && held(a.refs + info[b].page) == -(b + 1)) info[b].last = KEEPS;
        __syncthreads();
        for (int b = tid; b < batch; b += NT)
            if (info[b].last == KEEPS) __hip_atomic_store(a.refs + info[b].page, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    int all = 0;
    for (int b0 = 0, turn = 0; b0 < batch; b0 += NT, ++turn) {
        const int b = b0 + tid;
        const int need = b < batch ? info[b].wanted + (info[b].last == COPIES ? 1 : 0) : 0;
        int total;
        const int base = all + prefix(need, sums, turn, total);
        if (b < batch) info[b].base = base;
        all += total;
    }
    __syncthreads();         // the sums are free again
    return all;
}

// Sixteen counts from page p0 on, read past what this CU may hold of them; those past the
// pool as 1.
struct counts16 {
    uint64_t two[PER / 2];
};
__device__ __forceinline__ counts16 load_counts(const assign_args& a, int64_t p0) {
    counts16 c;
    if (p0 + PER <= a.c.pages) {
#pragma unroll
        for (int i = 0; i < PER / 2; ++i)
            c.two[i] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(a.refs + p0) + i, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
        return c;
    }
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
        c.two[i] = 0x0000000100000001ull;
        if (p0 + 2 * i + 1 < a.c.pages)
            c.two[i] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(a.refs + p0) + i, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
        else if (p0 + 2 * i < a.c.pages)
            c.two[i] = static_cast<uint32_t>(held(a.refs + p0 + 2 * i)) | 0x0000000100000000ull;
    }
    return c;
}
// A bit for each free page.
__device__ __forceinline__ uint32_t free_bits(const counts16& c) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < PER / 2; ++i)
        bits |= (static_cast<uint32_t>(c.two[i]) == 0 ? 1u : 0u) << (2 * i) | ((c.two[i] >> 32) == 0 ? 2u : 0u) << (2 * i);
    return bits;
}

// Gives a page to request number `rank`.
__device__ __forceinline__ void give(const assign_args& a, seq_info* info, int rank, int page) {
    int lo = 0, hi = a.c.batch - 1;           // the last sequence whose first request is not past it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (info[mid].base <= rank) lo = mid;
        else hi = mid - 1;
    }
    const seq_info w = info[lo];
    const int nth = rank - w.base - (w.last == COPIES ? 1 : 0);
    if (nth < 0) info[lo].copy = page;
    else a.table[static_cast<int64_t>(lo) * a.c.max_pages + w.kept + nth] = page;
    a.refs[page] = 1;
}

// Gives the free pages of a step, `before` of which come before it, to the requests; list: LDS for
// the step's free pages, so that every thread has a request.
__device__ __forceinline__ int give_step(const assign_args& a, seq_info* info, const counts16& counts, int64_t p0,
                                         int64_t before, int requests, wg_sums& sums, int* list) {
    const int64_t mine = p0 + threadIdx.x * PER;
    uint32_t bits = free_bits(counts);
    int total;
    int at = prefix(__popc(bits), sums, 0, total);
    for (; bits && before + at < requests; ++at) {
        list[at] = static_cast<int>(mine + __builtin_ctz(bits));
        bits &= bits - 1;
    }
    __syncthreads();
    const int64_t left = requests - before;
    for (int i = threadIdx.x; i < total && i < left; i += NT) give(a, info, static_cast<int>(before + i), list[i]);
    __syncthreads();
    return total;
}

// What the requests got.  Sequences whose copy was refused are holders of the page again, and then
// nobody may write into it.
__device__ __forceinline__ void finish(const assign_args& a, seq_info* info, int64_t found, int requests) {
    const int tid = threadIdx.x, batch = a.c.batch;
    bool refused = false;
    for (int b = tid; b < batch; b += NT) {
        const seq_info w = info[b];
        if (w.last != COPIES) continue;
        if (w.base < found) {
            a.table[static_cast<int64_t>(b) * a.c.max_pages + w.kept - 1] = w.copy;
        } else {
            atomicAdd(a.refs + w.page, 1);
            refused = true;
        }
    }
    if (found < requests) refused = __syncthreads_or(refused);
    for (int b = tid; a.room && b < batch; b += NT) {
        const seq_info w = info[b];
        const int copies = w.last == COPIES ? 1 : 0;
        const int64_t left = found - w.base - copies;
        const int got = static_cast<int>(left < 0 ? 0 : (left < w.wanted ? left : w.wanted));
        const int room = min(got * CACHE_TOKENS + w.slack, w.count);
        const bool alone = w.last == NONE || (copies && w.base < found) ||
                           (w.last == KEEPS && (!refused || held(a.refs + w.page) <= 1));
        a.room[b] = alone ? room : 0;
    }
}

// Up to NT sequences whose lists fit LDS, in a pool of LONE_STEPS steps: all but the copies.
__global__ __launch_bounds__(NT) void lists_alone_kernel(assign_args a) {
    __shared__ seq_info info[NT];
    __shared__ list_move moves[NT];
    __shared__ wg_sums sums;
    __shared__ int old[STEP];
    static_assert(LONE_ENTRIES <= STEP, "the lists' entries, then the free pages of a step");
    const int tid = threadIdx.x, m = a.c.max_pages, all = a.c.batch * m;
    const float per = 1.f / static_cast<float>(m);
    bool inside = false;
    for (int x = tid; x < all; x += NT) old[x] = a.table[x];
    if (tid < a.c.batch) {
        moves[tid] = move_of(a, tid);
        info[tid] = info_of(a, tid, inside);
    }
    __syncthreads();
    for (int x = tid; x < all; x += NT) {
        // x / m, off by at most 2^-22 of it: less than the half that is added is from a whole number
        const int b = static_cast<int>((static_cast<float>(x) + 0.5f) * per), s = x - b * m, was = old[x];
        const list_move w = moves[b];
        const int at = w.from(s, m);
        int e = at < 0 ? -1 : old[w.src * m + at];
        if (!is_page(a, e)) e = -1;
        if (is_page(a, was) && !w.retains(b, s)) atomicAdd(a.refs + was, -1);
        if (e >= 0 && w.src != b) atomicAdd(a.refs + e, 1);
        if (e != was) a.table[x] = e;
        if (s == w.kept - 1 && info[b].last == STUCK) info[b].page = e;
    }
    __syncthreads();
    counts16 counts = load_counts(a, tid * PER);        // under way while the requests are numbered
    const int requests = plan_requests(a, info, sums);
    int64_t found = 0;
    for (int64_t p0 = 0; p0 < a.c.pages && found < requests; p0 += STEP) {
        if (p0) counts = load_counts(a, p0 + tid * PER);
        found += give_step(a, info, counts, p0, found, requests, sums, old);
    }
    finish(a, info, found, requests);
    if (tid < a.c.batch) a.info[tid] = info[tid];
}

// Lists that other launches have moved: the pages, all of them (LONE) or in launches that follow.
template <bool LONE, bool FEW>
__global__ __launch_bounds__(NT) void lists_plan_kernel(assign_args a) {
    __shared__ seq_info own[FEW ? NT : 1];
    __shared__ wg_sums sums;
    __shared__ int list[LONE ? STEP : 1];
    seq_info* info = FEW ? own : a.info;
    counts16 counts = LONE ? load_counts(a, threadIdx.x * PER) : counts16{};
    for (int b = threadIdx.x; b < a.c.batch; b += NT) {
        bool inside;
        seq_info w = info_of(a, b, inside);
        if (inside) w.page = a.table[static_cast<int64_t>(b) * a.c.max_pages + w.kept - 1];
        info[b] = w;
    }
    const int requests = plan_requests(a, info, sums);
    if constexpr (LONE) {
        int64_t found = 0;
        for (int64_t p0 = 0; p0 < a.c.pages && found < requests; p0 += STEP) {
            if (p0) counts = load_counts(a, p0 + threadIdx.x * PER);
            found += give_step(a, info, counts, p0, found, requests, sums, list);
        }
        finish(a, info, found, requests);
        for (int b = threadIdx.x; FEW && b < a.c.batch; b += NT) a.info[b] = info[b];
    } else {
        if (threadIdx.x == 0) a.totals[0] = requests;
    }
}

// Large pools: a workgroup for every step, which counts its free pages first.
__global__ __launch_bounds__(NT) void lists_count_kernel(assign_args a) {
    __shared__ wg_sums sums;
    int total;
    prefix(__popc(free_bits(load_counts(a, static_cast<int64_t>(blockIdx.x) * STEP + threadIdx.x * PER))), sums, 0, total);
    if (threadIdx.x == 0) a.free_pages[blockIdx.x] = total;
}
__device__ __forceinline__ int64_t free_before(const assign_args& a, int steps, wg_sums& sums) {
    int mine = 0, total;             // pages are 31 bits, so is their sum
    for (int i = threadIdx.x; i < steps; i += NT) mine += a.free_pages[i];
    prefix(mine, sums, 1, total);
    return total;
}
__global__ __launch_bounds__(NT) void lists_give_kernel(assign_args a) {
    __shared__ wg_sums sums;
    __shared__ int list[STEP];
    const int64_t before = free_before(a, blockIdx.x, sums);
    const int requests = a.totals[0];
    if (before >= requests) return;
    const int64_t p0 = static_cast<int64_t>(blockIdx.x) * STEP;
    give_step(a, a.info, load_counts(a, p0 + threadIdx.x * PER), p0, before, requests, sums, list);
}
__global__ __launch_bounds__(NT) void lists_finish_kernel(assign_args a, int steps) {
    __shared__ wg_sums sums;
    finish(a, a.info, free_before(a, steps, sums), a.totals[0]);
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
// written list.
//
// A token's keys are whole 16-byte pieces, which go from page to page as they are.  Its
// values are one byte of every element's 64: the pages they come from are staged in LDS
// with an element's 64 bytes in a row, SLOTS pages at a time, and a lane puts together an
// element's new bytes; where a byte comes from is the same for all elements, so it is worked
// out once a token and read from another lane.  Bound by memory: 2 (D + 1) bytes read and
// written per token and KV head, and whole pages of values where tokens are picked.
// Rows of 72 bytes leave the banks that 64 lanes read at the same place of theirs
// different by pairs.  What is read or written once passes by the caches, so that they keep
// the values' pages for the neighbour that needs them, too.  29,793 tokens of 12 heads of
// 128, moved by part of a page: 40.9 us, 4.5 TB/s (51.4 through the caches; single bytes
// from memory instead of LDS 79); half of 4 x 20,000 tokens of 8 heads: 49.2 us (61.4; 87).
// ---------------------------------------------------------------------------
struct move_args {
    cache_view from, to;
    const int32_t *index, *start, *count;
    int n, chunks;
};

constexpr uint32_t ZERO_POWER = 27;      // 2^-100, as a row of zeros is written
constexpr int SLOTS = 3;                 // pages staged at a time
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
constexpr int ROW = 72;                  // bytes of an element's row in LDS

__device__ __forceinline__ int entry_at(const cache_view& c, int b, int h, int64_t pos) {
    if (pos < 0 || pos >= static_cast<int64_t>(c.max_pages) * CACHE_TOKENS) return -1;
    const int32_t* list = c.table + (static_cast<int64_t>(b) * c.table_heads + (c.table_heads > 1 ? h : 0)) * c.max_pages;
    const int e = list[pos / CACHE_TOKENS];
    return e >= 0 && e < c.pages ? e : -1;
}
template <int D>
__device__ __forceinline__ char* page_at(const cache_view& c, int e, int h) {
    return c.pool + (static_cast<int64_t>(e) * c.heads + h) * cache_page_bytes(D);
}

template <int D>
__global__ __launch_bounds__(256) void cache_move_kernel(move_args a) {
    constexpr int SLOT = D * ROW;                     // a page's values; behind the last slot one of zeros
    __shared__ __attribute__((aligned(16))) char rows[(SLOTS + 1) * SLOT];
    // neighbouring pages, which read a page of values both, on one XCD
    const int64_t item = xcd_item(blockIdx.x, gridDim.x);
    const int chunk = static_cast<int>(item % a.chunks);
    const int64_t bh = item / a.chunks;
    const int b = static_cast<int>(bh / a.to.heads), h = static_cast<int>(bh % a.to.heads);
    const int tid = threadIdx.x, lane = lane_id(), wave = wave_id();
    const int cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const int64_t start = a.start[b];
    // pages from the one that holds position `start` on
    const int64_t first_page = start >= 0 ? start / CACHE_TOKENS : -((-start + CACHE_TOKENS - 1) / CACHE_TOKENS);
    const int64_t pos0 = (first_page + chunk) * CACHE_TOKENS;
    if (pos0 >= start + cnt) return;
    const int target = entry_at(a.to, b, h, pos0);
    if (target < 0) return;
    char* to = page_at<D>(a.to, target, h);
    const int lo = static_cast<int>(max(start - pos0, static_cast<int64_t>(0)));
    const int hi = static_cast<int>(min(start + cnt - pos0, static_cast<int64_t>(64)));
    // lane j, in every wave: where token j comes from (its page, -1 for none, and its place there)
    int entry = -1, place = 0;
    const bool mine = lane >= lo && lane < hi;
    if (mine) {
        const int at = a.index[static_cast<int64_t>(b) * a.n + (pos0 + lane - start)];
        entry = entry_at(a.from, b, h, at);
        place = at & 63;
    }
    const uint64_t live = __ballot(mine), found = __ballot(entry >= 0);
    // runs of tokens of one page
    const int before = __shfl_up(entry, 1, 64);
    const uint64_t starts = __ballot(entry >= 0 && (lane == 0 || entry != before));
    const int runs = __builtin_popcountll(starts);

    // keys: requested here, stored when the values are requested, too
    u32x4_t keys[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const int u = tid + 256 * i, r = u & 15, t = u / D, rest = u & (D - 1) & ~15, j = 16 * t + r;
        const int e = __shfl(entry, j, 64), s = __shfl(place, j, 64);
        keys[i] = u32x4_t{0, 0, 0, 0};
        if (e >= 0)
            keys[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(page_at<D>(a.from, e, h)) + (s >> 4) * D + rest + (s & 15));
    }
    const auto store_keys = [&]() {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const int u = tid + 256 * i, j = 16 * (u / D) + (u & 15);
            if (j >= lo && j < hi) __builtin_nontemporal_store(keys[i], reinterpret_cast<u32x4_t*>(to) + u);
        }
    };
    // powers
    char power = 0, *power_to = nullptr;
    if (tid < 128) {
        const bool values = tid >= 64;
        const int j = values ? 16 * (lane >> 2 & 3) + 4 * (lane >> 4) + (lane & 3) : 16 * (lane & 3) + (lane >> 2);
        const int e = __shfl(entry, j, 64), s = __shfl(place, j, 64);
        if (j >= lo && j < hi) {
            const int at = values ? 64 + (s >> 2 & 3) * 16 + (s >> 4) * 4 + (s & 3) : (s & 15) * 4 + (s >> 4);
            power = e >= 0 ? page_at<D>(a.from, e, h)[128 * D + at] : static_cast<char>(ZERO_POWER);
            power_to = to + 128 * D + tid;
        }
    }
    u32x4_t* out = reinterpret_cast<u32x4_t*>(to + 64 * D);
    if (runs == 1 && found == ~0ull && __ballot(place != lane) == 0) {     // a page as it is
        const u32x4_t* in = reinterpret_cast<const u32x4_t*>(page_at<D>(a.from, __builtin_amdgcn_readfirstlane(entry), h) + 64 * D);
#pragma unroll
        for (int u = tid; u < 4 * D; u += 256) __builtin_nontemporal_store(__builtin_nontemporal_load(in + u), out + u);
        store_keys();
        if (power_to) *power_to = power;
        return;
    }
    // values: this thread's element and the groups g of its pieces
    constexpr int GROUPS = D / 64;                    // of 16 tokens
    const int el = tid & (D - 1), g0 = wave / (D / 64) * GROUPS;
    for (int x = tid; x < SLOT / 8; x += 256) reinterpret_cast<uint64_t*>(rows + SLOTS * SLOT)[x] = 0;
    const int run = __builtin_popcountll(starts & (~0ull >> (63 - lane))) - 1;
    const int within = (place >> 2 & 3) * 16 + (place >> 4) * 4 + (place & 3);
    uint32_t w[GROUPS][4] = {};
    for (int r0 = 0; r0 == 0 || r0 < runs; r0 += SLOTS) {
        if (r0) __syncthreads();
        uint64_t left = starts;
        for (int r = 0; r < r0; ++r) left &= left - 1;
        uint4 x[SLOTS][D / 64];
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if (r0 + k >= runs) continue;
            const int e = __builtin_amdgcn_readlane(entry, __builtin_ctzll(left));
            left &= left - 1;
            const uint4* in = reinterpret_cast<const uint4*>(page_at<D>(a.from, e, h) + 64 * D);
#pragma unroll
            for (int i = 0; i < D / 64; ++i) x[k][i] = in[tid + 256 * i];
        }
        if (r0 == 0) {
            store_keys();
            if (power_to) *power_to = power;
        }
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if (r0 + k >= runs) continue;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const int u = tid + 256 * i;
                uint2* at = reinterpret_cast<uint2*>(rows + k * SLOT + ((u >> 6) * 16 + (u & 15)) * ROW + (u >> 4 & 3) * 16);
                at[0] = make_uint2(x[k][i].x, x[k][i].y);
                at[1] = make_uint2(x[k][i].z, x[k][i].w);
            }
        }
        __syncthreads();
        const bool here = entry >= 0 && run >= r0 && run < r0 + SLOTS;
        const int offset = (here ? run - r0 : SLOTS) * SLOT + (here ? within : 0);
#pragma unroll
        for (int k = 0; k < GROUPS; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = __builtin_amdgcn_readlane(offset, 16 * t + 4 * (g0 + k) + i);
                    w[k][t] |= static_cast<uint32_t>(static_cast<uint8_t>(rows[at + el * ROW])) << (8 * i);
                }
    }
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
        const int u = (el >> 4) * 64 + (g0 + k) * 16 + (el & 15);
        if (live == ~0ull) {
            __builtin_nontemporal_store(u32x4_t{w[k][0], w[k][1], w[k][2], w[k][3]}, out + u);
            continue;
        }
        char* bytes = reinterpret_cast<char*>(out + u);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t four = static_cast<uint32_t>(live >> (16 * t + 4 * (g0 + k))) & 15u;
            if (four == 15u) {
                reinterpret_cast<uint32_t*>(bytes)[t] = w[k][t];
                continue;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((four >> i) & 1u) bytes[4 * t + i] = static_cast<char>(w[k][t] >> (8 * i));
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
    if (c.batch <= NT && entries <= (source || drop ? LONE_ENTRIES : LONE_TRIMS) && steps <= LONE_STEPS) {
        hipLaunchKernelGGL(lists_alone_kernel, dim3(1), dim3(NT), 0, s, a);
    } else {
        const dim3 wide(static_cast<unsigned>(std::min<int64_t>((entries + 255) / 256, 4096)));
        if (source && !drop && c.batch * 4 <= COLUMN_ENTRIES) {
            const int columns = static_cast<int>(std::max<int64_t>(
                1, std::min<int64_t>(COLUMN_ENTRIES / c.batch, (c.max_pages + 127) / 128)));
            hipLaunchKernelGGL(lists_columns_kernel, dim3(static_cast<unsigned>((c.max_pages + columns - 1) / columns)), dim3(256),
                               0, s, a, columns);
        } else if (source || drop) {
            hipLaunchKernelGGL(lists_save_kernel, wide, dim3(256), 0, s, a);
            hipLaunchKernelGGL(lists_write_kernel, wide, dim3(256), 0, s, a);
        } else {
            hipLaunchKernelGGL(lists_trim_kernel, wide, dim3(256), 0, s, a);
        }
        if (steps <= LONE_STEPS) {
            if (c.batch <= NT) hipLaunchKernelGGL((lists_plan_kernel<true, true>), dim3(1), dim3(NT), 0, s, a);
            else hipLaunchKernelGGL((lists_plan_kernel<true, false>), dim3(1), dim3(NT), 0, s, a);
        } else {
            hipLaunchKernelGGL((lists_plan_kernel<false, false>), dim3(1), dim3(NT), 0, s, a);
            hipLaunchKernelGGL(lists_count_kernel, dim3(static_cast<unsigned>(steps)), dim3(NT), 0, s, a);
            hipLaunchKernelGGL(lists_give_kernel, dim3(static_cast<unsigned>(steps)), dim3(NT), 0, s, a);
            hipLaunchKernelGGL(lists_finish_kernel, dim3(1), dim3(NT), 0, s, a, static_cast<int>(steps));
        }
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
