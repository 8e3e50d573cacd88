// Bookkeeping of a page pool on the device: room for new positions (with copy on write), forks, releases, compaction.
//
// State: table [rows][cols] of page numbers, refs [pages] = how many table entries hold a page; a page with 0 is free.  Nothing is
// handed over by the host, so a decode step with forked requests runs from one captured graph.
//
// Free pages are given out lowest first, in the order of the listed rows, so results do not depend on how the GPU schedules.  Finding
// the d-th free page: a first launch writes one bit per page, the free pages before each word within its chunk of 1024, and the count
// of each chunk; a second one adds up the chunk counts in shared memory (every CTA for itself: a few hundred values) and finds any d
// by a binary search there, one 64-byte read and one word.  The first launch also takes down what the listed rows need, since the
// second one changes the tables and counts while other CTAs are still at work.  Two launches, no CTA waits for another.
//
// Bound by launch latency and a handful of dependent reads for the tables, by memory where pages are copied.  Measured: release 2.4 us,
// fork of 24 rows 3.8, reserve for them with 20 copies 8.3 (two launches), 3500 pages for 7 prompts 6.9, a compaction that moves 388
// MB 131 us = 5.9 TB/s, 0.92 of the copy bandwidth.
#include "flux_internal.h"

namespace flux {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 1024;             // pages a scan CTA looks at
constexpr int kChunkWords = kChunk / 32;
constexpr int kForkThreads = 512;

__host__ __device__ constexpr size_t up16(size_t x) { return (x + 15) / 16 * 16; }

// Scratch: free bits | free pages before a word within its chunk | chunk counts | per listed row: demand, page to copy, its count |
// per (listed row, 32 columns): entries to be filled, and those before them in the row.
struct Scratch {
    uint32_t *bits;
    uint16_t *before;
    int32_t *chunk_free;
    int32_t *demand, *src, *src_refs;
    uint32_t *need;
    int32_t *need_before;
    size_t total;
    __host__ __device__ Scratch(void *base, int n_pages, int n_rows, int cols)
    {
        const size_t chunks = ((size_t)n_pages + kChunk - 1) / kChunk, words = ((size_t)cols + 31) / 32;
        if (n_rows > kMaxPageRows) n_rows = kMaxPageRows;        // as many as a call lists: a place in the list, not a row of the table
        unsigned char *p = (unsigned char *)base;
        size_t at = 0;
        bits = (uint32_t *)(p + at);        at = up16(at + chunks * kChunkWords * 4);
        before = (uint16_t *)(p + at);      at = up16(at + chunks * kChunkWords * 2);
        chunk_free = (int32_t *)(p + at);   at = up16(at + chunks * 4);
        demand = (int32_t *)(p + at);       at = up16(at + (size_t)n_rows * 4);
        src = (int32_t *)(p + at);          at = up16(at + (size_t)n_rows * 4);
        src_refs = (int32_t *)(p + at);     at = up16(at + (size_t)n_rows * 4);
        need = (uint32_t *)(p + at);        at = up16(at + words * n_rows * 4);
        need_before = (int32_t *)(p + at);  at = up16(at + words * n_rows * 4);
        total = at;
    }
};

struct PoolArgs {
    int32_t *table, *refs;
    void *const *slabs;
    void *scratch;
    int n_rows, cols, n_pages, shift, n_slabs;
    int64_t page_bytes;
    uint32_t *status;
};

struct ListArgs {
    int n;
    const int32_t *rows, *a, *b;         // rows NULL: 0 .. n - 1
    int32_t *granted;
    __device__ __forceinline__ int row(int i) const { return rows != nullptr ? rows[i] : i; }
};

__device__ __forceinline__ void begin_launch()
{
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
}

// ---- first launch: free pages, and what the listed rows need --------------------------------------------------------

__device__ __forceinline__ void scan_chunk(const PoolArgs &a, const Scratch &s, int chunk)
{
    __shared__ uint32_t words[kChunkWords];
    const int lane = threadIdx.x & 31, p0 = chunk * kChunk + 4 * (int)threadIdx.x;
    uint32_t nibble = 0;
    if (p0 + 4 <= a.n_pages) {
        const int4 r = *reinterpret_cast<const int4 *>(a.refs + p0);
        nibble = (r.x == 0 ? 1u : 0u) | (r.y == 0 ? 2u : 0u) | (r.z == 0 ? 4u : 0u) | (r.w == 0 ? 8u : 0u);
    } else {
        for (int k = 0; k < 4; ++k)
            if (p0 + k < a.n_pages && a.refs[p0 + k] == 0) nibble |= 1u << k;
    }
    uint32_t w = nibble << (4 * (lane & 7));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    w |= __shfl_xor_sync(0xffffffffu, w, 4);
    if ((lane & 7) == 0) words[threadIdx.x >> 3] = w;
    __syncthreads();
    if (threadIdx.x < kChunkWords) {
        const uint32_t mine = words[lane];
        int sum = __popc(mine);
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
        }
        s.bits[(size_t)chunk * kChunkWords + lane] = mine;
        s.before[(size_t)chunk * kChunkWords + lane] = (uint16_t)(sum - __popc(mine));
        if (lane == 31) s.chunk_free[chunk] = sum;
    }
}

// Listed row i, one CTA: the entries of positions a[i] .. b[i] - 1 that have to be filled, a thread per entry, the next 256 already
// asked for.  (A row is one CTA's chain: 8K new positions in pages of 16 take 5.1 us with the second launch, 128K 18, 1M 119.)
__device__ __forceinline__ void scan_row(const PoolArgs &a, const ListArgs &l, const Scratch &s, int i)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ int counts[2][kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = l.row(i), n0 = l.a[i], n1 = l.b[i];
    uint32_t flags = 0;
    if (r < 0 || r >= a.n_rows) flags |= FLUX_STATUS_BAD_PAGE;
    if (n0 < 0 || n1 < n0 || n1 > (int64_t)a.cols << a.shift) flags |= FLUX_STATUS_BAD_LENGTH;
    bool bad = false;
    for (int k = threadIdx.x; k < i && l.rows != nullptr; k += kThreads) bad = bad || l.rows[k] == r;
    int demand = 0;
    if (flags == 0 && n1 > n0) {
        const int j0 = n0 >> a.shift, j1 = (int)(((int64_t)n1 + (1 << a.shift) - 1) >> a.shift), words = (a.cols + 31) / 32;
        const bool begun = (n0 & ((1 << a.shift) - 1)) != 0;
        const int32_t *entries = a.table + (size_t)r * a.cols;
        auto ask = [&](int j) { return j >= j0 && j < j1 ? entries[j] : 0; };
        int j = j0 / 32 * 32 + (int)threadIdx.x, e = ask(j), turn = 0;
        for (int base = j0 / 32 * 32; base < j1; base += kThreads, j += kThreads, turn ^= 1) {
            const int ahead = ask(j + kThreads);
            const bool in = j >= j0 && j < j1;
            int refs = 0;
            if (in && e != FLUX_PAGE_NONE) {
                if (e < 0 || e >= a.n_pages) bad = true;
                else if ((refs = a.refs[e]) < 1) bad = true;
            }
            const uint32_t need = __ballot_sync(0xffffffffu, in && (e == FLUX_PAGE_NONE || refs > 1));
            if (lane == 0) counts[turn][warp] = __popc(need);
            __syncthreads();             // (two sets of counts: one barrier a turn)
            int before = demand;
            for (int w = 0; w < kWarps; ++w) {
                if (w < warp) before += counts[turn][w];
                demand += counts[turn][w];
            }
            if (lane == 0 && j < j1) {
                s.need[(size_t)i * words + j / 32] = need;
                s.need_before[(size_t)i * words + j / 32] = before;
            }
            if (j == j0) {               // a begun page that others hold too is copied
                s.src[i] = begun && refs > 1 ? e : FLUX_PAGE_NONE;
                s.src_refs[i] = refs;
            }
            e = ahead;
        }
    } else if (threadIdx.x == 0) {
        s.src[i] = FLUX_PAGE_NONE;
    }
    if (__syncthreads_or(bad)) flags |= FLUX_STATUS_BAD_PAGE;
    if (threadIdx.x == 0) {
        if (flags != 0) atomicOr(a.status, flags);
        s.demand[i] = flags != 0 ? -1 : demand;
    }
}

__global__ void __launch_bounds__(kThreads) scan_kernel(PoolArgs a, ListArgs l)
{
    begin_launch();
    const Scratch s(a.scratch, a.n_pages, a.n_rows, a.cols);
    const int chunks = (a.n_pages + kChunk - 1) / kChunk;
    if ((int)blockIdx.x < chunks) {
        scan_chunk(a, s, (int)blockIdx.x);
    } else {
        scan_row(a, l, s, (int)blockIdx.x - chunks);
    }
}

// ---- second launch ---------------------------------------------------------------------------------------------------

constexpr int kFull = 1 << 25;           // sums stop here: more than any pool has, whatever the listed rows ask for together
static_assert(kMaxPages < kFull - 1, "a row's demand may go down by one");

// Exclusive sums of v[0 .. n) (each at most kFull) in place, the total in v[n]; every thread of the CTA takes part.
__device__ __forceinline__ void sum_up(int *v, int n)
{
    __shared__ int warp_sum[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, each = (n + kThreads - 1) / kThreads, first = min(tid * each, n), last = min(first + each, n);
    auto add = [](int x, int y) { return min(x + y, kFull); };
    int run = 0;
    for (int k = first; k < last; ++k) run = add(run, v[k]);
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, run, d);
        if (lane >= d) run = add(run, y);
    }
    if (lane == 31) warp_sum[tid >> 5] = run;
    __syncthreads();
    int at = __shfl_up_sync(0xffffffffu, run, 1), total = 0;
    if (lane == 0) at = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < (tid >> 5)) at = add(at, warp_sum[w]);
        total = add(total, warp_sum[w]);
    }
    for (int k = first; k < last; ++k) {
        const int x = v[k];
        v[k] = at;
        at = add(at, x);
    }
    if (tid == 0) v[n] = total;
    __syncthreads();
}

// The free pages, with the chunks' sums in shared memory.
struct Free {
    const Scratch &s;
    const int *chunk_before;             // [chunks + 1]
    int chunks;
    // the d-th free page, or the d-th in use (there are more than d, below the pool's end)
    template <bool kUsed = false>
    __device__ __forceinline__ int page(int d) const
    {
        auto count = [](int all, int free) { return kUsed ? all - free : free; };
        int lo = 0, hi = chunks;         // the last chunk with at most d of them before it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (count(mid * kChunk, chunk_before[mid]) <= d) lo = mid; else hi = mid;
        }
        d -= count(lo * kChunk, chunk_before[lo]);
        const uint4 *b = reinterpret_cast<const uint4 *>(s.before + (size_t)lo * kChunkWords);
        int w = -1, there = 0;           // the last word with at most d of them before it
#pragma unroll
        for (int k = 0; k < kChunkWords / 8; ++k) {
            const uint4 x = b[k];
            const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int z = 0; z < 8; ++z) {
                const int c = count((8 * k + z) * 32, (int)(z & 1 ? y[z / 2] >> 16 : y[z / 2] & 0xffffu));
                if (c <= d) {
                    ++w;
                    there = c;
                }
            }
        }
        d -= there;
        uint32_t left = s.bits[(size_t)lo * kChunkWords + w];
        if (kUsed) left = ~left;
        int bit = 0;
#pragma unroll
        for (int half = 16; half > 0; half >>= 1) {
            const int c = __popc(left & ((1u << half) - 1u));
            if (d >= c) {
                d -= c;
                left >>= half;
                bit += half;
            }
        }
        return lo * kChunk + w * 32 + bit;
    }
    __device__ __forceinline__ bool is_free(int p) const { return (s.bits[p >> 5] >> (p & 31)) & 1u; }
    // free pages below p <= number of pages
    __device__ __forceinline__ int before(int p) const
    {
        const int chunk = p / kChunk;
        if (chunk >= chunks) return chunk_before[chunks];
        return chunk_before[chunk] + s.before[p >> 5] + __popc(s.bits[p >> 5] & ((1u << (p & 31)) - 1u));
    }
};

// `bytes` (a multiple of 16) of a page into another one of the same slab, all threads of the CTA.
__device__ __forceinline__ void copy_page(void *slab, int src, int dst, int64_t page_bytes, int64_t bytes)
{
    const uint4 *from = reinterpret_cast<const uint4 *>((const unsigned char *)slab + src * page_bytes);
    uint4 *to = reinterpret_cast<uint4 *>((unsigned char *)slab + dst * page_bytes);
    const int pieces = (int)(bytes / 16);
    constexpr int kAhead = 8;
    for (int i = threadIdx.x; i < pieces; i += kAhead * kThreads) {
        uint4 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * kThreads < pieces) x[k] = from[i + k * kThreads];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * kThreads < pieces) to[i + k * kThreads] = x[k];
    }
}

// Rows are served in the order of the list until the pages run out.  Of the rows that want to write one shared page the last keeps it if
// all who hold it are listed; the others get copies.  Which ones is settled here, where it is known which rows passed their checks.
__global__ void __launch_bounds__(kThreads) reserve_kernel(PoolArgs a, ListArgs l)
{
    extern __shared__ __align__(16) int sh[];
    begin_launch();
    const Scratch s(a.scratch, a.n_pages, a.n_rows, a.cols);
    const int tid = threadIdx.x, lane = tid & 31, chunks = (a.n_pages + kChunk - 1) / kChunk, words = (a.cols + 31) / 32;
    // start: first free page of a row; src: page to copy, or NONE, or kKept; kFailed: a row whose checks failed
    constexpr int kKept = FLUX_PAGE_NONE - 1, kFailed = FLUX_PAGE_NONE - 2;
    int *start = sh, *src = start + l.n + 1, *chunk_before = src + l.n;
    bool shares = false;
    for (int k = tid; k < chunks; k += kThreads) chunk_before[k] = s.chunk_free[k];
    for (int i = tid; i < l.n; i += kThreads) {
        const int d = s.demand[i], page = s.src[i];
        start[i] = min(max(d, 0), kFull);
        src[i] = d < 0 ? kFailed : page;
        shares = shares || (d >= 0 && page >= 0);
    }
    // Who keeps a shared page: every listed row with every other, in every CTA.  Nothing beside a launch for a beam search's rows (24 rows 8 us in
    // all, 256 16), but it is quadratic: 1024 rows 133 us, 4096 1.9 ms.
    if (__syncthreads_or(shares)) {
        uint32_t keeps = 0;              // of the rows tid, tid + 256, ...
        static_assert(kMaxPageRows <= 32 * kThreads, "a bit for each row of a thread");
        for (int i = tid, z = 0; i < l.n; i += kThreads, ++z) {
            if (src[i] < 0) continue;
            int writers = 0, last = 0;
            for (int k = 0; k < l.n; ++k)
                if (src[k] == src[i]) {
                    ++writers;
                    last = k;
                }
            if (last == i && writers == s.src_refs[i]) keeps |= 1u << z;
        }
        __syncthreads();
        for (int i = tid, z = 0; i < l.n; i += kThreads, ++z)
            if ((keeps >> z) & 1u) {     // the row's first entry is not filled after all
                src[i] = kKept;
                --start[i];
            }
        __syncthreads();
    }
    sum_up(start, l.n);
    sum_up(chunk_before, chunks);
    const Free free_pages{s, chunk_before, chunks};
    const int total = chunk_before[chunks];
    auto granted = [&](int i) { return src[i] != kFailed && start[i + 1] <= total; };

    if (blockIdx.x == 0) {
        bool out = false;
        for (int i = tid; i < l.n; i += kThreads) {
            out = out || (src[i] != kFailed && start[i + 1] > total);
            if (l.granted != nullptr) l.granted[i] = granted(i) ? 1 : 0;
        }
        if (out) atomicOr(a.status, FLUX_STATUS_NO_PAGES);
    }

    // the entries: a group of warps per row, 32 columns each
    const int warps = (int)gridDim.x * (kThreads / 32), warp = (int)blockIdx.x * (kThreads / 32) + (tid >> 5);
    const int group = max(warps / l.n, 1);
    for (int i = warp / group; i < l.n; i += warps / group) {
        if (warp / group >= warps / group || !granted(i) || start[i + 1] == start[i]) continue;
        const int n0 = l.a[i], n1 = l.b[i], j0 = n0 >> a.shift, j1 = (int)(((int64_t)n1 + (1 << a.shift) - 1) >> a.shift);
        const bool keeps = src[i] == kKept;
        int32_t *entries = a.table + (size_t)l.row(i) * a.cols;
        for (int w = j0 / 32 + warp % group; w <= (j1 - 1) / 32; w += group) {
            uint32_t need = s.need[(size_t)i * words + w];
            int d = start[i] + s.need_before[(size_t)i * words + w];
            if (keeps) {
                if (w == j0 / 32) need &= ~(1u << (j0 & 31));
                else --d;
            }
            if (!((need >> lane) & 1u)) continue;
            const int page = free_pages.page(d + __popc(need & ((1u << lane) - 1u)));
            const int old = entries[32 * w + lane];
            if (old != FLUX_PAGE_NONE) atomicSub(a.refs + old, 1);
            entries[32 * w + lane] = page;
            a.refs[page] = 1;
        }
    }

    // the begun pages: only the rows that hold positions
    const int64_t row_bytes = a.page_bytes >> a.shift;
    for (int64_t item = blockIdx.x; item < (int64_t)l.n * a.n_slabs; item += gridDim.x) {
        const int i = (int)(item / a.n_slabs);
        if (src[i] < 0 || !granted(i)) continue;
        copy_page(a.slabs[item - (int64_t)i * a.n_slabs], src[i], free_pages.page(start[i]), a.page_bytes, (l.a[i] & ((1 << a.shift) - 1)) * row_bytes);
    }
}

// Pages in use beyond their number move to the free pages below it, in order: the m-th of the former to the m-th of the latter.
__global__ void __launch_bounds__(kThreads) compact_kernel(PoolArgs a, int32_t *map_out, int32_t *used_out)
{
    extern __shared__ __align__(16) int sh[];
    begin_launch();
    const Scratch s(a.scratch, a.n_pages, a.n_rows, a.cols);
    const int tid = threadIdx.x, chunks = (a.n_pages + kChunk - 1) / kChunk;
    for (int k = tid; k < chunks; k += kThreads) sh[k] = s.chunk_free[k];
    __syncthreads();
    sum_up(sh, chunks);
    const Free free_pages{s, sh, chunks};
    const int used = a.n_pages - sh[chunks], holes = free_pages.before(used);
    auto target = [&](int p) {           // of a page in use
        return p < used ? p : free_pages.page(p - free_pages.before(p) - (used - holes));
    };
    // the contents: (page, slab) items in strides, 256 of a CTA's places at a time
    __shared__ int2 move[kThreads];
    const int64_t items = (int64_t)holes * a.n_slabs;
    for (int64_t first = blockIdx.x; first < items; first += (int64_t)gridDim.x * kThreads) {
        const int64_t mine = first + (int64_t)tid * gridDim.x;
        if (mine < items) {
            const int m = (int)(mine / a.n_slabs);
            move[tid] = make_int2(free_pages.page<true>(used - holes + m), free_pages.page(m));
        }
        __syncthreads();
        for (int k = 0; k < kThreads; ++k) {
            const int64_t item = first + (int64_t)k * gridDim.x;
            if (item >= items) break;
            copy_page(a.slabs[item % a.n_slabs], move[k].x, move[k].y, a.page_bytes, a.page_bytes);
        }
        __syncthreads();
    }
    const int64_t threads = (int64_t)gridDim.x * kThreads, me = (int64_t)blockIdx.x * kThreads + tid;
    if (me == 0 && used_out != nullptr) *used_out = used;
    for (int64_t p = me; p < a.n_pages; p += threads) {
        const bool live = !free_pages.is_free((int)p);
        const int to = live ? target((int)p) : FLUX_PAGE_NONE;
        if (map_out != nullptr) map_out[p] = to;
        if (live && to != p) {           // `to` was free: nobody else looks at its count
            a.refs[to] = a.refs[p];
            a.refs[p] = 0;
        }
    }
    bool bad = false;
    for (int64_t i = me; i < (int64_t)a.n_rows * a.cols; i += threads) {
        const int e = a.table[i];
        if (e == FLUX_PAGE_NONE) continue;
        int to = FLUX_PAGE_NONE;
        if (e < 0 || e >= a.n_pages || free_pages.is_free(e)) bad = true;      // an entry that is not counted: its page may be given away
        else to = target(e);
        if (to != e) a.table[i] = to;
    }
    if (bad) atomicOr(a.status, FLUX_STATUS_BAD_PAGE);
}

// ---- one launch ------------------------------------------------------------------------------------------------------

// One entry less holds page e; false: it is none of the pool's, or was not counted and stays free.
__device__ __forceinline__ bool give_up(const PoolArgs &a, int e)
{
    if (e < 0 || e >= a.n_pages) return false;
    if (atomicSub(a.refs + e, 1) >= 1) return true;
    atomicAdd(a.refs + e, 1);
    return false;
}

// Rows dst[i] take the first entries of rows src[i], all at once: a CTA owns some columns of all listed rows, so it reads every
// source before it writes.  rows: src, a: dst, b: len.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(PoolArgs a, ListArgs l, int width)
{
    extern __shared__ __align__(16) int sh[];
    int *dst = sh, *src = dst + l.n, *cols = src + l.n, *taken = cols + l.n;     // cols: entries to take, -1: a check failed; taken: [n][width]
    const int tid = threadIdx.x, c0 = (int)blockIdx.x * width;
    begin_launch();
    uint32_t flags = 0;
    for (int i = tid; i < l.n; i += kForkThreads) {
        const int from = l.row(i), to = l.a[i], len = l.b[i];
        dst[i] = to;
        src[i] = from;
        cols[i] = (int)(((int64_t)max(len, 0) + (1 << a.shift) - 1) >> a.shift);
        uint32_t f = 0;
        if (from < 0 || from >= a.n_rows || to < 0 || to >= a.n_rows) f |= FLUX_STATUS_BAD_PAGE;
        if (len < 0 || len > (int64_t)a.cols << a.shift) f |= FLUX_STATUS_BAD_LENGTH;
        if (f != 0) cols[i] = -1;
        flags |= f;
    }
    __syncthreads();
    for (int i = tid >> 5; i < l.n; i += kForkThreads / 32)
        for (int k = tid & 31; k < i; k += 32)
            if (dst[k] == dst[i]) {      // listed twice
                cols[i] = -1;
                flags |= FLUX_STATUS_BAD_PAGE;
            }
    __syncthreads();
    // sources and what they replace, before anything is written
    constexpr int kHeld = 4;             // entries that a thread keeps of the latter; beyond them they are read again
    int olds[kHeld];
#pragma unroll 4
    for (int x = tid, z = 0; x < l.n * width; x += kForkThreads, ++z) {
        const int i = x / width, c = c0 + x - i * width;
        int e = FLUX_PAGE_NONE, old = FLUX_PAGE_NONE;
        if (cols[i] >= 0 && c < a.cols) {
            old = a.table[(size_t)dst[i] * a.cols + c];
            if (c < cols[i]) e = a.table[(size_t)src[i] * a.cols + c];
            if (e != FLUX_PAGE_NONE && (e < 0 || e >= a.n_pages)) {
                e = FLUX_PAGE_NONE;
                flags |= FLUX_STATUS_BAD_PAGE;
            }
        }
        taken[x] = e;
#pragma unroll
        for (int y = 0; y < kHeld; ++y)
            if (y == z) olds[y] = old;
    }
    // A page that is not counted may be given away, so nobody takes it over.  (Other CTAs may be changing counts by now, but the source's
    // entry is in a column of this one, which changes none before the barrier: a page that was counted still is.)
#pragma unroll 4
    for (int x = tid; x < l.n * width; x += kForkThreads) {
        const int e = taken[x];
        if ((e != FLUX_PAGE_NONE ? a.refs[e] : 1) < 1) {
            taken[x] = FLUX_PAGE_NONE;
            flags |= FLUX_STATUS_BAD_PAGE;
        }
    }
    __syncthreads();
    for (int x = tid, z = 0; x < l.n * width; x += kForkThreads, ++z) {
        const int i = x / width, c = c0 + x - i * width;
        if (cols[i] < 0 || c >= a.cols) continue;
        int32_t *entry = a.table + (size_t)dst[i] * a.cols + c;
        int old = 0;
        if (z < kHeld) {
#pragma unroll
            for (int y = 0; y < kHeld; ++y)
                if (y == z) old = olds[y];
        } else {
            old = *entry;
        }
        const int e = taken[x];
        if (old == e) continue;
        if (e != FLUX_PAGE_NONE) atomicAdd(a.refs + e, 1);
        if (old != FLUX_PAGE_NONE && !give_up(a, old)) flags |= FLUX_STATUS_BAD_PAGE;
        *entry = e;
    }
    if (flags != 0) atomicOr(a.status, flags);
}

// Entries whose positions all lie in [a, b) are given up.  Taking an entry out is an exchange, so a row listed twice is released once.
__global__ void __launch_bounds__(kThreads) release_kernel(PoolArgs a, ListArgs l)
{
    begin_launch();
    uint32_t flags = 0;
    const int blocks = (a.cols + kThreads - 1) / kThreads;
    for (int64_t task = blockIdx.x; task < (int64_t)l.n * blocks; task += gridDim.x) {
        const int i = (int)(task / blocks), j = (int)(task - (int64_t)i * blocks) * kThreads + (int)threadIdx.x;
        const int r = l.row(i), begin = l.a[i], end = l.b[i];
        if (r < 0 || r >= a.n_rows) {
            flags |= FLUX_STATUS_BAD_PAGE;
            continue;
        }
        if (begin < 0) {
            flags |= FLUX_STATUS_BAD_LENGTH;
            continue;
        }
        if (j >= a.cols || (int64_t)j << a.shift < begin || ((int64_t)j + 1) << a.shift > end) continue;
        int32_t *entry = a.table + (size_t)r * a.cols + j;
        if (*entry == FLUX_PAGE_NONE) continue;
        const int e = atomicExch(entry, FLUX_PAGE_NONE);
        if (e != FLUX_PAGE_NONE && !give_up(a, e)) flags |= FLUX_STATUS_BAD_PAGE;
    }
    if (flags != 0) atomicOr(a.status, flags);
}

// ---- host ------------------------------------------------------------------------------------------------------------

PoolArgs pool_args(flux_plan *p, const flux_page_pool &pool)
{
    PoolArgs a;
    a.table = pool.table; a.refs = pool.refs; a.slabs = pool.slabs; a.scratch = pool.scratch;
    a.n_rows = pool.n_rows; a.cols = pool.max_pages; a.n_pages = pool.n_pages; a.n_slabs = pool.n_slabs;
    a.shift = 0;
    while ((1 << a.shift) < pool.page_size) ++a.shift;
    a.page_bytes = (int64_t)pool.page_size * p->cfg.n_kv_heads * kRowBytes;
    a.status = (uint32_t *)((char *)p->ws + p->lay.status);
    return a;
}

template <class... Args>
int launch(flux_plan *p, void (*fn)(Args...), int64_t ctas, int threads, size_t smem, cudaStream_t st, const char *what, Args... args)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)ctas);
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    p->launches++;
    p->page_calls.add(st);           // a paged decode right behind it must not read the table ahead of its wait
    return check_cuda(cudaLaunchKernelEx(&lc, fn, args...), what);
}

int64_t chunks_of(const flux_page_pool &pool) { return ((int64_t)pool.n_pages + kChunk - 1) / kChunk; }

int launch_scan(flux_plan *p, const PoolArgs &a, const ListArgs &l, int64_t chunks, cudaStream_t st)
{
    return launch(p, scan_kernel, chunks + l.n, kThreads, 0, st, "page scan kernel launch", a, l);
}

}  // namespace

size_t pages_scratch_size(const flux_page_pool &pool) { return Scratch(nullptr, pool.n_pages, pool.n_rows, pool.max_pages).total; }

int pages_setup(flux_plan *p)
{
    const size_t most = (size_t)(2 * kMaxPageRows + 2 + kMaxPages / kChunk) * sizeof(int), fork = (size_t)(3 + 32) * 1024 * sizeof(int);
    const size_t fork_most = (size_t)(3 + 8) * kMaxPageRows * sizeof(int);
    if ((size_t)p->dev.smem_optin < most || (size_t)p->dev.smem_optin < fork_most || (size_t)p->dev.smem_optin < fork)
        return fail(FLUX_E_CUDA, "device offers %d bytes of shared memory per block, the page kernels need %zu", p->dev.smem_optin, most > fork ? most : fork);
    int rc = check_cuda(cudaFuncSetAttribute(reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most), "cudaFuncSetAttribute(reserve_kernel)");
    if (!rc) rc = check_cuda(cudaFuncSetAttribute(compact_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most), "cudaFuncSetAttribute(compact_kernel)");
    if (!rc) rc = check_cuda(cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(fork > fork_most ? fork : fork_most)), "cudaFuncSetAttribute(fork_kernel)");
    return rc;
}

int launch_pages_reserve(flux_plan *p, const flux_page_pool &pool, int n, const int32_t *rows, const int32_t *len, const int32_t *new_len, int32_t *granted,
                         cudaStream_t st)
{
    const PoolArgs a = pool_args(p, pool);
    const ListArgs l = {n, rows, len, new_len, granted};
    const int64_t chunks = chunks_of(pool);
    int rc = launch_scan(p, a, l, chunks, st);
    if (rc) return rc;
    const size_t smem = (size_t)(2 * n + 2 + chunks) * sizeof(int);
    int64_t ctas = (int64_t)n * (pool.n_slabs > 8 ? pool.n_slabs : 8);
    const int64_t most = 4 * (int64_t)p->dev.n_sms;
    if (ctas > most) ctas = most;
    return launch(p, reserve_kernel, ctas, kThreads, smem, st, "page reserve kernel launch", a, l);
}

int launch_pages_fork(flux_plan *p, const flux_page_pool &pool, int n, const int32_t *src, const int32_t *dst, const int32_t *len, cudaStream_t st)
{
    const PoolArgs a = pool_args(p, pool);
    const ListArgs l = {n, src, dst, len, nullptr};
    const int width = n <= 1024 ? 32 : 8;        // up to 140 KB and 176 KB
    return launch(p, fork_kernel, (pool.max_pages + width - 1) / width, kForkThreads, (size_t)n * (3 + width) * sizeof(int), st, "page fork kernel launch", a, l, width);
}

int launch_pages_release(flux_plan *p, const flux_page_pool &pool, int n, const int32_t *rows, const int32_t *begin, const int32_t *end, cudaStream_t st)
{
    const PoolArgs a = pool_args(p, pool);
    const ListArgs l = {n, rows, begin, end, nullptr};
    int64_t ctas = (int64_t)n * ((pool.max_pages + kThreads - 1) / kThreads);
    const int64_t most = 8 * (int64_t)p->dev.n_sms;
    if (ctas > most) ctas = most;
    return launch(p, release_kernel, ctas, kThreads, 0, st, "page release kernel launch", a, l);
}

int launch_pages_compact(flux_plan *p, const flux_page_pool &pool, int32_t *map_out, int32_t *used_out, cudaStream_t st)
{
    const PoolArgs a = pool_args(p, pool);
    const int64_t chunks = chunks_of(pool);
    int rc = launch_scan(p, a, ListArgs{0, nullptr, nullptr, nullptr, nullptr}, chunks, st);
    if (rc) return rc;
    const int64_t entries = (int64_t)pool.n_rows * pool.max_pages, work = entries > pool.n_pages ? entries : pool.n_pages;
    int64_t ctas = (work + kThreads - 1) / kThreads;
    if (ctas < (int64_t)pool.n_pages * pool.n_slabs) ctas = (int64_t)pool.n_pages * pool.n_slabs;
    const int64_t most = 8 * (int64_t)p->dev.n_sms;        // two waves: a CTA's list of moves is short enough for the ends to even out (one: 6 % slower)
    if (ctas > most) ctas = most;
    return launch(p, compact_kernel, ctas, kThreads, (size_t)(chunks + 1) * sizeof(int), st, "page compact kernel launch", a, map_out, used_out);
}

}  // namespace flux
