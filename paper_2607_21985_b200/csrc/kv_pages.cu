// The pages of a key/value cache between steps: taken for growing requests, freed, forked, copied, brought together.  The state is the
// caller's, on the device: a table of each request's pages and a count of the table's entries that name each page; a page that none names is
// free.  What a call does follows from these alone, page by page in their order, so the same state gives the same pages; and all of it
// may be captured together with the steps that use the pages.
//
// Counting and naming are integers; what takes time is moving pages (2 bytes of traffic to each byte of a page, in every layer): 3000 pages of
// 12 layers of 16.5 KB in 207 us, 5.7 TB/s; 1000 of 33 KB in 141 us, 5.6 TB/s.  300 of 16.5 KB take 18 to 20 us, which is no rate of the memory's: 74 of their 119 MB
// reach it, the rest stays in the second-level cache.  Calls on few pages are the latency of a kernel's loads, one after another.
#include <mutex>

#include "kv8.cuh"

namespace spdp {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMostRequests = 4096;
constexpr unsigned kAll = 0xFFFFFFFFu;

// A number for each thread -> the sum of those of the threads before it; the sum of all in *total.  (All threads; `sums`: a word to a
// warp and one more.  Ends with a barrier.)
__device__ __forceinline__ int64_t sum_before(int64_t mine, int64_t* sums, int64_t* total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t up_to = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t v = __shfl_up_sync(kAll, up_to, d);
        if (lane >= d) up_to += v;
    }
    if (lane == 31) sums[w] = up_to;
    __syncthreads();
    if (w == 0) {
        const int64_t all = sums[lane];
        int64_t s = all;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t v = __shfl_up_sync(kAll, s, d);
            if (lane >= d) s += v;
        }
        __syncwarp();
        sums[lane] = s - all;
        if (lane == 31) sums[kWarps] = s;
    }
    __syncthreads();
    const int64_t r = sums[w] + up_to - mine;
    *total = sums[kWarps];
    __syncthreads();
    return r;
}

struct Table {
    int32_t* entries;
    int64_t stride;
    int rows, pages;                    // entries of a row
};
__device__ __forceinline__ int within(int v, int most) { return v < 0 ? 0 : v < most ? v : most; }

// Free pages, lowest first, to the places 0 .. wanted - 1: give(place, page) for each, page -1 where there are no more.  One CTA, which first brings
// the pages of a run together, in `found` (kRun words), so that the places are served side by side (200 places on 6000 pages: 14.8 us where each
// thread served what it had found, 6.9 this way).
constexpr int kAhead = 8;               // pages of a lane that are looked at at once
constexpr int kRun = kThreads * kAhead;
template <typename Give>
__device__ __forceinline__ int64_t give_pages(int32_t* ref, int pages, int64_t wanted, int64_t* sums, int32_t* found, Give give) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t given = 0;
    for (int64_t base = 0; base < pages && given < wanted; base += kRun) {
        const int64_t mine = base + w * (32 * kAhead) + lane;
        unsigned free[kAhead];
        int count = 0;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) free[i] = mine + 32 * i < pages ? ref[mine + 32 * i] <= 0 : 0;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            free[i] = __ballot_sync(kAll, free[i] != 0);
            count += __popc(free[i]);
        }
        int64_t total;
        int at = static_cast<int>(__shfl_sync(kAll, sum_before(lane == 0 ? count : 0, sums, &total), 0));
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (free[i] >> lane & 1) found[at + __popc(free[i] & ((1u << lane) - 1))] = static_cast<int>(mine + 32 * i);
            at += __popc(free[i]);
        }
        __syncthreads();
        const int64_t stop = given + total < wanted ? given + total : wanted;
        for (int64_t place = given + threadIdx.x; place < stop; place += kThreads) {
            const int page = found[place - given];
            ref[page] = 1;
            give(place, page);
        }
        given += total;
        __syncthreads();
    }
    for (int64_t place = given + threadIdx.x; place < wanted; place += kThreads) give(place, -1);
    return wanted > given ? wanted - given : 0;
}

// Which of n ascending starts place u lies behind: the last that is not above it (and not empty).
__device__ __forceinline__ int owner_of(const int64_t* start, int n, int64_t u) {
    int b = 0;
    for (int lo = 0, hi = n - 1; lo <= hi;) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= u) b = mid, lo = mid + 1;
        else hi = mid - 1;
    }
    return b;
}

// start[i]: the sum of count(0) .. count(i - 1); returns the sum of all n.
template <typename Count>
__device__ __forceinline__ int64_t starts_of(int n, int64_t* start, int64_t* sums, Count count) {
    int64_t before = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + threadIdx.x;
        int64_t total;
        const int64_t mine = i < n ? count(i) : 0, at = before + sum_before(mine, sums, &total);
        if (i < n) start[i] = at;
        before += total;
    }
    __syncthreads();
    return before;
}

__global__ void __launch_bounds__(kThreads) take_kernel(int32_t* ref, int pages, Table t, const int32_t* row, const int32_t* from, const int32_t* to, int n, int32_t* short_out) {
    extern __shared__ int64_t start[];                          // [kMostRequests], then what give_pages() wants
    int64_t* sums = start + kMostRequests;
    int32_t* found = reinterpret_cast<int32_t*>(sums + kWarps + 1);
    dev::programmatic_start();
    const int64_t wanted = starts_of(n, start, sums, [&](int i) -> int64_t {
        return row[i] < 0 || row[i] >= t.rows ? 0 : max(0, within(to[i], t.pages) - within(from[i], t.pages));
    });
    const int64_t missing = give_pages(ref, pages, wanted, sums, found, [&](int64_t place, int page) {
        const int i = owner_of(start, n, place);
        t.entries[row[i] * t.stride + within(from[i], t.pages) + (place - start[i])] = page;
    });
    if (short_out != nullptr && threadIdx.x == 0) *short_out = static_cast<int>(missing < INT32_MAX ? missing : INT32_MAX);
}

__global__ void __launch_bounds__(256) free_kernel(int32_t* ref, int pages, Table t, const int32_t* row, const int32_t* from, const int32_t* to) {
    dev::programmatic_start();
    const int i = blockIdx.x, r = row[i];
    if (r < 0 || r >= t.rows) return;
    const int64_t end = within(to[i], t.pages);                 // a row may have nearly 2^31 entries
    for (int64_t e = within(from[i], t.pages) + static_cast<int64_t>(threadIdx.x); e < end; e += blockDim.x) {
        const int page = atomicExch(&t.entries[r * t.stride + e], -1);      // so that an entry that is named twice is freed once
        if (page >= 0 && page < pages) atomicSub(&ref[page], 1);
    }
}

constexpr size_t kGiveBytes = (kMostRequests + kWarps + 1) * sizeof(int64_t) + kRun * sizeof(int32_t);

struct Forks {
    const int32_t* parent;
    const int32_t* child;
    const int32_t* length;
    int n, page_shift;
    __device__ __forceinline__ bool exists(const Table& t, int i) const { return parent[i] >= 0 && parent[i] < t.rows && child[i] >= 0 && child[i] < t.rows; }
    __device__ __forceinline__ int tokens(const Table& t, int i) const {
        const int64_t most = static_cast<int64_t>(t.pages) << page_shift;
        return static_cast<int>(length[i] < 0 ? 0 : length[i] < most ? length[i] : most);
    }
    __device__ __forceinline__ bool partly(int tokens) const { return (tokens & ((1 << page_shift) - 1)) != 0; }
};

// Block 0 takes pages for the children's last pages; the others share the full ones.
__global__ void __launch_bounds__(kThreads) fork_kernel(int32_t* ref, int pages, Table t, const Forks f, int32_t* short_out) {
    extern __shared__ int64_t start[];                          // [kMostRequests], then what give_pages() wants
    int64_t* sums = start + kMostRequests;
    int32_t* found = reinterpret_cast<int32_t*>(sums + kWarps + 1);
    dev::programmatic_start();
    if (blockIdx.x > 0) {
        for (int i = blockIdx.x - 1; i < f.n; i += gridDim.x - 1) {
            if (!f.exists(t, i)) continue;
            const int full = f.tokens(t, i) >> f.page_shift;
            for (int64_t e = threadIdx.x; e < full; e += kThreads) {
                const int page = t.entries[f.parent[i] * t.stride + e];
                const bool ok = page >= 0 && page < pages;
                t.entries[f.child[i] * t.stride + e] = ok ? page : -1;
                if (ok) atomicAdd(&ref[page], 1);
            }
        }
        return;
    }
    const int64_t wanted = starts_of(f.n, start, sums, [&](int i) -> int64_t {
        if (!f.exists(t, i) || !f.partly(f.tokens(t, i))) return 0;
        const int e = f.tokens(t, i) >> f.page_shift, page = t.entries[f.parent[i] * t.stride + e];
        if (page >= 0 && page < pages) return 1;
        t.entries[f.child[i] * t.stride + e] = -1;
        return 0;
    });
    const int64_t missing = give_pages(ref, pages, wanted, sums, found, [&](int64_t place, int page) {
        const int i = owner_of(start, f.n, place);
        t.entries[f.child[i] * t.stride + (f.tokens(t, i) >> f.page_shift)] = page;
    });
    if (short_out != nullptr && threadIdx.x == 0) *short_out = static_cast<int>(missing);
}

// ---- moving pages

struct Pages {
    unsigned char* cache;
    int64_t layer_stride, page_bytes;   // bytes
    int layers, pages;
};
constexpr int kMoveThreads = 256, kMoveLoads = 4;
constexpr int kPiece = 32 * kMoveLoads * 16;                    // bytes that a warp moves at a time

// Pages from_page(i) to to_page(i), i < n, in all layers; pairs of which one is no page are left out.  Every `warps`-th piece of a page is the warp's: the place of the
// next one by additions with carries, not by divisions.
template <typename From, typename To>
__device__ __forceinline__ void move_pages(const Pages& p, From from_page, To to_page, int64_t n, int64_t warp, int64_t warps) {
    const int64_t pieces = (p.page_bytes + kPiece - 1) / kPiece, of_pair = pieces * p.layers;
    int64_t i = warp / of_pair, layer = warp % of_pair / pieces, piece = warp % pieces;
    const int64_t step_i = warps / of_pair, step_layer = warps % of_pair / pieces, step_piece = warps % pieces;
    for (; i < n;) {
        const int a = from_page(i), b = to_page(i);
        if (a >= 0 && a < p.pages && b >= 0 && b < p.pages && a != b) {
            const int64_t at = piece * kPiece + 16 * (threadIdx.x & 31);
            const unsigned char* from = p.cache + layer * p.layer_stride + a * p.page_bytes + at;
            unsigned char* to = p.cache + layer * p.layer_stride + b * p.page_bytes + at;
            uint4 v[kMoveLoads];
#pragma unroll
            for (int j = 0; j < kMoveLoads; ++j)
                if (at + 512 * j < p.page_bytes) v[j] = __ldcs(reinterpret_cast<const uint4*>(from + 512 * j));
#pragma unroll
            for (int j = 0; j < kMoveLoads; ++j)
                if (at + 512 * j < p.page_bytes) __stcs(reinterpret_cast<uint4*>(to + 512 * j), v[j]);
        }
        piece += step_piece, layer += step_layer, i += step_i;
        if (piece >= pieces) piece -= pieces, ++layer;
        if (layer >= p.layers) layer -= p.layers, ++i;
    }
}
constexpr int kMoveWarps = kMoveThreads / 32;
__device__ __forceinline__ int64_t my_warp() { return static_cast<int64_t>(blockIdx.x) * kMoveWarps + (threadIdx.x >> 5); }
__global__ void __launch_bounds__(kMoveThreads) copy_kernel(const Pages p, const int32_t* src, const int32_t* dst, int64_t n) {
    dev::programmatic_start();
    move_pages(p, [&](int64_t i) { return src[i]; }, [&](int64_t i) { return dst[i]; }, n, my_warp(), static_cast<int64_t>(gridDim.x) * kMoveWarps);
}
// The partly filled pages of forks: where they come from and go to stands in the table.
__global__ void __launch_bounds__(kMoveThreads) copy_forks_kernel(const Pages p, const Table t, const Forks f) {
    dev::programmatic_start();
    auto entry = [&](const int32_t* row, int64_t i64) {
        const int i = static_cast<int>(i64), n = f.exists(t, i) ? f.tokens(t, i) : 0;
        return f.partly(n) ? t.entries[row[i] * t.stride + (n >> f.page_shift)] : -1;
    };
    move_pages(p, [&](int64_t i) { return entry(f.parent, i); }, [&](int64_t i) { return entry(f.child, i); }, f.n, my_warp(), static_cast<int64_t>(gridDim.x) * kMoveWarps);
}
unsigned move_ctas(const Pages& p, int64_t pairs, int sms) {
    const int64_t all = (pairs * p.layers * ((p.page_bytes + kPiece - 1) / kPiece) + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    return static_cast<unsigned>(all < 8 * sms ? (all > 0 ? all : 1) : 8 * sms);
}

// ---- bringing together
//
// With `live` pages in use, the i-th free page below `live` gets the i-th page in use from there on.  The pages are cut into runs, a CTA to each, up to
// kMostRuns of them.  Every run's place follows from the counts of all of them: a kernel of their own finds these where the pages are
// more than kCountPages; else each CTA looks at all pages itself.  A last kernel moves and renames.

constexpr int kMostRuns = 1024, kRunPages = 1024, kCountPages = 16384;
constexpr int kListThreads = 256;
struct Lists {
    int32_t* counts;                    // [runs] pages in use; null: not counted
    int32_t* place;                     // [pages] of the pages from `live` on: the one's place in the lists, or -1
    int32_t* src;                       // [pages / 2] pages to move
    int32_t* dst;                       // [pages / 2] and where to
    int32_t* moved;                     // how many, and behind it: pages in use
    int run, runs;                      // pages of a run
};

__global__ void __launch_bounds__(kListThreads) count_kernel(const int32_t* ref, int pages, Lists l) {
    __shared__ int count;
    dev::programmatic_start();
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * l.run, end = min(begin + l.run, static_cast<int64_t>(pages));
    int mine = 0;
    for (int64_t i = begin + threadIdx.x; i < end; i += kListThreads) mine += ref[i] > 0 ? 1 : 0;
    mine = __reduce_add_sync(kAll, mine);
    if ((threadIdx.x & 31) == 0) atomicAdd(&count, mine);
    __syncthreads();
    if (threadIdx.x == 0) l.counts[blockIdx.x] = count;
}

__device__ __forceinline__ int block_sum(int mine, int* word) {
    mine = __reduce_add_sync(kAll, mine);
    if (threadIdx.x == 0) *word = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) atomicAdd(word, mine);
    __syncthreads();
    const int r = *word;
    __syncthreads();
    return r;
}

__global__ void __launch_bounds__(kListThreads) list_kernel(const int32_t* ref, int pages, Lists l, int32_t* live_out) {
    __shared__ int word, warp_counts[kListThreads / 32];
    dev::programmatic_start();
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * l.run, end = min(begin + l.run, static_cast<int64_t>(pages));
    int all = 0, before = 0, below = 0, live;                   // pages in use: all of them, before this run, below `live`
    if (l.counts != nullptr) {
        for (int i = threadIdx.x; i < l.runs; i += kListThreads) {
            all += l.counts[i];
            if (i < blockIdx.x) before += l.counts[i];
        }
        live = block_sum(all, &word);
        const int cut = live / l.run;
        for (int i = threadIdx.x; i < cut; i += kListThreads) below += l.counts[i];
        for (int64_t i = static_cast<int64_t>(cut) * l.run + threadIdx.x; i < live; i += kListThreads) below += ref[i] > 0 ? 1 : 0;
    } else {
#pragma unroll 8
        for (int i = threadIdx.x; i < pages; i += kListThreads) {
            const int used = ref[i] > 0 ? 1 : 0;
            all += used;
            if (i < begin) before += used;
        }
        live = block_sum(all, &word);
#pragma unroll 8
        for (int i = threadIdx.x; i < live; i += kListThreads) below += ref[i] > 0 ? 1 : 0;
    }
    before = block_sum(before, &word);
    below = block_sum(below, &word);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        l.moved[0] = live - below, l.moved[1] = live;
        if (live_out != nullptr) *live_out = live;
    }
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int64_t base = begin; base < end; base += kListThreads) {
        const int64_t i = base + threadIdx.x;
        const bool used = i < end && ref[i] > 0;
        const unsigned bits = __ballot_sync(kAll, used);
        if (lane == 0) warp_counts[w] = __popc(bits);
        __syncthreads();
        int at = before + __popc(bits & ((1u << lane) - 1));    // pages in use before page i
        for (int j = 0; j < kListThreads / 32; ++j) {
            if (j < w) at += warp_counts[j];
            before += warp_counts[j];
        }
        if (i < end) {
            if (i < live) {
                if (!used) l.dst[i - at] = static_cast<int>(i);
            } else {
                l.place[i] = used ? at - below : -1;
                if (used) l.src[at - below] = static_cast<int>(i);
            }
        }
        __syncthreads();
    }
}

// The last `renamers` CTAs rename the table's entries and hand over the counts, the others move.
__global__ void __launch_bounds__(kMoveThreads) compact_kernel(const Pages p, int32_t* ref, Table t, Lists l, int renamers) {
    dev::programmatic_start();
    const int moved = *l.moved, movers = static_cast<int>(gridDim.x) - renamers;
    if (static_cast<int>(blockIdx.x) < movers) {
        move_pages(p, [&](int64_t i) { return l.src[i]; }, [&](int64_t i) { return l.dst[i]; }, moved, my_warp(), static_cast<int64_t>(movers) * kMoveWarps);
        return;
    }
    const int live = l.moved[1];
    const int64_t at = static_cast<int64_t>(blockIdx.x - movers) * kMoveThreads + threadIdx.x, step = static_cast<int64_t>(renamers) * kMoveThreads;
    for (int64_t i = at; i < moved; i += step) {
        ref[l.dst[i]] = ref[l.src[i]];
        ref[l.src[i]] = 0;
    }
    int64_t row = at / t.pages, column = at % t.pages;          // of the thread's entry; the next one's by additions with a carry
    const int64_t step_rows = step / t.pages, step_columns = step % t.pages;
    while (row < t.rows) {
        int32_t* entry = t.entries + row * t.stride + column;
        const int page = *entry;
        if (page >= live && page < p.pages) {
            const int place = l.place[page];
            if (place >= 0) *entry = l.dst[place];
        }
        row += step_rows, column += step_columns;
        if (column >= t.pages) column -= t.pages, ++row;
    }
}

// The current device, whose kernels that give pages may use the shared memory they want.
spdp_status ready(int* device, int* sms) {
    const spdp_status st = current_device(device, sms);
    if (st != SPDP_OK) return st;
    static std::mutex mu;
    static bool configured[64] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!configured[*device]) {
        SPDP_CUDA_TRY(cudaFuncSetAttribute(take_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kGiveBytes)));
        SPDP_CUDA_TRY(cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kGiveBytes)));
        configured[*device] = true;
    }
    return SPDP_OK;
}

Table table_of(const KvPagesCall& c) { return Table{c.table, c.table_stride, static_cast<int>(c.rows), static_cast<int>(c.table_pages)}; }
Pages pages_of(const KvPagesCall& c) { return Pages{c.cache, c.layer_stride, c.page_bytes, c.layers, static_cast<int>(c.pages)}; }

}  // namespace

spdp_status launch_kv_pages_take(const KvPagesCall& c, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = ready(&device, &sms);
    if (st != SPDP_OK) return st;
    SPDP_CUDA_TRY(launch_programmatic(take_kernel, dim3(1), kThreads, kGiveBytes, s, c.ref, static_cast<int>(c.pages), table_of(c), c.row, c.from, c.to, static_cast<int>(c.n), c.short_out));
    return SPDP_OK;
}

spdp_status launch_kv_pages_free(const KvPagesCall& c, cudaStream_t s) {
    if (c.n == 0) return SPDP_OK;
    SPDP_CUDA_TRY(launch_programmatic(free_kernel, dim3(static_cast<unsigned>(c.n)), 256, 0, s, c.ref, static_cast<int>(c.pages), table_of(c), c.row, c.from, c.to));
    return SPDP_OK;
}

spdp_status launch_kv_pages_copy(const KvPagesCall& c, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK || c.n == 0) return st;
    const Pages p = pages_of(c);
    SPDP_CUDA_TRY(launch_programmatic(copy_kernel, dim3(move_ctas(p, c.n, sms)), kMoveThreads, 0, s, p, c.row, c.to, c.n));
    return SPDP_OK;
}

spdp_status launch_kv_pages_fork(const KvPagesCall& c, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = ready(&device, &sms);
    if (st != SPDP_OK) return st;
    Forks f = {c.row, c.from, c.to, static_cast<int>(c.n), 0};
    while ((1 << f.page_shift) < c.page_tokens) ++f.page_shift;
    const Pages p = pages_of(c);
    const unsigned sharers = static_cast<unsigned>(c.n < sms ? c.n : sms);
    SPDP_CUDA_TRY(launch_programmatic(fork_kernel, dim3(1 + sharers), kThreads, kGiveBytes, s, c.ref, static_cast<int>(c.pages), table_of(c), f, c.short_out));
    if (c.n > 0) SPDP_CUDA_TRY(launch_programmatic(copy_forks_kernel, dim3(move_ctas(p, c.n, sms)), kMoveThreads, 0, s, p, table_of(c), f));
    return SPDP_OK;
}

spdp_status launch_kv_pages_compact(const KvPagesCall& c, cudaStream_t s) {
    int device = 0, sms = 0;
    spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    const int pages = static_cast<int>(c.pages);
    void* scratch = nullptr;
    Lists l;
    l.run = kRunPages * ((pages + kMostRuns * kRunPages - 1) / (kMostRuns * kRunPages)), l.runs = (pages + l.run - 1) / l.run;
    st = scratch_alloc(device, (l.runs + 2 + 2ll * pages + 2) * sizeof(int32_t), s, &scratch);
    if (st != SPDP_OK) return st;
    l.moved = static_cast<int32_t*>(scratch);
    l.place = l.moved + 2;
    l.src = l.place + pages;
    l.dst = l.src + pages / 2 + 1;
    l.counts = pages > kCountPages ? l.dst + pages / 2 + 1 : nullptr;
    const Pages p = pages_of(c);
    // CTAs that rename: an entry to a thread up to 4 of them to an SM, and 16 at least, for the counts.  With 16 for any table, 4096 rows of 512
    // entries take 721 us instead of 103, 1024 of 512 193 instead of 39, 64 of 29 the same 39.
    const int64_t entries = c.rows * c.table_pages, most = 4ll * sms, all = (entries + kMoveThreads - 1) / kMoveThreads;
    const int renamers = static_cast<int>(all < 16 ? 16 : all < most ? all : most);
    const int32_t* ref = c.ref;
    cudaError_t e = cudaSuccess;
    if (l.counts != nullptr) e = launch_programmatic(count_kernel, dim3(static_cast<unsigned>(l.runs)), kListThreads, 0, s, ref, pages, l);
    if (e == cudaSuccess) e = launch_programmatic(list_kernel, dim3(static_cast<unsigned>(l.runs)), kListThreads, 0, s, ref, pages, l, c.short_out);
    if (e == cudaSuccess) e = launch_programmatic(compact_kernel, dim3(move_ctas(p, pages / 2 + 1, sms) + renamers), kMoveThreads, 0, s, p, c.ref, table_of(c), l, renamers);
    const cudaError_t freed = cudaFreeAsync(scratch, s);
    SPDP_CUDA_TRY(e);
    SPDP_CUDA_TRY(freed);
    return SPDP_OK;
}

}  // namespace spdp
