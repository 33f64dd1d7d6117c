// The pages of a paged cache, kept on the device: sequences that share pages (fork), room for more tokens (extend), pages
// given back (free), pages and rows moved (copy, compact).
//
// State (PageTable): block_table[s][i] is the page of tokens i * page_size .. of sequence s or -1, page_refs[p] counts the
// table entries that name page p, free_pages[0 .. free_count) are the pages nobody names; the next one
// taken is the last of them. Every call leaves the same state whatever order its workgroups run in: references are
// counted with integer atomics, whose sum does not depend on the order; pages are taken by rank in the list given, and
// given back in ascending order.
//
// What bounds them: launches and chains of dependent reads (a table entry, then its page's count), a few us each; a
// copy moves its rows once.
#include "plx_device.h"
#include "plx_kernels.h"

namespace plx {

namespace {

constexpr int kBookThreads = 1024;

// Sum over the threads before this one, and over all, of a small count; every thread takes part
__device__ __forceinline__ int block_scan(int x, int *wave_sums, int &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
        const int up = __shfl_up(sum, step, 64);
        if (lane >= step) sum += up;
    }
    __syncthreads();  // (the sums of the scan before have been read)
    if (lane == 63) wave_sums[w] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
        const int s = wave_sums[i];
        before += i < w ? s : 0;
        total += s;
    }
    return before + sum - x;
}

__device__ __forceinline__ int pages_of(int tokens, int page_size) { return tokens / page_size + (tokens % page_size != 0); }

}  // namespace

// Child i's row := parent i's. One workgroup per pair.
__global__ __launch_bounds__(256) void cache_fork_kernel(PageTable t, const int32_t *parents, const int32_t *children, int n) {
    __shared__ int refused;
    const int i = blockIdx.x, tid = threadIdx.x;
    const int parent = parents[i], child = children[i];
    if (parent < 0 || parent >= t.sequences || child < 0 || child >= t.sequences || parent == child) return;  // (uniform)
    if (tid == 0) refused = 0;
    __syncthreads();
    for (int j = tid; j < n; j += 256)
        if (parents[j] == child || (j < i && children[j] == child)) refused = 1;
    if (t.seq_lens[child] != 0 && tid == 0) refused = 1;
    __syncthreads();
    if (refused) return;
    const int length = min(max(t.seq_lens[parent], 0), t.pages_per_sequence * t.page_size);
    const int held = pages_of(length, t.page_size);
    const int32_t *from = t.block_table + (int64_t)parent * t.stride;
    int32_t *to = t.block_table + (int64_t)child * t.stride;
    for (int p = tid; p < t.pages_per_sequence; p += 256) {
        int page = p < held ? from[p] : -1;
        if (page >= t.num_pages || page < 0) page = -1;
        to[p] = page;
        if (page >= 0) atomicAdd(t.page_refs + page, 1);
    }
    if (tid == 0) t.seq_lens[child] = length;  // (read by no other pair: it is nobody's parent, and later pairs with it are refused)
}

// Room for new_lens[i] tokens in sequence seqs[i]: one workgroup, a thread per listed sequence, then a thread per table entry
// to fill. The entries of all sequences are numbered one after the other: of sequence i that of its partly filled last
// page, if it takes a page there (a copy, or the first where that page had been given back), then those behind it.
__global__ __launch_bounds__(kBookThreads) void cache_extend_kernel(PageTable t, const int32_t *seqs, const int32_t *new_lens, int n,
                                                                    int32_t *src, int32_t *dst, int32_t *rows, int32_t *missing) {
    __shared__ int wave_sums[kBookThreads / 64];
    __shared__ int seq[kBookThreads], tail_page[kBookThreads], first_entry[kBookThreads], first_page[kBookThreads];
    __shared__ bool copies[kBookThreads];
    const int tid = threadIdx.x;
    int s = tid < n ? seqs[tid] : -1;
    if (s < 0 || s >= t.sequences) s = -1;
    seq[tid] = s;
    __syncthreads();
    for (int j = 0; j < min(tid, n); ++j)  // (a sequence listed twice: the first time counts)
        if (seq[j] == seq[tid]) s = -1;
    const int capacity = t.pages_per_sequence * t.page_size;
    int length = 0, to = 0, tail = -1;
    bool hole = false;  // the last page, partly filled, has been given back
    if (s >= 0) {
        length = min(max(t.seq_lens[s], 0), capacity);
        to = min(max(new_lens[tid], length), capacity);
        if (to > length && length % t.page_size != 0) {
            tail = t.block_table[(int64_t)s * t.stride + length / t.page_size];
            hole = tail < 0;
            if (tail >= t.num_pages) tail = -1;
        }
    }
    tail_page[tid] = tail;
    __syncthreads();
    // A last page that others name too is copied before it is written. The others listed before this one have left
    // it by then; whoever names it alone keeps it.
    bool copied = false;
    if (tail >= 0) {
        int earlier = 0;
        for (int j = 0; j < tid; ++j) earlier += tail_page[j] == tail;
        copied = t.page_refs[tail] - earlier > 1;
    }
    const int from = pages_of(length, t.page_size) - (copied || hole ? 1 : 0);
    int n_entries;
    first_entry[tid] = block_scan(pages_of(to, t.page_size) - from, wave_sums, n_entries);
    first_page[tid] = from, copies[tid] = copied;
    if (tid < n) src[tid] = dst[tid] = -1, rows[tid] = 0;
    __syncthreads();
    // entry e -> which of the listed sequences, and where its table entry is; does it take a page?
    auto entry = [&](int e, int &i) {
        int lo = 0, hi = n - 1;  // the last sequence whose first entry is not behind e
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first_entry[mid] <= e)
                lo = mid;
            else
                hi = mid - 1;
        }
        i = lo;
        return t.block_table + (int64_t)seq[lo] * t.stride + first_page[lo] + (e - first_entry[lo]);
    };
    auto takes = [&](int e, int i, const int32_t *at) { return (copies[i] && e == first_entry[i]) || *at < 0; };
    const int available = min(max(*t.free_count, 0), t.num_pages);
    struct Found {
        int32_t *at;
        int i, rank;
        bool take;
    };
    auto find = [&](int e0, int taken, int &sum) {
        Found f{};
        if (e0 + tid < n_entries) f.at = entry(e0 + tid, f.i), f.take = takes(e0 + tid, f.i, f.at);
        f.rank = taken + block_scan(f.take ? 1 : 0, wave_sums, sum);
        return f;
    };
    int total = 0;
    Found first_found{};  // (most calls have no more than these)
    for (int e0 = 0; e0 < n_entries; e0 += kBookThreads) {
        int sum;
        const Found f = find(e0, total, sum);
        if (e0 == 0) first_found = f;
        total += sum;
    }
    if (tid == 0) *missing = max(total - available, 0);
    if (total > available) return;  // (uniform) all or nothing
    int taken = 0;
    for (int e0 = 0; e0 < n_entries; e0 += kBookThreads) {
        int sum = 0;
        const Found f = e0 == 0 ? first_found : find(e0, taken, sum);
        if (n_entries > kBookThreads && e0 == 0) block_scan(f.take ? 1 : 0, wave_sums, sum);
        taken += sum;
        const int e = e0 + tid, i = f.i;
        if (!f.take) continue;
        int32_t *slot = t.free_pages + (available - 1 - f.rank);
        const int page = *slot;
        *slot = -1;
        if (page < 0 || page >= t.num_pages) continue;  // (a list that was not kept by these calls)
        if (copies[i] && e == first_entry[i]) {
            atomicSub(t.page_refs + tail_page[i], 1);
            src[i] = tail_page[i], dst[i] = page;
        }
        *f.at = page;
        t.page_refs[page] = 1;
    }
    if (copied) rows[tid] = length % t.page_size;
    if (s >= 0) t.seq_lens[s] = max(length, to);
    if (tid == 0) *t.free_count = available - total;
}

// Marks a page that has just lost its last reference, until cache_collect_kernel puts it on the free list
constexpr int kJustFreed = -1;

// The whole pages inside [first, last) of every listed sequence lose the sequence's reference
__global__ __launch_bounds__(256) void cache_release_kernel(PageTable t, const int32_t *seqs, const int32_t *first, const int32_t *last) {
    const int i = blockIdx.x, s = seqs[i];
    if (s < 0 || s >= t.sequences) return;
    const int length = min(max(t.seq_lens[s], 0), t.pages_per_sequence * t.page_size);
    const int from = first ? max(first[i], 0) : 0, to = last ? last[i] : length;
    const int lo = pages_of(from, t.page_size);
    const int hi = to >= length ? pages_of(length, t.page_size) : max(to, 0) / t.page_size;  // (the end takes the partial page along)
    for (int p = lo + blockIdx.y * 256 + threadIdx.x; p < hi; p += 256 * gridDim.y) {
        // (exchanged: of two listings of a sequence one finds the page)
        const int page = atomicExch(t.block_table + (int64_t)s * t.stride + p, -1);
        if (page < 0 || page >= t.num_pages) continue;
        if (atomicSub(t.page_refs + page, 1) == 1) atomicExch(t.page_refs + page, kJustFreed);
    }
}

// ... and the pages that nobody names any more go on top of the free list, in ascending order; sequences whose end has
// gone are shorter. One workgroup, 16 pages a thread at a time: the counts of 16384 pages are fetched together, and one barrier
// tells every wave how many pages were freed before each of its 64-page runs (16384 pages: 10.8 us with four pages a thread, four
// rounds of two barriers; now 8.7).
__global__ __launch_bounds__(kBookThreads) void cache_collect_kernel(PageTable t, const int32_t *seqs, const int32_t *first,
                                                                     const int32_t *last, int n) {
    constexpr int RUNS = 16, WAVES = kBookThreads / 64;
    __shared__ int counts[2][RUNS * WAVES];  // freed pages of run j of wave w, pages ascending
    static_assert(RUNS * WAVES == 4 * 64, "four runs a lane");
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    // (all lengths are read before any is changed: a sequence may be listed again; 65535 of them are 64 a thread)
    uint64_t ends = 0;
    for (int i = tid, bit = 0; i < n; i += kBookThreads, ++bit) {
        const int s = seqs[i];
        if (s >= 0 && s < t.sequences && (!last || last[i] >= t.seq_lens[s])) ends |= 1ull << bit;
    }
    int count = min(max(*t.free_count, 0), t.num_pages), buffer = 0;
    for (int64_t p0 = 0; p0 < t.num_pages; p0 += RUNS * kBookThreads, buffer ^= 1) {
        int refs[RUNS];
        uint64_t freed[RUNS];
#pragma unroll
        for (int j = 0; j < RUNS; ++j) refs[j] = t.page_refs[min(p0 + j * kBookThreads + tid, (int64_t)t.num_pages - 1)];
#pragma unroll
        for (int j = 0; j < RUNS; ++j) {
            freed[j] = __ballot((refs[j] == kJustFreed) & (p0 + j * kBookThreads + tid < t.num_pages));
            if (lane == 0) counts[buffer][WAVES * j + w] = __popcll(freed[j]);
        }
        __syncthreads();  // (of two buffers the one written next was read before the barrier in between)
        // lane l: the runs 4 l .. 4 l + 3; its sum over all runs before
        int run[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) run[j] = sum, sum += counts[buffer][4 * lane + j];
        int before = sum;
#pragma unroll
        for (int step = 1; step < 64; step <<= 1) {
            const int up = __shfl_up(before, step, 64);
            if (lane >= step) before += up;
        }
        const int all = __shfl(before, 63, 64);
        before -= sum;
#pragma unroll
        for (int j = 0; j < RUNS; ++j) {
            const int r = WAVES * j + w;  // (uniform) r % 4 of lane r / 4
            const int inside = r % 4 == 0 ? run[0] : r % 4 == 1 ? run[1] : r % 4 == 2 ? run[2] : run[3];
            const int at = count + __shfl(before + inside, r / 4, 64) + __popcll(freed[j] & ((1ull << lane) - 1));
            if ((freed[j] >> lane) & 1) {
                const int64_t p = p0 + j * kBookThreads + tid;
                t.page_refs[p] = 0;
                if (at < t.num_pages) t.free_pages[at] = (int)p;
            }
        }
        count += all;
    }
    __syncthreads();
    for (int i = tid, bit = 0; i < n; i += kBookThreads, ++bit)
        if ((ends >> bit) & 1) atomicMin(t.seq_lens + seqs[i], first ? max(first[i], 0) : 0);
    if (tid == 0) *t.free_count = min(count, t.num_pages);
}

// rows[i] rows (NULL: all) of page src[i] -> page dst[i] of every pool, 16 bytes a thread
__global__ __launch_bounds__(256) void cache_copy_kernel(CachePools c, const int32_t *src, const int32_t *dst, const int32_t *rows) {
    const int i = blockIdx.x, from = src[i], to = dst[i];
    if (from < 0 || from >= c.num_pages || to < 0 || to >= c.num_pages || from == to) return;
    const int n_rows = rows ? min(max(rows[i], 0), c.page_size) : c.page_size;
    // (up to 2^30 - 1 chunks a pool, 2^31 - 2 in all, and a stride of up to 2^24 behind the last: 32 bits without a sign)
    const uint32_t pool_chunks = (uint32_t)c.heads * n_rows * c.row_chunks;
    const uint32_t total = c.v ? 2 * pool_chunks : pool_chunks;
    for (uint32_t e = blockIdx.y * 256 + threadIdx.x; e < total; e += 256 * gridDim.y) {
        const bool second = e >= pool_chunks;
        const int x = (int)(second ? e - pool_chunks : e);
        const int chunk = x % c.row_chunks, hr = x / c.row_chunks, row = hr % n_rows, head = hr / n_rows;
        char *base = second ? c.v : c.k;
        const int64_t *st = second ? c.vs : c.ks;
        const int64_t at = head * st[1] + row * st[2] + 16 * chunk;
        *(u32x4 *)(base + to * st[0] + at) = *(const u32x4 *)(base + from * st[0] + at);
    }
}

// Row base + accepted[i] -> base + i, i ascending, of every head of every pool. A thread owns 16 bytes of a row and moves
// them for all i, eight rows at a time, loads before stores: accepted[i] >= i and ascending, so no row is
// written before it has been read.
__global__ __launch_bounds__(256) void cache_compact_kernel(CacheCompact a) {
    __shared__ int64_t at[2][2][256];  // byte offsets [pool][from, to][move]
    __shared__ bool moves[256];
    const CachePools &c = a.pools;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int length = min(max(a.seq_lens[b], 0), a.capacity);
    const int n = min(min(a.draft_lens ? max(a.draft_lens[b], 0) : a.max_draft, a.max_draft), length), base = length - n;
    const int count = min(min(max(a.n_accepted[b], 0), n), a.max_accepted);
    if (blockIdx.y == 0 && tid == 0) a.new_lens[b] = base + count;
    auto row_at = [&](int key, const int64_t (&st)[3]) -> int64_t {
        if (a.block_table == nullptr) return (int64_t)b * st[0] + (int64_t)key * st[2];
        const int page = a.block_table[(int64_t)b * a.table_stride + key / c.page_size];
        if (page < 0 || page >= c.num_pages) return -1;  // (no page: no row is moved from or to it)
        return (int64_t)page * st[0] + (int64_t)(key % c.page_size) * st[2];
    };
    for (int i = tid; i < count; i += 256) {
        const int node = min(max(a.accepted[(int64_t)b * a.max_accepted + i], i), n - 1);
        at[0][0][i] = row_at(base + node, c.ks), at[0][1][i] = row_at(base + i, c.ks);
        moves[i] = node != i && at[0][0][i] >= 0 && at[0][1][i] >= 0;
        if (c.v) at[1][0][i] = row_at(base + node, c.vs), at[1][1][i] = row_at(base + i, c.vs);
    }
    __syncthreads();
    const int e = blockIdx.y * 256 + tid, pool_chunks = c.heads * c.row_chunks;
    if (e >= (c.v ? 2 : 1) * pool_chunks) return;
    const int pool = e >= pool_chunks, x = e - pool * pool_chunks;
    char *mine = (pool ? c.v + (x / c.row_chunks) * c.vs[1] : c.k + (x / c.row_chunks) * c.ks[1]) + 16 * (x % c.row_chunks);
    for (int i0 = 0; i0 < count; i0 += 8) {
        u32x4 row[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i0 + j < count && moves[i0 + j]) row[j] = *(const u32x4 *)(mine + at[pool][0][i0 + j]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i0 + j < count && moves[i0 + j]) *(u32x4 *)(mine + at[pool][1][i0 + j]) = row[j];
    }
}

hipError_t launch_cache_fork(const PageTable &t, const int32_t *parents, const int32_t *children, int n, hipStream_t stream) {
    hipLaunchKernelGGL(cache_fork_kernel, dim3(n), dim3(256), 0, stream, t, parents, children, n);
    return hipGetLastError();
}

hipError_t launch_cache_extend(const PageTable &t, const int32_t *seqs, const int32_t *new_lens, int n, int32_t *src, int32_t *dst,
                               int32_t *rows, int32_t *missing, hipStream_t stream) {
    hipLaunchKernelGGL(cache_extend_kernel, dim3(1), dim3(kBookThreads), 0, stream, t, seqs, new_lens, n, src, dst, rows, missing);
    return hipGetLastError();
}

hipError_t launch_cache_free(const PageTable &t, const int32_t *seqs, const int32_t *first, const int32_t *last, int n,
                             hipStream_t stream) {
    const int parts = (t.pages_per_sequence + 255) / 256;
    hipLaunchKernelGGL(cache_release_kernel, dim3(n, parts < 64 ? parts : 64), dim3(256), 0, stream, t, seqs, first, last);
    if (hipError_t err = hipGetLastError()) return err;
    hipLaunchKernelGGL(cache_collect_kernel, dim3(1), dim3(kBookThreads), 0, stream, t, seqs, first, last, n);
    return hipGetLastError();
}

hipError_t launch_cache_copy(const CachePools &c, const int32_t *src, const int32_t *dst, const int32_t *rows, int n,
                             hipStream_t stream) {
    const int64_t chunks = (int64_t)c.heads * c.page_size * c.row_chunks * (c.v ? 2 : 1);
    const int64_t parts = (chunks + 1023) / 1024;  // (four chunks a thread)
    hipLaunchKernelGGL(cache_copy_kernel, dim3(n, (unsigned)(parts < 65535 ? parts : 65535)), dim3(256), 0, stream, c, src, dst, rows);
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheCompact &a, hipStream_t stream) {
    const int chunks = a.pools.heads * a.pools.row_chunks * (a.pools.v ? 2 : 1);
    hipLaunchKernelGGL(cache_compact_kernel, dim3(a.B, (chunks + 255) / 256), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace plx
