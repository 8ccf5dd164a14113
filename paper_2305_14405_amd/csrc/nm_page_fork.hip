// Block tables of a new batch whose rows go on from rows of the old one (nm_page_fork).
//
// Nothing is counted from call to call: who refers to a page is found from the tables.  Each page has marks: that an old row refers to it; that one with
// children does so in front of its partial last page; how many rows with children have it as that.  From them follow which rows take a page
// of their own (a scan over the rows) and which pages become free (a scan over the pages).  Marks are set by stores of one value, and counted by integer
// atomics, whose order does not change their result.
//   Small batches: one workgroup, marks in LDS, a chain of dependent steps: 16 rows of up to 135 entries 7.2 us.  Others: four kernels, marks in the workspace.  Clear them
// and find every old row's first child; mark (a row leaves out what the row in front of it marks as well: hypotheses of a request share most of their pages,
// and 4096 rows that all marked theirs by atomics took 53 us, 13 so); decide for the rows, and count the freed pages of every block; write the tables and the
// list.  4096 rows, 860000 entries, a pool of 332000 pages (6.9 MB that the call cannot do without): 3.2 + 13.2 + 4.7 + 4.6 us, each a chain of three
// or four dependent loads; marks are bytes at scattered places.  (The decisions for all rows in one workgroup took 12 to 17: 8192 lines through one CU.)
#include <algorithm>

#include "nm_decode.h"

namespace nm {

constexpr int kForkThreads = 256;
constexpr int kForkBlocks = 1024;                  // of pages at most
constexpr int kForkBlock = 4096;                   // pages of one at least
constexpr int kRowThreads = 1024, kRows = NM_PLAN_MAX_REQUESTS / kRowThreads;
constexpr int kRowBlocks = NM_PLAN_MAX_REQUESTS / kForkThreads;   // of rows at most
// What one workgroup does alone: rows, entries of either table, pages, the list.  (GPU time there and by four kernels: 16 rows of 135 entries 7.2 and 10.1 us, 64 10.0 and
// 10.7, 128 13.8 and 11.5, 256 23.6 and 11.6, of 38 18.1 and 11.1; but it is one launch, and they are four.)
constexpr int kSmallRows = 128, kSmallEntries = 16384, kSmallPages = 65536, kSmallList = 65536;

struct ForkArgs {
    nm_fork_desc d;
    int shift;
    int blocks, block;                             // of pages, and their length
    int list_blocks;
    int* marks;                                    // [num_pages, up to a multiple of kRun]: kKept, and kPart for every row with children that has it as its last
    uint8_t* old;                                  // [2, likewise]: an old row refers to the page; one with children does, in front of its partial last page
    long padded;                                   // num_pages up to a multiple of kRun
    int* first;                                    // [B_in]: lowest-numbered child, B_out: none
    int4* rows;                                    // [B_out]: parent (-1: none), its length, its partial last page (-1: none), whether this is its first child;
                                                   // then: its place among its block's rows that take a page, -1 where it does not
    int* taken;                                    // [B_out]: what the list holds from its begin on (which may be written over before it is asked for)
    int* freed;                                    // [blocks]: pages that become free
    int* sums;                                     // [kRowBlocks]: of a block of rows, pages wanted, and rows with a parent from bit 16 on
    int* bad;                                      // [1]: whether a length is bad
};
enum { kOld = 1, kFull = 2, kKept = 4, kPart = 8 };   // kKept: by keep; kPart and above: how many rows with children have it as their partial last page
constexpr int kRun = 16;                           // neighbouring pages of a thread

// Tokens of an old row, 0 where its length is bad.
__device__ __forceinline__ int good_length(const ForkArgs& a, int n) { return n < 0 || n > (long)a.d.max_pages << a.shift ? 0 : n; }
__device__ __forceinline__ int length_of(const ForkArgs& a, int r) { return good_length(a, a.d.lens[r]); }
__device__ __forceinline__ int held_of(const ForkArgs& a, int n) { return (int)(((long)n + a.d.page_size - 1) >> a.shift); }
__device__ __forceinline__ bool is_page(const ForkArgs& a, int e) { return e >= 0 && e < a.d.num_pages; }
__device__ __forceinline__ bool is_row(const ForkArgs& a, int p) { return p >= 0 && p < a.d.B_in; }

// By a page's marks: whether its one user with children may keep it as its partial last page, and whether it becomes free.
__device__ __forceinline__ bool stays(int m) { return !(m & (kFull | kKept)) && m / kPart == 1; }
__device__ __forceinline__ bool goes(int m) { return (m & (kOld | kFull | kKept)) == kOld && m / kPart != 1; }

// Sums over the workgroup's threads in front, and over all.  s: LDS of a number for each wavefront.
struct Sums { int before, all; };
template <int kThreads>
__device__ __forceinline__ Sums scan(int mine, int* s)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int in = mine;
    for (int step = 1; step < 64; step <<= 1) {
        const int t = __shfl_up(in, step);
        if (lane >= step) in += t;
    }
    __syncthreads();                               // s may be in use
    if (lane == 63) s[wave] = in;
    __syncthreads();
    Sums r{in - mine, 0};
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const int x = s[w];
        r.before += w < wave ? x : 0;
        r.all += x;
    }
    return r;
}

// Flags of a call from those of its lengths, the pages wanted and the pages that become free; where the list begins behind it.
__device__ __forceinline__ int all_flags(const ForkArgs& a, int flags, int begin, int wanted, int freed)
{
    if (begin >= 0 && begin <= a.d.n_free) {
        if ((long)begin + wanted > a.d.n_free) flags |= NM_FORK_NO_PAGES;
        if ((long)begin + wanted - freed < 0) flags |= NM_FORK_LIST_FULL;
    }
    return flags;
}
__device__ __forceinline__ void report(const ForkArgs& a, int flags, int wanted, int freed, int parents, int end)
{
    a.d.status[0] = flags;
    a.d.status[1] = wanted;
    a.d.status[2] = freed;
    a.d.status[3] = parents;
    *a.d.free_end = end;
}

__global__ __launch_bounds__(kRowThreads) void fork_clear_kernel(ForkArgs a)
{
    __shared__ int s_first[NM_PLAN_MAX_REQUESTS];
    if (blockIdx.x) {
        const long first = (long)(blockIdx.x - 1) * kRowThreads + threadIdx.x, step = (long)(gridDim.x - 1) * kRowThreads;
        for (long i = first; i < a.padded; i += step) a.marks[i] = a.d.keep && i < a.d.num_pages && a.d.keep[i] ? kKept : 0;
        for (long i = first; i < a.padded / 2; i += step) reinterpret_cast<int*>(a.old)[i] = 0;
        return;
    }
    for (int r = threadIdx.x; r < a.d.B_in; r += kRowThreads) s_first[r] = a.d.B_out;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int b = threadIdx.x + i * kRowThreads, p = b < a.d.B_out ? a.d.parents[b] : -1;
        if (is_row(a, p)) atomicMin(&s_first[p], b);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < a.d.B_in; r += kRowThreads) a.first[r] = s_first[r];
}

// Workgroups: of new rows, what is to be decided for them, a thread to each; then of old rows, which set their marks, a wavefront to each.
__global__ __launch_bounds__(kForkThreads) void fork_mark_kernel(ForkArgs a)
{
    const nm_fork_desc& d = a.d;
    const int news = (d.B_out + kForkThreads - 1) / kForkThreads, lane = threadIdx.x & 63;
    if ((int)blockIdx.x < news) {
        const int b = blockIdx.x * kForkThreads + threadIdx.x;
        if (b >= d.B_out) return;
        const int p = d.parents[b];
        const long at = (long)*d.free_begin + b;
        a.taken[b] = at >= 0 && at < d.n_free ? d.free_pages[at] : -1;
        if (!is_row(a, p)) {
            a.rows[b] = make_int4(-1, 0, -1, 0);
            return;
        }
        const int n = length_of(a, p), page = n & (d.page_size - 1) ? d.block_table[p * d.table_stride + (n >> a.shift)] : -1;
        a.rows[b] = make_int4(p, n, is_page(a, page) ? page : -1, a.first[p] == b);
        return;
    }
    const int r = ((int)blockIdx.x - news) * (kForkThreads / 64) + (int)(threadIdx.x / 64), q = max(r - 1, 0);
    if (r >= d.B_in) return;
    const int n = length_of(a, r), whole = n >> a.shift, held = held_of(a, n);
    const bool lives = a.first[r] < d.B_out;
    // of the row in front: how many entries it marks, and how many of them as kFull
    const int n_front = r ? length_of(a, q) : 0, held_front = held_of(a, n_front), full_front = a.first[q] < d.B_out ? n_front >> a.shift : 0;
    const int* row = d.block_table + r * d.table_stride;
    const int* front = d.block_table + q * d.table_stride;
    constexpr int kAtOnce = 4;
    for (int i0 = lane; i0 < held; i0 += 64 * kAtOnce) {
        int page[kAtOnce], same[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = min(i0 + 64 * k, held - 1);
            page[k] = row[i];
            same[k] = front[held_front ? min(i, held_front - 1) : 0];   // (a row without entries: its first is not looked at)
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = i0 + 64 * k;
            if (i >= held || !is_page(a, page[k])) continue;
            int mark = kOld | (lives && i < whole ? kFull : 0);
            if (i < held_front && same[k] == page[k]) mark &= i < full_front ? 0 : ~kOld;
            // one value, whoever writes it
            if (mark & kOld) __hip_atomic_store(a.old + page[k], (uint8_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (mark & kFull) __hip_atomic_store(a.old + a.padded + page[k], (uint8_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (lives && i >= whole) atomicAdd(a.marks + page[k], kPart);
        }
    }
}

// A run of pages from p on: those that become free, as bits.
__device__ __forceinline__ unsigned freed_of(const ForkArgs& a, long p)
{
    const v4i old = *reinterpret_cast<const v4i*>(a.old + p), full = *reinterpret_cast<const v4i*>(a.old + a.padded + p);
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < kRun; i += 4) {
        const v4i m = *reinterpret_cast<const v4i*>(a.marks + p + i);
        const int free = old[i / 4] & ~full[i / 4];            // a byte each, 0 or 1
#pragma unroll
        for (int k = 0; k < 4; ++k) bits |= free >> 8 * k & 1 && !(m[k] & kKept) && m[k] / kPart != 1 ? 1u << (i + k) : 0u;
    }
    return bits;
}

// Workgroups: of blocks of pages, then of rows; and one that looks at the lengths.
__global__ __launch_bounds__(kForkThreads) void fork_decide_kernel(ForkArgs a)
{
    __shared__ int s[kForkThreads / 64];
    const nm_fork_desc& d = a.d;
    const int tid = threadIdx.x, block = blockIdx.x, news = (d.B_out + kForkThreads - 1) / kForkThreads;
    if (block < a.blocks) {
        const long p0 = (long)block * a.block, p1 = min(p0 + a.block, (long)d.num_pages);
        int n = 0;
        for (long p = p0 + tid * kRun; p < p1; p += kForkThreads * kRun) n += __popc(freed_of(a, p));
        const Sums all = scan<kForkThreads>(n, s);
        if (tid == 0) a.freed[block] = all.all;
    } else if (block - a.blocks < news) {
        const int b = (block - a.blocks) * kForkThreads + tid;
        const int4 row = b < d.B_out ? a.rows[b] : make_int4(-1, 0, -1, 0);
        bool need = false;
        if (row.z >= 0) need = !row.w || !stays(a.marks[row.z] | (a.old[a.padded + row.z] ? kFull : 0));
        const Sums sums = scan<kForkThreads>((int)need | (int)(row.x >= 0) << 16, s);
        if (b < d.B_out) a.rows[b].w = need ? sums.before & 0xffff : -1;
        if (tid == 0) a.sums[block - a.blocks] = sums.all;
    } else {
        const int begin = *d.free_begin;
        bool bad = begin < 0 || begin > d.n_free;
        for (int r = tid; r < d.B_in; r += kForkThreads) {
            const int n = d.lens[r];
            bad |= n != good_length(a, n);
        }
        bad = __syncthreads_or(bad);
        if (tid == 0) *a.bad = bad;
    }
}

// Workgroups: blocks of pages, then rows, a wavefront to each, then blocks of the list.
__global__ __launch_bounds__(kForkThreads) void fork_write_kernel(ForkArgs a)
{
    __shared__ int s[kForkThreads / 64];
    const nm_fork_desc& d = a.d;
    const int block = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    // asked for ahead of what decides whether they are written
    const int b = (block - a.blocks) * (kForkThreads / 64) + tid / 64;
    const bool pages = block < a.blocks, rows = !pages && block - a.blocks < (d.B_out + kForkThreads / 64 - 1) / (kForkThreads / 64);
    const int4 row = rows && b < d.B_out ? a.rows[b] : make_int4(-1, 0, -1, 0);
    int before = 0, all = 0;                       // freed pages of the blocks in front of this one, and of all
    for (int i = tid; i < a.blocks; i += kForkThreads) {
        const int n = a.freed[i];
        all += n;
        before += i < block ? n : 0;
    }
    // pages that rows want, and rows with a parent; what the blocks in front of this wavefront's row want
    const int sum = lane * kForkThreads < d.B_out ? a.sums[lane] : 0, sums = group_reduce<64>(sum, AddI32{});
    const int front = group_reduce<64>(lane < b / kForkThreads ? sum & 0xffff : 0, AddI32{});
    all = scan<kForkThreads>(all, s).all;
    const int begin = *d.free_begin, wanted = sums & 0xffff, flags = all_flags(a, *a.bad ? NM_FORK_BAD_LENGTH : 0, begin, wanted, all);
    const bool ok = flags == 0;
    const int end = ok ? begin + wanted - all : begin;
    if (block == 0 && tid == 0) report(a, flags, wanted, all, sums >> 16, end);
    if (pages) {
        if (!ok) return;
        long at = (long)end + scan<kForkThreads>(before, s).all;
        const long p0 = (long)block * a.block, p1 = min(p0 + a.block, (long)d.num_pages);
        for (long p = p0; p < p1; p += kForkThreads * kRun) {
            unsigned bits = p + tid * kRun < p1 ? freed_of(a, p + tid * kRun) : 0;
            const Sums sums = scan<kForkThreads>(__popc(bits), s);
            for (long to = at + sums.before; bits; bits &= bits - 1) d.free_out[to++] = (int)p + tid * kRun + __ffs((int)bits) - 1;
            at += sums.all;
        }
    } else if (rows) {
        if (b >= d.B_out) return;
        const int n = ok ? row.y : 0, held = held_of(a, n);
        const bool need = ok && row.w >= 0;
        const int dst = need ? a.taken[front + row.w] : -1;
        const int* from = d.block_table + (long)max(row.x, 0) * d.table_stride;
        int* to = d.table_out + b * d.table_out_stride;
        constexpr int kAtOnce = 4;
        for (int i0 = lane; i0 < held; i0 += 64 * kAtOnce) {
            int x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) x[k] = from[min(i0 + 64 * k, held - 1)];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (i0 + 64 * k < held) to[i0 + 64 * k] = need && i0 + 64 * k == n >> a.shift ? dst : x[k];
        }
        if (lane == 0) {
            d.lens_out[b] = n;
            d.copy_src[b] = need ? row.z : -1;
            d.copy_dst[b] = dst;
            d.copy_slots[b] = need ? n & (d.page_size - 1) : 0;
        }
    } else if (d.free_out != d.free_pages && begin >= 0) {
        const int first = block - a.blocks - (d.B_out + kForkThreads / 64 - 1) / (kForkThreads / 64);
        for (long i = (long)begin + (ok ? wanted : 0) + (long)first * kForkThreads + tid; i < d.n_free; i += (long)a.list_blocks * kForkThreads)
            d.free_out[i] = d.free_pages[i];
    }
}

// All of it in one workgroup.  A page's marks are four bits in LDS: kOld, kFull, one row's partial last page, and another's.
__global__ __launch_bounds__(kRowThreads) void fork_small_kernel(ForkArgs a)
{
    extern __shared__ unsigned s_marks[];          // eight pages to a word
    __shared__ int s_first[kRowThreads], s_n[kRowThreads], s_src[kRowThreads], s_dst[kRowThreads], s[kRowThreads / 64];
    const nm_fork_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, words = (d.num_pages + 7) / 8;
    const int begin = *d.free_begin;
    // a thread to a row, of either batch
    const int raw = tid < d.B_in ? d.lens[tid] : 0, parent = tid < d.B_out ? d.parents[tid] : -1;
    const bool child = is_row(a, parent);
    for (int i = tid; i < words; i += kRowThreads) s_marks[i] = 0;
    s_first[tid] = d.B_out;
    s_n[tid] = good_length(a, raw);
    const bool bad = __syncthreads_or(raw != good_length(a, raw) || begin < 0 || begin > d.n_free);
    if (child) atomicMin(&s_first[parent], tid);
    __syncthreads();
    auto marks_of = [&](int page) {
        const unsigned m = s_marks[page / 8] >> page % 8 * 4;
        return (int)(m & (kOld | kFull)) + (int)((m >> 2 & 1) + (m >> 3 & 1)) * kPart + (d.keep && d.keep[page] ? kKept : 0);
    };
    for (int r = wave; r < d.B_in; r += kRowThreads / 64) {
        const int n = s_n[r], whole = n >> a.shift, held = held_of(a, n);
        const bool lives = s_first[r] < d.B_out;
        for (int i = lane; i < held; i += 64) {
            const int page = d.block_table[r * d.table_stride + i];
            if (!is_page(a, page)) continue;
            const int at = page % 8 * 4;
            const bool part = lives && i >= whole;
            const unsigned was = atomicOr(&s_marks[page / 8], (unsigned)(kOld | (part ? 4 : lives ? kFull : 0)) << at);
            if (part && (was >> at & 4)) atomicOr(&s_marks[page / 8], 8u << at);
        }
    }
    __syncthreads();
    // the rows
    const int n = child ? s_n[parent] : 0;
    int page = -1;
    if (n & (d.page_size - 1)) page = d.block_table[parent * d.table_stride + (n >> a.shift)];
    const bool need = is_page(a, page) && (s_first[parent] != tid || !stays(marks_of(page)));
    const Sums rows = scan<kRowThreads>((int)need | (int)child << 16, s), wanted{rows.before & 0xffff, rows.all & 0xffff};
    const long from = (long)begin + wanted.before;
    const int dst = need && from >= 0 && from < d.n_free ? d.free_pages[from] : -1;
    // the pages, a run of words to a thread
    const int each = (words + kRowThreads - 1) / kRowThreads, w0 = min(tid * each, words), w1 = min(w0 + each, words);
    auto freed = [&](int p) { return p < d.num_pages && s_marks[p / 8] >> p % 8 * 4 & kOld && goes(marks_of(p)); };
    int mine = 0;
    for (int p = w0 * 8; p < w1 * 8; ++p) mine += freed(p);
    const Sums gone = scan<kRowThreads>(mine, s);
    const int flags = all_flags(a, bad ? NM_FORK_BAD_LENGTH : 0, begin, wanted.all, gone.all);
    const bool ok = flags == 0;
    const int end = ok ? begin + wanted.all - gone.all : begin;
    if (tid == 0) report(a, flags, wanted.all, gone.all, rows.all >> 16, end);
    if (tid < d.B_out) {
        d.lens_out[tid] = ok ? n : 0;
        d.copy_src[tid] = ok && need ? page : -1;
        d.copy_dst[tid] = ok ? dst : -1;
        d.copy_slots[tid] = ok && need ? n & (d.page_size - 1) : 0;
    }
    s_src[tid] = need ? n >> a.shift : -1;         // the entry that is another
    s_dst[tid] = dst;
    __syncthreads();                               // also: what is taken has been read, where the list is written in place
    if (ok) {
        int to = end + gone.before;
        for (int p = w0 * 8; mine && p < w1 * 8; ++p)
            if (freed(p)) d.free_out[to++] = p;
        for (int b = wave; b < d.B_out; b += kRowThreads / 64) {
            const int p = d.parents[b];
            if (!is_row(a, p)) continue;
            const int held = held_of(a, s_n[p]);
            for (int i = lane; i < held; i += 64) d.table_out[b * d.table_out_stride + i] = i == s_src[b] ? s_dst[b] : d.block_table[p * d.table_stride + i];
        }
    }
    if (d.free_out != d.free_pages && begin >= 0)
        for (long i = (long)begin + (ok ? wanted.all : 0) + tid; i < d.n_free; i += kRowThreads) d.free_out[i] = d.free_pages[i];
}

static int32_t plan_fork(const nm_fork_desc* d, ForkArgs* a, size_t* bytes, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    if (d->B_in < 0 || d->B_out < 0 || d->num_pages < 0 || d->max_pages < 0 || d->n_free < 0) return fail(NM_ERR_INVALID_ARG, "%s: negative size", what);
    if (d->B_in > NM_PLAN_MAX_REQUESTS || d->B_out > NM_PLAN_MAX_REQUESTS) return fail(NM_ERR_UNSUPPORTED, "%s: B_in %d or B_out %d > %d", what, d->B_in, d->B_out, NM_PLAN_MAX_REQUESTS);
    if (d->n_free > 1 << 30) return fail(NM_ERR_UNSUPPORTED, "%s: n_free > 2^30", what);
    const int shift = page_shift(d->page_size);
    if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "%s: page_size %d is no power of two up to 65536", what, d->page_size);
    if (d->num_pages > 1 << 30 || d->max_pages > 1 << 30) return fail(NM_ERR_UNSUPPORTED, "%s: num_pages or max_pages > 2^30", what);
    if ((int64_t)d->num_pages << shift > 0x7fffffffLL || (int64_t)d->max_pages << shift > 0x7fffffffLL)
        return fail(NM_ERR_UNSUPPORTED, "%s: num_pages * page_size or max_pages * page_size >= 2^31", what);
    *a = ForkArgs{};
    a->d = *d;
    a->shift = shift;
    a->padded = ((long)d->num_pages + kRun - 1) / kRun * kRun;
    a->block = std::max(kForkBlock, ((d->num_pages + kForkBlocks - 1) / kForkBlocks + kRun - 1) / kRun * kRun);
    a->blocks = (d->num_pages + a->block - 1) / a->block;
    a->list_blocks = std::min((d->n_free + 8 * kForkThreads - 1) / (8 * kForkThreads), 512);
    *bytes = 6 * (size_t)a->padded + sizeof(int) * (5 * (size_t)d->B_out + d->B_in + a->blocks + kRowBlocks + 1);
    return NM_OK;
}

}  // namespace nm

using namespace nm;

extern "C" {

int32_t nm_page_fork_workspace(const nm_fork_desc* d, size_t* bytes)
{
    ForkArgs a;
    size_t n;
    const int32_t rc = plan_fork(d, &a, &n, "nm_page_fork_workspace");
    if (rc) return rc;
    if (!bytes) return fail(NM_ERR_INVALID_ARG, "nm_page_fork_workspace: bytes is NULL");
    *bytes = n;
    return NM_OK;
}

int32_t nm_page_fork(const nm_fork_desc* d, void* ws, size_t ws_bytes, void* stream)
{
    ForkArgs a;
    size_t need;
    const int32_t rc = plan_fork(d, &a, &need, "nm_page_fork");
    if (rc) return rc;
    if ((d->B_in && d->table_stride < d->max_pages) || (d->B_out && d->table_out_stride < d->max_pages))
        return fail(NM_ERR_INVALID_ARG, "nm_page_fork: a table's stride is shorter than max_pages");
    if (!d->free_begin || !d->free_end || !d->status) return fail(NM_ERR_INVALID_ARG, "nm_page_fork: free_begin, free_end or status is NULL");
    if (d->B_in && (!d->lens || (d->max_pages && !d->block_table))) return fail(NM_ERR_INVALID_ARG, "nm_page_fork: lens or block_table is NULL");
    if (d->B_out && (!d->parents || !d->lens_out || !d->copy_src || !d->copy_dst || !d->copy_slots || (d->max_pages && !d->table_out)))
        return fail(NM_ERR_INVALID_ARG, "nm_page_fork: parents, table_out, lens_out or one of the copies is NULL");
    if (d->n_free && (!d->free_pages || !d->free_out)) return fail(NM_ERR_INVALID_ARG, "nm_page_fork: free_pages or free_out is NULL");
    const int32_t* in[] = {d->block_table, d->lens, d->parents, d->keep, d->free_begin, d->free_pages};
    const int32_t* out[] = {d->table_out, d->lens_out, d->free_end, d->copy_src, d->copy_dst, d->copy_slots, d->status, d->free_out};
    for (const int32_t*& q : out) {
        for (const int32_t*& p : in)
            if (p && p == q && !(p == d->free_pages && &q == &out[7])) return fail(NM_ERR_INVALID_ARG, "nm_page_fork: an output is an input");
        for (const int32_t*& p : out)
            if (&p != &q && p && p == q) return fail(NM_ERR_INVALID_ARG, "nm_page_fork: two outputs are one");
    }
    if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_page_fork: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_page_fork: workspace must be 256-byte aligned");
    a.marks = static_cast<int*>(ws);
    a.old = reinterpret_cast<uint8_t*>(a.marks + a.padded);
    a.rows = reinterpret_cast<int4*>(a.old + 2 * a.padded);
    a.taken = reinterpret_cast<int*>(a.rows + d->B_out);
    a.first = a.taken + d->B_out;
    a.freed = a.first + d->B_in;
    a.sums = a.freed + a.blocks;
    a.bad = a.sums + kRowBlocks;
    const hipStream_t s = (hipStream_t)stream;
    const dim3 threads(kForkThreads);
    if (std::max(d->B_in, d->B_out) <= kSmallRows && (long)std::max(d->B_in, d->B_out) * d->max_pages <= kSmallEntries && d->num_pages <= kSmallPages && d->n_free <= kSmallList) {
        queue_kernel(fork_small_kernel, dim3(1), dim3(kRowThreads), sizeof(unsigned) * ((d->num_pages + 7) / 8), s, a);
        return check_hip(hipGetLastError(), "nm_page_fork launch");
    }
    const int per = kForkThreads / 64, news = (d->B_out + kForkThreads - 1) / kForkThreads, olds = (d->B_in + per - 1) / per;
    queue_kernel(fork_clear_kernel, dim3(1 + std::min((d->num_pages + kRowThreads - 1) / kRowThreads, 1024)), dim3(kRowThreads), 0, s, a);
    if (news + olds) queue_kernel(fork_mark_kernel, dim3(news + olds), threads, 0, s, a);
    queue_kernel(fork_decide_kernel, dim3(a.blocks + news + 1), threads, 0, s, a);
    queue_kernel(fork_write_kernel, dim3(std::max(1, a.blocks + (d->B_out + per - 1) / per + a.list_blocks)), threads, 0, s, a);
    return check_hip(hipGetLastError(), "nm_page_fork launch");
}

}  // extern "C"
