// Block tables of a new batch whose rows go on from rows of the old one (nm_page_fork).
//
// Nothing is counted from call to call: who refers to a page is found from the tables.  A word of the workspace for each page is marked by
// every old row (that a row refers to it), by every row with children (that one refers to it in front of its partial last page), and counts the rows with
// children whose partial last page it is.  From that follow which rows take a page of their own (a scan over the rows) and which pages become free (a
// scan over the pages, in blocks).  Four kernels: clear the words and find every old row's first child; mark; decide for the rows, and count
// the freed pages of every block; write the tables and the list.
//   The marks are set by integer atomics, whose order does not change their result, and a mark that is there already is not set again.
#include <algorithm>

#include "nm_decode.h"

namespace nm {

constexpr int kForkThreads = 256;
constexpr int kForkBlocks = 1024;                  // of pages at most

struct ForkArgs {
    nm_fork_desc d;
    int shift;
    int blocks, block;                             // of pages, and their length
    int list_blocks;
    int* marks;                                    // [num_pages]
    int* first;                                    // [B_in]: lowest-numbered child, B_out: none
    int* freed;                                    // [blocks]: pages that become free
    int* sums;                                     // [4]: flags of the rows, pages wanted, rows with a parent
};
enum { kOld = 1, kFull = 2, kPart = 4 };           // kPart and above: how many rows with children have it as their partial last page

// Tokens of an old row, 0 where its length is bad.
__device__ __forceinline__ int length_of(const ForkArgs& a, int r, bool* bad = nullptr)
{
    const int n = a.d.lens[r];
    const bool off = n < 0 || n > (long)a.d.max_pages << a.shift;
    if (bad) *bad = off;
    return off ? 0 : n;
}
__device__ __forceinline__ bool is_page(const ForkArgs& a, int e) { return e >= 0 && e < a.d.num_pages; }
__device__ __forceinline__ bool is_row(const ForkArgs& a, int p) { return p >= 0 && p < a.d.B_in; }

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
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) r.before += s[w];
        r.all += s[w];
    }
    return r;
}

__global__ __launch_bounds__(kForkThreads) void fork_clear_kernel(ForkArgs a)
{
    __shared__ int s_first[NM_PLAN_MAX_REQUESTS];
    if (blockIdx.x) {
        for (long i = (long)(blockIdx.x - 1) * kForkThreads + threadIdx.x; i < a.d.num_pages; i += (long)(gridDim.x - 1) * kForkThreads) a.marks[i] = 0;
        return;
    }
    for (int r = threadIdx.x; r < a.d.B_in; r += kForkThreads) s_first[r] = a.d.B_out;
    __syncthreads();
    for (int b = threadIdx.x; b < a.d.B_out; b += kForkThreads) {
        const int p = a.d.parents[b];
        if (is_row(a, p)) atomicMin(&s_first[p], b);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < a.d.B_in; r += kForkThreads) a.first[r] = s_first[r];
}

// A workgroup to an old row.
__global__ __launch_bounds__(kForkThreads) void fork_mark_kernel(ForkArgs a)
{
    const int r = blockIdx.x, n = length_of(a, r), whole = n >> a.shift, held = whole + (n & (a.d.page_size - 1) ? 1 : 0);
    const bool lives = a.first[r] < a.d.B_out;
    for (int i = threadIdx.x; i < held; i += kForkThreads) {
        const int page = a.d.block_table[r * a.d.table_stride + i];
        if (!is_page(a, page)) continue;
        const int mark = kOld | (lives && i < whole ? kFull : 0);
        if ((__hip_atomic_load(a.marks + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & mark) != mark) atomicOr(a.marks + page, mark);
        if (lives && i >= whole) atomicAdd(a.marks + page, kPart);
    }
}

__device__ __forceinline__ bool becomes_free(const ForkArgs& a, int page)
{
    const int m = a.marks[page];
    return (m & (kOld | kFull)) == kOld && m / kPart != 1 && !(a.d.keep && a.d.keep[page]);
}

// Workgroup 0: the rows.  The others: a block of pages each.
__global__ __launch_bounds__(kForkThreads) void fork_decide_kernel(ForkArgs a)
{
    __shared__ int s[kForkThreads / 64];
    const nm_fork_desc& d = a.d;
    if (blockIdx.x) {
        const int block = blockIdx.x - 1;
        const long p0 = (long)block * a.block, p1 = min(p0 + a.block, (long)d.num_pages);
        int n = 0;
        for (long p = p0 + threadIdx.x; p < p1; p += kForkThreads) n += becomes_free(a, (int)p);
        const Sums all = scan<kForkThreads>(n, s);
        if (threadIdx.x == 0) a.freed[block] = all.all;
        return;
    }
    const int begin = *d.free_begin;
    bool bad = begin < 0 || begin > d.n_free;
    for (int r = threadIdx.x; r < d.B_in; r += kForkThreads) {
        bool off;
        length_of(a, r, &off);
        bad |= off;
    }
    // a thread has a run of rows
    const int per = (d.B_out + kForkThreads - 1) / kForkThreads, b0 = min((int)threadIdx.x * per, d.B_out), b1 = min(b0 + per, d.B_out);
    int wants = 0, rows = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int at = 0;
        if (pass) {
            const Sums pages = scan<kForkThreads>(wants, s), parents = scan<kForkThreads>(rows, s);
            const bool any = __syncthreads_or(bad);
            at = pages.before;
            if (threadIdx.x == 0) {
                a.sums[0] = any ? NM_FORK_BAD_LENGTH : 0;
                a.sums[1] = pages.all;
                a.sums[2] = parents.all;
            }
        }
        for (int b = b0; b < b1; ++b) {
            const int p = d.parents[b];
            int src = -1, dst = -1, slots = 0;
            if (is_row(a, p)) {
                const int n = length_of(a, p);
                if (!pass) ++rows;
                if (n & (d.page_size - 1)) {
                    const int page = d.block_table[p * d.table_stride + (n >> a.shift)];
                    if (is_page(a, page)) {
                        const int m = a.marks[page];
                        if (a.first[p] != b || (m & kFull) || m / kPart != 1 || (d.keep && d.keep[page])) {
                            if (!pass) ++wants;
                            src = page;
                            slots = n & (d.page_size - 1);
                            const long i = (long)begin + at++;
                            if (i >= 0 && i < d.n_free) dst = d.free_pages[i];
                        }
                    }
                }
            }
            if (pass) {
                d.copy_src[b] = src;
                d.copy_dst[b] = dst;
                d.copy_slots[b] = slots;
            }
        }
    }
}

// Workgroups: rows, then blocks of pages, then blocks of the list.
__global__ __launch_bounds__(kForkThreads) void fork_write_kernel(ForkArgs a)
{
    __shared__ int s[kForkThreads / 64];
    const nm_fork_desc& d = a.d;
    const int block = (int)blockIdx.x - d.B_out, tid = threadIdx.x;
    int before = 0, all = 0;                       // freed pages of the blocks in front of this one, and of all
    for (int i = tid; i < a.blocks; i += kForkThreads) {
        const int n = a.freed[i];
        all += n;
        before += i < block ? n : 0;
    }
    all = scan<kForkThreads>(all, s).all;
    const int begin = *d.free_begin, wanted = a.sums[1];
    int flags = a.sums[0];
    if (begin >= 0 && begin <= d.n_free) {
        if ((long)begin + wanted > d.n_free) flags |= NM_FORK_NO_PAGES;
        if ((long)begin + wanted - all < 0) flags |= NM_FORK_LIST_FULL;
    }
    const bool ok = flags == 0;
    const int end = ok ? begin + wanted - all : begin;

    if (blockIdx.x == 0 && tid == 0) {
        d.status[0] = flags;
        d.status[1] = wanted;
        d.status[2] = all;
        d.status[3] = a.sums[2];
        *d.free_end = end;
    }
    if (block < 0) {
        const int b = blockIdx.x, p = d.parents[b];
        const bool lives = ok && is_row(a, p);
        const int n = lives ? length_of(a, p) : 0, held = (int)(((long)n + d.page_size - 1) >> a.shift);
        const int dst = lives ? d.copy_dst[b] : -1, src = lives ? d.copy_src[b] : -1;
        __syncthreads();
        for (int i = tid; i < held; i += kForkThreads)
            d.table_out[b * d.table_out_stride + i] = src >= 0 && i == n >> a.shift ? dst : d.block_table[p * d.table_stride + i];
        if (tid == 0) {
            d.lens_out[b] = n;
            if (!ok) {
                d.copy_src[b] = d.copy_dst[b] = -1;
                d.copy_slots[b] = 0;
            }
        }
    } else if (block < a.blocks) {
        if (!ok) return;
        long at = (long)end + scan<kForkThreads>(before, s).all;
        const long p0 = (long)block * a.block, p1 = min(p0 + a.block, (long)d.num_pages);
        for (long p = p0; p < p1; p += kForkThreads) {
            const bool goes = p + tid < p1 && becomes_free(a, (int)(p + tid));
            const Sums sums = scan<kForkThreads>(goes, s);
            if (goes) d.free_out[at + sums.before] = (int)(p + tid);
            at += sums.all;
        }
    } else if (d.free_out != d.free_pages && begin >= 0) {
        for (long i = (long)begin + (ok ? wanted : 0) + (long)(block - a.blocks) * kForkThreads + tid; i < d.n_free; i += (long)a.list_blocks * kForkThreads)
            d.free_out[i] = d.free_pages[i];
    }
}

static int32_t plan_fork(const nm_fork_desc* d, ForkArgs* a, size_t* bytes, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    if (d->B_in < 0 || d->B_out < 0 || d->num_pages < 0 || d->max_pages < 0 || d->n_free < 0) return fail(NM_ERR_INVALID_ARG, "%s: negative size", what);
    if (d->B_in > NM_PLAN_MAX_REQUESTS || d->B_out > NM_PLAN_MAX_REQUESTS) return fail(NM_ERR_UNSUPPORTED, "%s: B_in %d or B_out %d > %d", what, d->B_in, d->B_out, NM_PLAN_MAX_REQUESTS);
    if (d->n_free > 1 << 30) return fail(NM_ERR_UNSUPPORTED, "%s: n_free > 2^30", what);
    const int shift = page_shift(d->page_size);
    if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "%s: page_size %d is no power of two up to 65536", what, d->page_size);
    if ((int64_t)d->num_pages << shift > 0x7fffffffLL || (int64_t)d->max_pages << shift > 0x7fffffffLL)
        return fail(NM_ERR_UNSUPPORTED, "%s: num_pages * page_size or max_pages * page_size >= 2^31", what);
    *a = ForkArgs{};
    a->d = *d;
    a->shift = shift;
    a->block = std::max(4096, (d->num_pages + kForkBlocks - 1) / kForkBlocks);
    a->blocks = (d->num_pages + a->block - 1) / a->block;
    a->list_blocks = std::min((d->n_free + 8 * kForkThreads - 1) / (8 * kForkThreads), 512);
    *bytes = sizeof(int) * ((size_t)d->num_pages + d->B_in + a->blocks + 4);
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
    a.first = a.marks + d->num_pages;
    a.freed = a.first + d->B_in;
    a.sums = a.freed + a.blocks;
    const hipStream_t s = (hipStream_t)stream;
    const dim3 threads(kForkThreads);
    queue_kernel(fork_clear_kernel, dim3(1 + std::min((d->num_pages + 4 * kForkThreads - 1) / (4 * kForkThreads), 2048)), threads, 0, s, a);
    if (d->B_in) queue_kernel(fork_mark_kernel, dim3(d->B_in), threads, 0, s, a);
    queue_kernel(fork_decide_kernel, dim3(1 + a.blocks), threads, 0, s, a);
    queue_kernel(fork_write_kernel, dim3(std::max(1, d->B_out + a.blocks + a.list_blocks)), threads, 0, s, a);
    return check_hip(hipGetLastError(), "nm_page_fork launch");
}

}  // extern "C"
