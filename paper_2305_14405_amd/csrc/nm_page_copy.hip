// Copies of pages inside the caches of a model (nm_page_copy).
//
// Bound by memory: every element that is moved is read and written once.  A copy's part of one cache is cut into pieces of up to 1024 groups of 16 bytes, a
// workgroup to each; a thread has up to four groups under way.  Groups are numbered as they lie in memory, so that neighbouring lanes move
// neighbouring bytes: by slots and then heads, or by heads and then slots, whichever is further apart.  A row of a
// head that is not whole groups is moved by pieces of 8, 4, 2 or 1 bytes.
//   154 pages of 32 slots, 8 heads of 128 bf16, through 64 caches: whole 257 us, 5.0 TB/s, the rate of a large copy; their first 16 slots 146 us, 4.4 TB/s,
// by heads or by tokens, for the first halves of pages are not spread evenly over the memory's channels.  (Four caches to a workgroup, with four times the
// loads under way: the same.)  16 rows through 24 caches of 12 heads of 64: 4.6 us, a launch and two dependent loads.
#include <algorithm>

#include "nm_decode.h"

namespace nm {

constexpr int kCopyThreads = 256, kCopyEach = 4;

struct CopyArgs {
    void* cache[NM_COPY_MAX_CACHES];
    const int32_t* src;
    const int32_t* dst;
    const int32_t* slots;
    int n, hk, num_pages, page_size, pieces;
    int slots_inside;                                // slots of a head are nearer than heads of a slot
    FastDiv unit_row;                                // units of a head's row
    long page_stride, slot_stride, head_stride;      // in units
};

template <typename U>
__global__ __launch_bounds__(kCopyThreads) void page_copy_kernel(CopyArgs a)
{
    const int i = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
    const int src = a.src[i], dst = a.dst[i], slots = a.slots ? min(a.slots[i], a.page_size) : a.page_size;
    if (src == dst || src < 0 || dst < 0 || src >= a.num_pages || dst >= a.num_pages || slots < 1) return;
    const unsigned inside = a.slots_inside ? slots : a.hk, all = (unsigned)slots * a.hk * a.unit_row.d;
    const unsigned first = piece * (kCopyThreads * kCopyEach) + threadIdx.x;
    if (first >= all) return;
    const long near = a.slots_inside ? a.slot_stride : a.head_stride, far = a.slots_inside ? a.head_stride : a.slot_stride;
    const long from = src * a.page_stride, to = dst * a.page_stride;
    long at[kCopyEach];
#pragma unroll
    for (int e = 0; e < kCopyEach; ++e) {
        const unsigned u = min(first + e * kCopyThreads, all - 1), row = quotient(u, a.unit_row);
        at[e] = row / inside * far + row % inside * near + (u - row * a.unit_row.d);
    }
    U* cache = static_cast<U*>(a.cache[blockIdx.y]);
    U x[kCopyEach];
#pragma unroll
    for (int e = 0; e < kCopyEach; ++e) x[e] = cache[from + at[e]];
#pragma unroll
    for (int e = 0; e < kCopyEach; ++e)
        if (first + e * kCopyThreads < all) cache[to + at[e]] = x[e];
}

}  // namespace nm

using namespace nm;

extern "C" int32_t nm_page_copy(const nm_copy_desc* d, void* stream)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: desc is NULL");
    if (d->n < 0 || d->n_caches < 0 || d->hk < 1 || d->d < 1 || d->num_pages < 0) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: bad shape");
    if (!float_dtype(d->dtype) && d->dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: bad dtype");
    if (d->page_stride < 0 || d->slot_stride < 0 || d->head_stride < 0) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: negative stride");
    if (d->n > 1 << 20) return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: n > 2^20");
    if (d->n_caches > NM_COPY_MAX_CACHES) return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: n_caches %d > %d", d->n_caches, NM_COPY_MAX_CACHES);
    const int shift = page_shift(d->page_size);
    if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: page_size %d is no power of two up to 65536", d->page_size);
    const int bytes = dtype_bytes(d->dtype);
    if ((int64_t)d->num_pages << shift > 0x7fffffffLL || ((double)d->hk * d->d) * d->page_size >= 2147483648.0)
        return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: num_pages * page_size or page_size * hk * d >= 2^31");
    if (d->n == 0 || d->n_caches == 0 || d->num_pages == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->caches || !d->src || !d->dst) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: caches, src or dst is NULL");
    CopyArgs a{};
    // the widest unit that every row's address and length is a multiple of
    uintptr_t low = (uintptr_t)(d->d * (int64_t)bytes);
    if (d->num_pages > 1) low |= (uintptr_t)(d->page_stride * bytes);
    if (d->page_size > 1) low |= (uintptr_t)(d->slot_stride * bytes);
    if (d->hk > 1) low |= (uintptr_t)(d->head_stride * bytes);
    for (int i = 0; i < d->n_caches; ++i) {
        a.cache[i] = d->caches[i];
        if (!a.cache[i]) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: cache %d is NULL", i);
        if (begins_as(a.cache[i], {d->src, d->dst, d->slots})) return fail(NM_ERR_INVALID_ARG, "nm_page_copy: cache %d is src, dst or slots", i);
        if (!aligned(a.cache[i], bytes)) return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: cache %d is not aligned to its elements", i);
        low |= reinterpret_cast<uintptr_t>(a.cache[i]);
    }
    const int unit = low % 16 == 0 ? 16 : low % 8 == 0 ? 8 : low % 4 == 0 ? 4 : low % 2 == 0 ? 2 : 1;
    a.src = d->src;
    a.dst = d->dst;
    a.slots = d->slots;
    a.n = d->n;
    a.hk = d->hk;
    a.num_pages = d->num_pages;
    a.page_size = d->page_size;
    a.slots_inside = d->slot_stride < d->head_stride;
    a.unit_row = fast_div((int)(d->d * (int64_t)bytes / unit));
    // strides of dimensions of one are never used, and need not be multiples
    a.page_stride = d->page_stride * bytes / unit;
    a.slot_stride = d->slot_stride * bytes / unit;
    a.head_stride = d->head_stride * bytes / unit;
    const long units = (long)a.unit_row.d * d->hk * d->page_size, piece = kCopyThreads * kCopyEach;
    a.pieces = (int)((units + piece - 1) / piece);
    if ((double)a.pieces * d->n * kCopyThreads >= 4294967296.0) return fail(NM_ERR_UNSUPPORTED, "nm_page_copy: n pages of this size are too many for one call");
    const dim3 grid(a.pieces * d->n, d->n_caches);
    const hipStream_t s = (hipStream_t)stream;
    if (unit == 16) queue_kernel(page_copy_kernel<v4i>, grid, dim3(kCopyThreads), 0, s, a);
    else if (unit == 8) queue_kernel(page_copy_kernel<int2>, grid, dim3(kCopyThreads), 0, s, a);
    else if (unit == 4) queue_kernel(page_copy_kernel<int>, grid, dim3(kCopyThreads), 0, s, a);
    else if (unit == 2) queue_kernel(page_copy_kernel<short>, grid, dim3(kCopyThreads), 0, s, a);
    else queue_kernel(page_copy_kernel<int8_t>, grid, dim3(kCopyThreads), 0, s, a);
    return check_hip(hipGetLastError(), "nm_page_copy launch");
}
