// Block tables, slots and positions of a decode step from the requests' lengths (nm_page_plan).
//
// What is needed of all requests is two prefix sums, over the new tokens and over the new pages.  Every workgroup makes both for itself
// (two numbers of each request, from L2) and keeps them in LDS, so that no workgroup waits for another and one launch does;
// then each token, and each new page, finds its request by bisection.  Bound by latency: a launch, and dependent steps (lengths, the
// scan, a bisection, an entry of the table or the list, a store): 4.1 us for 8 requests of one token, where a kernel that fills one
// line takes 1.8.  500000 tokens of 500 requests, 6 MB of stores, take 8.3 us (1.2 at the rate of a copy): as long a chain, with a scan of
// two requests a thread and a bisection of nine steps.
#include "nm_decode.h"

namespace nm {

constexpr int kPlanThreads = 256;

// The last i in [0, n) with start[i] <= x (start ascends, start[0] = 0 <= x < start[n]): the request that owns x, for those of no
// tokens (start[i] == start[i + 1]) lie in front of it.
__device__ __forceinline__ int owner(const int* start, int n, int x)
{
    int lo = 0;
    for (int step = n; step > 0; ) {
        const int half = step >> 1, mid = lo + half;   // the answer is in [lo, lo + step)
        const bool right = start[mid] <= x;
        lo = right ? mid : lo;
        step = half == 0 ? 0 : right ? step - half : half;
    }
    return lo;
}

__device__ __forceinline__ int saturated(long x) { return (int)(x < 0x7fffffffL ? x : 0x7fffffffL); }

// V: neighbouring tokens of a thread, 1 or 4.
template <int V>
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(nm_plan_desc d, int shift, int tokens_per_block, int whole)
{
    extern __shared__ int s_start[];          // [B + 1] tokens in front of a request, [B + 1] pages
    int* s_tok = s_start;
    int* s_page = s_start + d.B + 1;
    __shared__ long s_wave_tok[kPlanThreads / 64], s_wave_page[kPlanThreads / 64];
    __shared__ int s_wave_max[kPlanThreads / 64], s_wave_bad[kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int begin = *d.free_begin;
    const long round = (1L << shift) - 1;

    // a thread's own run of requests, then the threads'
    const int per = (d.B + kPlanThreads - 1) / kPlanThreads, b0 = min(tid * per, d.B), b1 = min(b0 + per, d.B);
    long tok = 0, page = 0, most = 0;
    int bad = begin < 0 ? NM_PLAN_BAD_LENGTH : 0;
    for (int b = b0; b < b1; ++b) {
        const int c = d.cached[b], f = d.fresh[b];
        const long after = (long)c + f, want = (after + round) >> shift;
        if (c < 0 || f < 0) bad |= NM_PLAN_BAD_LENGTH;
        if (want > d.max_pages) bad |= NM_PLAN_TABLE_FULL;
        s_tok[b] = (int)tok;                  // within the thread's run; meaningless where a sum passes 2^31, and not used then
        s_page[b] = (int)page;
        tok += max(f, 0);
        page += f > 0 && c >= 0 ? want - (((long)c + round) >> shift) : 0;
        most = after > most ? after : most;
    }
    long tok_in = tok, page_in = page;        // inclusive sums over the wavefront
    for (int step = 1; step < 64; step <<= 1) {
        const long t = __shfl_up(tok_in, step), p = __shfl_up(page_in, step);
        if (lane >= step) { tok_in += t; page_in += p; }
    }
    for (int step = 32; step > 0; step >>= 1) {
        const long m = __shfl_xor(most, step);
        most = m > most ? m : most;
        bad |= __shfl_xor(bad, step);
    }
    if (lane == 63) { s_wave_tok[wave] = tok_in; s_wave_page[wave] = page_in; s_wave_max[wave] = saturated(most); s_wave_bad[wave] = bad; }
    __syncthreads();
    long tok_before = tok_in - tok, page_before = page_in - page, tokens = 0, pages = 0;
    int longest = 0;
    bad = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) { tok_before += s_wave_tok[w]; page_before += s_wave_page[w]; }
        tokens += s_wave_tok[w];
        pages += s_wave_page[w];
        longest = max(longest, s_wave_max[w]);
        bad |= s_wave_bad[w];
    }
    if (tokens > d.max_tokens) bad |= NM_PLAN_NO_ROWS;
    if (pages > 0 ? begin + pages > d.n_free : begin > d.n_free) bad |= NM_PLAN_NO_PAGES;
    for (int b = b0; b < b1; ++b) {
        s_tok[b] += (int)tok_before;
        s_page[b] += (int)page_before;
    }
    if (tid == 0) { s_tok[d.B] = saturated(tokens); s_page[d.B] = saturated(pages); }
    __syncthreads();
    const bool ok = bad == 0;

    const int block = blockIdx.x, threads = gridDim.x * kPlanThreads, gid = block * kPlanThreads + tid;
    if (gid == 0) {
        d.status[0] = bad;
        d.status[1] = saturated(tokens);
        d.status[2] = saturated(pages);
        d.status[3] = longest;
        *d.free_end = ok ? begin + (int)pages : begin;
        if (d.row_start) d.row_start[d.B] = ok ? (int)tokens : 0;
    }
    for (int b = gid; b < d.B; b += threads) {
        if (d.lens) d.lens[b] = ok ? d.cached[b] + d.fresh[b] : d.cached[b];
        if (d.row_start) d.row_start[b] = ok ? s_tok[b] : 0;
    }
    if (ok)
        for (int k = gid; k < (int)pages; k += threads) {
            const int b = owner(s_page, d.B, k);
            const int column = (int)(((long)d.cached[b] + round) >> shift) + k - s_page[b];
            d.block_table[b * d.table_stride + column] = d.free_pages[begin + k];
        }
    // Of a thread's tokens the first is looked up, another only where the request ends among them; one entry of the table does as long
    // as the page is the same.
    const int t0 = (int)min((long)block * tokens_per_block, (long)d.max_tokens), t1 = (int)min((long)t0 + tokens_per_block, (long)d.max_tokens);
    for (int t = t0 + tid * V; t < t1; t += kPlanThreads * V) {
        int slot[V], position[V], request[V];
        int r = -1, at = -1, entry = -1, c = 0, first = 0, end = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            slot[i] = request[i] = -1;
            position[i] = 0;
            if (!ok || t + i >= (int)tokens) continue;
            if (t + i >= end) {
                r = owner(s_tok, d.B, t + i);
                first = s_tok[r];
                end = s_tok[r + 1];
                c = d.cached[r];
                at = -1;
            }
            const int p = c + t + i - first;
            if (p >> shift != at) {
                at = p >> shift;
                const int held = (int)(((long)c + round) >> shift);
                entry = at < held ? d.block_table[r * d.table_stride + at] : d.free_pages[begin + s_page[r] + at - held];
            }
            request[i] = r;
            position[i] = p;
            if (entry >= 0 && entry < d.num_pages) slot[i] = (entry << shift) + (p & (int)round);
        }
        if (V == 4 && whole && t + V <= t1) {
            *reinterpret_cast<int4*>(d.slots + t) = make_int4(slot[0], slot[V / 4], slot[V / 2], slot[V - 1]);
            if (d.positions) *reinterpret_cast<int4*>(d.positions + t) = make_int4(position[0], position[V / 4], position[V / 2], position[V - 1]);
            if (d.requests) *reinterpret_cast<int4*>(d.requests + t) = make_int4(request[0], request[V / 4], request[V / 2], request[V - 1]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (t + i < t1) {
                    d.slots[t + i] = slot[i];
                    if (d.positions) d.positions[t + i] = position[i];
                    if (d.requests) d.requests[t + i] = request[i];
                }
        }
    }
}

}  // namespace nm

using namespace nm;

extern "C" int32_t nm_page_plan(const nm_plan_desc* d, void* stream)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "nm_page_plan: desc is NULL");
    if (d->B < 0 || d->num_pages < 0 || d->max_pages < 0 || d->n_free < 0 || d->max_tokens < 0)
        return fail(NM_ERR_INVALID_ARG, "nm_page_plan: negative size");
    if (d->B > NM_PLAN_MAX_REQUESTS) return fail(NM_ERR_UNSUPPORTED, "nm_page_plan: B %d > %d", d->B, NM_PLAN_MAX_REQUESTS);
    if (d->max_tokens > 1 << 30 || d->n_free > 1 << 30) return fail(NM_ERR_UNSUPPORTED, "nm_page_plan: max_tokens or n_free > 2^30");
    const int shift = page_shift(d->page_size);
    if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "nm_page_plan: page_size %d is no power of two up to 65536", d->page_size);
    if ((int64_t)d->num_pages << shift > 0x7fffffffLL) return fail(NM_ERR_UNSUPPORTED, "nm_page_plan: num_pages * page_size >= 2^31");
    if ((int64_t)d->max_pages << shift > 0x7fffffffLL) return fail(NM_ERR_UNSUPPORTED, "nm_page_plan: max_pages * page_size >= 2^31");   // a position is an int
    if (d->B && d->table_stride < d->max_pages) return fail(NM_ERR_INVALID_ARG, "nm_page_plan: table_stride < max_pages");
    if (!d->free_begin || !d->free_end || !d->status || (d->max_tokens && !d->slots))
        return fail(NM_ERR_INVALID_ARG, "nm_page_plan: free_begin, free_end, status or slots is NULL");
    if (d->B && (!d->cached || !d->fresh || (d->max_pages && !d->block_table)))
        return fail(NM_ERR_INVALID_ARG, "nm_page_plan: cached, fresh or block_table is NULL");
    if (d->n_free && !d->free_pages) return fail(NM_ERR_INVALID_ARG, "nm_page_plan: free_pages is NULL");
    const int32_t* in[] = {d->cached, d->fresh, d->free_pages, d->free_begin};
    const int32_t* out[] = {d->free_end, d->block_table, d->lens, d->row_start, d->slots, d->positions, d->requests, d->status};
    for (const int32_t* p : in)
        for (const int32_t* q : out)
            if (p && p == q) return fail(NM_ERR_INVALID_ARG, "nm_page_plan: an output is an input");
    // A workgroup's scan costs it a few microseconds whatever it then writes.  Few tokens: 256 to a workgroup, one to a thread (8 tokens of 8
    // requests 4.1 us so, 5.9 by four to a thread).  Many: 1024 and more, four to a thread (500000 tokens of 500 requests 8.3 us so, 9.5 by one).
    const bool few = d->max_tokens <= 65536;
    const int per = few ? 256 : d->max_tokens <= 512 * 1024 ? 1024 : ((d->max_tokens + 511) / 512 + 3) / 4 * 4;
    const int blocks = d->max_tokens ? (d->max_tokens + per - 1) / per : 1;
    const int whole = aligned(d->slots, 16) && aligned(d->positions, 16) && aligned(d->requests, 16);
    queue_kernel(few ? page_plan_kernel<1> : page_plan_kernel<4>, dim3(blocks), dim3(kPlanThreads), sizeof(int) * 2 * ((size_t)d->B + 1), (hipStream_t)stream, *d,
                 shift, per, whole);
    return check_hip(hipGetLastError(), "nm_page_plan launch");
}
