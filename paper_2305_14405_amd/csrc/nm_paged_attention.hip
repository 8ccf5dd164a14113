// Attention of one new token per request over a paged cache (nm_paged_attention).
//
// Bound by memory: every key and value is read once, with 2 * (query heads of its group) operations an element.  A row of work is one
// request's key head with up to 16 query heads of its group; its length is counted in units of 128 positions.  A fixed number of
// workgroups share all rows' units evenly, each a contiguous run of them, whatever the lengths are: a run may begin and end inside a
// row, and only those two pieces of it need joining by a second kernel; rows inside a run are written at once.  (Where no row can be long,
// a workgroup takes a row, of eight wavefronts if rows are few, and there is no second kernel.)  The four wavefronts of a workgroup walk a unit's four tiles of 32
// positions, each with a running maximum, sum and output of its own, and are joined through LDS at the end of the row's piece.
// The next tile's keys and values are on their way into registers while one is computed.
//   Scores: keys are the rows of the 16x16x32 matrix instruction, query heads its columns, so a lane has eight positions of one head:
// its maximum and sum are in-lane steps and two across lanes.  Those registers are already the second product's operand: the contraction
// index of a matrix instruction may be permuted, so "row 4 j + i of the first, then of the second 16 keys" is what lane group j contributes, and
// the values are fetched from LDS in that order by the transposing read.  Output: columns are heads again, so the rescaling factor
// is in the lane that needs it.
//   Precision: scores and sums fp32; exp(s - m) goes into the second product as two terms of 16 bits (2^-17 of itself, below what a 16-bit result
// shows; three terms where the result is fp32), queries that are no 16-bit numbers of the matrix instructions' type as three terms of it, scaled by a
// power of two so that nothing overflows.  int8 codes are exact in either 16-bit type.
//   bf16, 32 query and 8 key heads of 128: one request of 131071 positions (537 MB) 105 us and 8 for the second kernel, 5.1 TB/s in the first, a
// copy's rate; 48 requests of up to 8192 (649 MB) 120 + 5, 5.4 TB/s.  int8, 16 heads of 64, two taken as one, 64 requests of up to 4097 (216 MB): 53 + 5,
// 4.1 TB/s: a run has 13 units or so, and begins and ends two rows in them; codes become 16-bit numbers in vector instructions.  12 heads of 300 positions of one request: 9.4 us (one position 7.6), a chain of dependent loads (length, page, keys) and code that runs once.
#include "nm_paged_parts.h"

namespace nm {

struct PagedDesc { nm_paged_desc d; };
struct PagedArgs : PagedDesc, PagedSplit {
    int shift;            // log2 of page_size
    int extra;            // units that starting and ending a row costs
    float* part_o;        // [share, workers, 2, 16, d]: a run's first and last piece, not yet divided by the sum
    float2* part_ml;      // [share, workers, 2, 16]: maximum (of scores in units of log 2) and sum
    int4* joined;         // [share, workers]: the row that begins in a run and ends in another: request, first query head, the run's slot for
                          // it, and how many runs have some of it (0: there is no such row)
};

// Number of a piece's first query head in part_o and part_ml.
__device__ __forceinline__ long part_of(const PagedArgs& a, int member, long worker, int slot) { return (((long)member * a.workers + worker) * 2 + slot) * 16; }

// The positions of request b that take part are [low, n).
struct Span { int low, n; };
__device__ __forceinline__ Span span_of(const PagedArgs& a, int b)
{
    const int n = (int)min((long)max(a.d.lens[b], 0), (long)a.d.max_pages << a.shift);
    return Span{a.d.window ? max(n - a.d.window, 0) : 0, n};
}
__device__ __forceinline__ int units_of(const PagedArgs& a, int b)
{
    const Span s = span_of(a, b);
    return (s.n - s.low + kUnit - 1) / kUnit;
}

// What one of a request's rows counts for when the work is shared: starting and ending a row costs a workgroup about as much as a.extra units.
__device__ __forceinline__ int cost_of(const PagedArgs& a, int b) { return units_of(a, b) + a.extra; }

// The cost of one of a request's rows, summed over the requests in front of each thread's run of them, and over all.  s: LDS of one number a wavefront.
struct Scan { long before, mine, all; int b0, b1; };
__device__ __forceinline__ Scan scan_units(const PagedArgs& a, long* s)
{
    const int per = (a.d.B + kPagedThreads - 1) / kPagedThreads, tid = threadIdx.x;
    Scan r;
    r.b0 = min(tid * per, a.d.B);
    r.b1 = min(r.b0 + per, a.d.B);
    r.mine = 0;
    for (int b = r.b0; b < r.b1; ++b) r.mine += cost_of(a, b);
    long in = r.mine;
    for (int step = 1; step < 64; step <<= 1) {
        const long t = __shfl_up(in, step);
        if ((tid & 63) >= step) in += t;
    }
    if ((tid & 63) == 63) s[tid >> 6] = in;
    __syncthreads();
    r.before = in - r.mine;
    r.all = 0;
    for (int w = 0; w < kPagedWaves; ++w) {
        if (w < tid >> 6) r.before += s[w];
        r.all += s[w];
    }
    return r;
}

// What a workgroup has of a row: positions [k0, k1) of request b for key head g and query heads h0 .. h0 + heads - 1; slot: where its part goes,
// -1 where it is the whole row.  b: -1 for none.
struct Piece { int b, g, h0, heads, k0, k1, slot; };

// C: type of the cache; T: of the matrix instructions; DP: d rounded up to 64, 128 or 256; kQ: terms of a query (1 or 3); kP: of the weights
// (2 or 3); W: wavefronts (more than kPagedWaves: each workgroup has a row whole).
template <typename C, typename T, int DP, int kQ, int kP, int W>
__global__ __launch_bounds__(64 * W, W == kPagedWaves ? workgroups_of(DP) : W / 4) void paged_attention_kernel(PagedArgs a)
{
    constexpr int kRowPieces = DP * (int)sizeof(C) / 16;      // 16-byte pieces of a row: lanes to a row
    constexpr int kPer16 = 16 / (int)sizeof(C);               // elements of one
    constexpr int kRowsAtOnce = 64 / kRowPieces, kLoads = kTile / kRowsAtOnce;
    constexpr int kStride = DP + 8;                           // elements between rows in LDS
    constexpr int kSteps = DP / 32, kBlocks = DP / 16;
    constexpr int kStep = kTile * W;                          // positions of all wavefronts' tiles
    constexpr float kLift = std::is_same<T, f16>::value ? 10.0f : 0.0f;   // fp16 weights are held times 2^10, where small ones have more bits
    __shared__ __attribute__((aligned(16))) union {
        short tile[W][kTile * kStride];
        float o[W][16][DP];
    } s;
    __shared__ __attribute__((aligned(16))) short s_q[kQ][16 * kStride];
    __shared__ float s_qscale[16], s_m[W][16], s_l[W][16];
    __shared__ long s_scan[kPagedWaves], s_before;
    __shared__ int s_b;

    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int column = lane & 15, j = lane >> 4;              // head (and row of an operand), lane group
    const int row_piece = lane % kRowPieces, row_first = lane / kRowPieces;
    // Position in a tile of a group of lanes' i-th row: the lanes of a row have the places of their rows between them, and two groups that
    // share a line of 128 bytes (rows of 64) have neighbouring rows at a time.
    constexpr bool kPairs = kRowPieces == 4;
    auto position_of = [](int group, int i) { return kPairs ? (group >> 1) * 2 * kLoads + 2 * i + (group & 1) : group * kLoads + i; };
    const int my_position = position_of(row_first, lane % kLoads);
    short* tile = s.tile[wave];
    constexpr bool kPack = paged_packs(sizeof(C), DP);
    const int pack = kPack ? a.pack : 1, width = d.d * pack;
    const int rows = (kPack ? paged_rows(d.hk, pack, a.groups) : d.hk * a.groups) / a.share;   // sets of rows of a request
    // workgroup i runs on XCD i mod 8: a team's members are neighbours there
    const int member = blockIdx.x / 8 % a.share, worker = blockIdx.x / 8 / a.share * 8 + blockIdx.x % 8;

    const bool in_row = row_piece * kPer16 < width;

    // this workgroup's units [u, u1); before: the units of the requests in front of b
    int b;
    long u, u1, first, before, each = 0, longer = 0;
    int4 joined = make_int4(0, 0, 0, 0);
    bool early = false;
    int early_entry = 0;
    if (W == kPagedWaves && a.workers) {
        const Scan scan = scan_units(a, s_scan);
        const long all = scan.all * rows;
        const Shares shares(all, a.workers);
        first = u = shares.begin(worker);
        u1 = shares.begin(worker + 1);
        if (worker >= a.workers || u >= u1) {
            if (worker < a.workers && tid == 0) a.joined[member * a.workers + worker] = make_int4(0, 0, 0, 0);
            return;
        }
        each = shares.each;
        longer = shares.more;
        if (scan.before * rows <= u && u < (scan.before + scan.mine) * rows) {
            int at = scan.b0;
            long front = scan.before;
            for (long n; front * rows + (n = cost_of(a, at)) * rows <= u; front += n) ++at;
            s_b = at;
            s_before = front * rows;
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(s_b);
        before = s_before;
    } else {
        b = worker / rows;
        if (b >= d.B) return;
        before = 0;
        u = first = worker % rows;                            // a row of no positions is written too
        u1 = u + 1;
        // the first tile's pages, while the length is under way
        early = !d.window && d.max_pages;
        if (early) early_entry = d.block_table[b * d.table_stride + min((wave * kTile + my_position) >> a.shift, d.max_pages - 1)];
    }

    // The next piece of a row in this workgroup's run.
    auto advance = [&]() -> Piece {
        while (u < u1) {
            const Span span = span_of(a, b);
            const int units = (span.n - span.low + kUnit - 1) / kUnit, cost = a.workers ? units + a.extra : 1;
            if (u >= before + (long)cost * rows) {            // the next request
                before += (long)cost * rows;
                ++b;
                continue;
            }
            const int r = (int)((u - before) / cost);
            const long begin = before + (long)r * cost, end = min(u1, begin + cost);
            // a row's cost comes first, then its units
            const int from = a.workers ? max((int)(u - begin) - a.extra, 0) : 0, to = a.workers ? max((int)(end - begin) - a.extra, 0) : units;
            const bool starts = u == begin;
            u = end;
            if (units ? to == 0 : !starts) continue;          // another workgroup has what there is of it
            Piece n;
            n.b = b;
            // requests begin with different heads, so that workgroups in step with one another do not read the same part of every page
            const PagedRow row = paged_row((r + b) % rows * a.share + member, a.group, a.groups);
            n.g = row.g;
            n.h0 = row.h0;
            n.heads = row.heads;
            n.k0 = span.low + from * kUnit;
            n.k1 = (int)min((long)span.low + (long)to * kUnit, (long)span.n);
            n.slot = from == 0 && to == units ? -1 : begin > first;
            if (from == 0 && to < units) joined = make_int4(b, n.h0, n.slot, (int)(Shares(each, longer, 0).owner(begin + a.extra + units - 1) - worker) + 1);
            return n;
        }
        return Piece{-1, 0, 0, 0, 0, 0, -1};
    };
    // A tile's places: a lane has one position's distance into the cache in 16 bytes, 0 where it takes no part.  Loads are not
    // conditional (a branch around one would wait for those before it): a lane of no part reads the first page, and zeros are put
    // in the place of what it read.
    auto entry_of = [&](const Piece& n, int t0) {
        const int* table = d.max_pages && n.b >= 0 ? d.block_table + n.b * d.table_stride : reinterpret_cast<const int*>(g_zero_line);
        return table[n.k1 > 0 && n.b >= 0 ? min(t0 + my_position, n.k1 - 1) >> a.shift : 0];
    };
    auto place_of = [&](const Piece& n, int t0, int entry, unsigned long& valid) -> unsigned {
        const int k = t0 + my_position;
        const bool ok = k < n.k1 && entry >= 0 && entry < d.num_pages;
        valid = __ballot(ok);
        return ok ? (unsigned)(((long)entry * d.page_stride + (long)(k & (d.page_size - 1)) * d.slot_stride) / kPer16) : 0u;
    };
    const int lane_bytes = in_row ? row_piece * 16 : 0;
    auto fetch = [&](const void* cache, const Piece& n, unsigned place, v4u (&to)[kLoads]) {
        const char* base = d.num_pages ? static_cast<const char*>(cache) + (long)n.g * (pack * d.head_stride) * sizeof(C) + lane_bytes : reinterpret_cast<const char*>(g_zero_line);
        fetch_rows<kLoads>(base, place, to, std::make_integer_sequence<int, kLoads>{});
        __builtin_amdgcn_sched_barrier(0);                    // the order of the loads is what is waited for
    };
    auto stage = [&](const v4u (&from)[kLoads], unsigned long valid) {
        constexpr int kStep = (kPairs ? 2 : 1) * kStride;
        short* to = tile + position_of(row_first, 0) * kStride + row_piece * kPer16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) put<C, T>(to + i * kStep, from[i]);
        if (valid != ~0ul || width != DP) {
#pragma unroll 1
            for (int i = 0; i < kLoads; ++i)
                if (!in_row || !(valid >> (lane - row_piece + i) & 1)) {
#pragma unroll
                    for (int e = 0; e < kPer16; e += 8) *reinterpret_cast<v4u*>(to + i * kStep + e) = v4u{};
                }
        }
    };
    // whether the lane's score number i, of position i / 4 * 16 + j * 4 + i % 4, takes part
    auto scored = [&](int i, unsigned long valid) {
        const int at = i / 4 * 16 + j * 4 + i % 4;
        const int group = kPairs ? at / (2 * kLoads) * 2 + (at & 1) : at / kLoads, nth = kPairs ? at % (2 * kLoads) / 2 : at % kLoads;
        return valid >> (group * kRowPieces + nth) & 1;
    };

    // Queries of a piece: 16 rows (zeros behind the group's), 16 lanes each.
    const int qrow = tid >> 4, qc = tid & 15;
    // Packed key heads are one whose query rows are zero but in their own head's part (codes are finite): this thread's row's, and column's.
    const int row_part = kPack ? paged_part(qrow, a.group, pack) : 0, column_part = kPack ? paged_part(column, a.group, pack) : 0;
    // They stay as they were read until they are used: to convert one earlier would be to wait for the tiles that are under way.
    constexpr bool kLater = W == kPagedWaves;                 // (a workgroup with one row has none yet)
    unsigned q_raw[DP / 16];
    auto query = [&](unsigned raw) {
        return d.q_dtype == NM_DT_F32 ? __uint_as_float(raw) : d.q_dtype == NM_DT_BF16 ? __uint_as_float(raw << 16) : (float)__builtin_bit_cast(f16, (unsigned short)raw);
    };
    auto fetch_queries = [&](const Piece& n) {
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int c = qc + 16 * i - row_part * d.d;
            const long at = n.b * d.q_stride + (long)(n.h0 + qrow) * d.d + c;
            const bool there = n.b >= 0 && qrow < n.heads && (unsigned)c < (unsigned)d.d;
            if (kLater)
                q_raw[i] = !there ? 0u : d.q_dtype == NM_DT_F32 ? static_cast<const unsigned*>(d.q)[at] : (unsigned)static_cast<const unsigned short*>(d.q)[at];
            else
                q_raw[i] = __float_as_uint(!there ? 0.0f : d.q_dtype == NM_DT_F32 ? static_cast<const float*>(d.q)[at]
                                                         : d.q_dtype == NM_DT_BF16 ? (float)static_cast<const bf16*>(d.q)[at] : (float)static_cast<const f16*>(d.q)[at]);
        }
    };

    // What the first tile of a piece needs is requested while the piece before is under way.
    Piece now = advance();
    if (now.b < 0) {
        if (a.workers && tid == 0) a.joined[member * a.workers + worker] = joined;
        return;
    }
    int t0 = now.k0 + wave * kTile;
    int entry = early ? early_entry : entry_of(now, t0), entry2 = entry_of(now, t0 + kStep);
    fetch_queries(now);
    v4u kr[kLoads], vr[kLoads];
    unsigned long valid;
    {
        const unsigned place = place_of(now, t0, entry, valid);
        fetch(d.k_cache, now, place, kr);
        fetch(d.v_cache, now, place, vr);
    }
    while (true) {
        const Piece then = advance();
        const int then_t0 = then.k0 + wave * kTile;
        const int then_entry = entry_of(then, then_t0), then_entry2 = entry_of(then, then_t0 + kStep);
        entry = entry2;
        const int b = now.b, g = now.g, h0 = now.h0, heads = now.heads, k1 = now.k1;

        // the sign of the scale goes with the queries
        const float by = d.scale * 1.44269504088896340736f * (sizeof(C) == 1 ? d.k_scale[g * pack + row_part] : 1.0f);
        const float by_column = kPack ? d.scale * 1.44269504088896340736f * d.k_scale[g * pack + column_part] : by;
        float x[DP / 16], top_q = 0.0f, down = 1.0f, up = 1.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            x[i] = kLater ? query(q_raw[i]) : __uint_as_float(q_raw[i]);
        }
        if (kQ > 1) {
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) top_q = fmaxf(top_q, fabsf(x[i]));
            top_q = __int_as_float(group_reduce<16>(__float_as_int(top_q), MaxF32{}));
            const int e = max(-126, min((int)(__float_as_uint(top_q) >> 23) - 127, 126));   // the row goes below 4
            down = __uint_as_float((unsigned)(127 - e) << 23);
            up = __uint_as_float((unsigned)(127 + e) << 23);
        }
        __syncthreads();                                      // the piece before is done with LDS
        if (W == kPagedWaves || qrow < 16)
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            float rest = copysignf(down, by) * x[i];
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
                const T t = (T)rest;
                rest -= (float)t;
                s_q[q][qrow * kStride + qc + 16 * i] = __builtin_bit_cast(short, t);
            }
        }
        if (qc == 0 && (W == kPagedWaves || qrow < 16)) s_qscale[qrow] = up;
        __syncthreads();
        // never 0, so that it takes a masked score, minus infinity, for what it is
        const float factor = fmaxf(fabsf(by_column) * s_qscale[column], 1.17549435e-38f);

        if (t0 >= k1) {                                       // no tile for this wavefront
            const unsigned place = place_of(then, then_t0, then_entry, valid);
            fetch(d.k_cache, then, place, kr);
            fetch(d.v_cache, then, place, vr);
        }
        v4f o[kBlocks];
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) o[i] = v4f{0, 0, 0, 0};
        float m = -INFINITY, l = 0.0f;
        for (; t0 < k1; t0 += kStep) {
            unsigned long next_valid;
            const bool more = t0 + kStep < k1;
            const Piece& of = more ? now : then;
            const unsigned next = place_of(of, more ? t0 + kStep : then_t0, more ? entry : then_entry, next_valid);
            entry = entry_of(now, t0 + 2 * kStep);
            // scores
            stage(kr, valid);
            fetch(d.k_cache, of, next, kr);
            v4f sc[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                sc[blk] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int step = 0; step < kSteps; ++step) {
                    const v8s ka = *reinterpret_cast<const v8s*>(tile + (blk * 16 + column) * kStride + step * 32 + j * 8);
#pragma unroll
                    for (int q = kQ - 1; q >= 0; --q) {
                        const v8s qb = *reinterpret_cast<const v8s*>(s_q[q] + column * kStride + step * 32 + j * 8);
                        sc[blk] = Mma<T>::mma(ka, qb, sc[blk]);
                    }
                }
            }
            if (valid != ~0ul) {
                asm volatile("");                             // a branch: few tiles need it
#pragma unroll
                for (int i = 0; i < 8; ++i) sc[i / 4][i % 4] = scored(i, valid) ? sc[i / 4][i % 4] : -INFINITY;
            }
            float top = sc[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i / 4][i % 4]);
            top = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(top), MaxF32{}), MaxF32{}));
            top = fmaxf(m, top == -INFINITY ? top : top * factor);
            const float base = top == -INFINITY ? 0.0f : top;
            const float shrink = __builtin_amdgcn_exp2f(m - base);
            m = top;
            l *= shrink;
            const float lifted = kLift - base;
            v8s p[kP];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i / 4][i % 4], factor, lifted));
                l += e;
#pragma unroll
                for (int q = 0; q < kP; ++q) {
                    const T t = (T)e;
                    e = __builtin_fmaf((float)t, -1.0f, e);
                    p[q][i] = __builtin_bit_cast(short, t);
                }
            }
            // values
            stage(vr, valid);
            fetch(d.v_cache, of, next, vr);
            if (__any(shrink != 1.0f)) {
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[blk][i] *= shrink;
            }
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk) {
                const short* at = tile + (j * 4 + column / 4) * kStride + blk * 16 + column % 4 * 4;
                const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at));
                const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 16 * kStride));
                const v8s va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q) o[blk] = Mma<T>::mma(va, p[q], o[blk]);
            }
            valid = next_valid;
        }
        fetch_queries(then);
        l = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l), AddF32{}), AddF32{}));

        // the wavefronts' results as one
        if (j == 0) { s_m[wave][column] = m; s_l[wave][column] = l; }
        __syncthreads();                                      // also: no tile is read any more
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, s_m[w][column]);
        const float base = top == -INFINITY ? 0.0f : top;
        const float mine = __builtin_amdgcn_exp2f(m - base - kLift);
#pragma unroll
        for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i) s.o[wave][column][blk * 16 + j * 4 + i] = o[blk][i] * mine;
        __syncthreads();
        const float vscale = sizeof(C) == 1 ? d.v_scale[g * pack + row_part] : 1.0f;
        const int row = tid >> 4;
        if (row < heads) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s_m[w][row]);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += s_l[w][row] * __builtin_amdgcn_exp2f(s_m[w][row] - base - kLift);
            if ((tid & 15) == 0) {
                if (now.slot >= 0) a.part_ml[part_of(a, member, worker, now.slot) + row] = make_float2(top, sum);
                else if (d.lse) d.lse[(long)b * d.hq + h0 + row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
            }
            const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * vscale;
            for (int c = (tid & 15) * 4; c < d.d; c += 64) {
                v4f x{0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < W; ++w) x += *reinterpret_cast<const v4f*>(&s.o[w][row][row_part * d.d + c]);
                if (now.slot >= 0) {
                    *reinterpret_cast<v4f*>(a.part_o + (part_of(a, member, worker, now.slot) + row) * d.d + c) = x;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) store1(d.out, d.out_dtype, b * d.out_stride + (long)(h0 + row) * d.d + c + i, x[i] * by, d.out_inv_scale);
                }
            }
        }
        if (then.b < 0) {
            if (a.workers && tid == 0) a.joined[member * a.workers + worker] = joined;
            break;
        }
        now = then;
        t0 = then_t0;
        entry2 = then_entry2;
    }
}

// The rows that several runs have a piece of: a workgroup to a run and query head of its last row.  Lanes of four elements read every
// so-manieth piece's output and join them as they come; their results are joined through LDS.
__global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(PagedArgs a)
{
    __shared__ __attribute__((aligned(16))) float s_o[kPagedThreads * 4];
    __shared__ float s_m[kPagedThreads / 4], s_l[kPagedThreads / 4];
    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, member = blockIdx.x / a.workers, w0 = blockIdx.x % a.workers, nth = blockIdx.y;
    const int4 row = a.joined[blockIdx.x];
    const int used = row.w, h = row.y + nth, g = row.y / a.group;
    if (!used || h >= (g + 1) * a.group) return;
    const long bh = (long)row.x * d.hq + h;

    const int lanes = d.d / 4, at_once = kPagedThreads / lanes, mine = tid / lanes, c = tid % lanes * 4;
    float m = -INFINITY, l = 0.0f;
    v4f x{0, 0, 0, 0};
    if (mine < at_once) {
#pragma unroll 4
        for (int i = mine; i < used; i += at_once) {
            const long part = part_of(a, member, w0 + i, i == 0 ? row.z : 0) + nth;
            const float2 ml = a.part_ml[part];
            const v4f y = *reinterpret_cast<const v4f*>(a.part_o + part * d.d + c);
            const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
            const float shrink = __builtin_amdgcn_exp2f(m - base), by = __builtin_amdgcn_exp2f(ml.x - base);
            l = l * shrink + ml.y * by;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = x[e] * shrink + y[e] * by;
            m = top;
        }
        *reinterpret_cast<v4f*>(&s_o[mine * d.d + c]) = x;
        if (c == 0) { s_m[mine] = m; s_l[mine] = l; }
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.0f, v = 0.0f;
    for (int i = 0; i < at_once; ++i) top = fmaxf(top, s_m[i]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int i = 0; i < at_once; ++i) {
        const float by = __builtin_amdgcn_exp2f(s_m[i] - base);
        sum += s_l[i] * by;
        if (tid < d.d) v += s_o[i * d.d + tid] * by;
    }
    const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * (d.cache_dtype == NM_DT_I8 ? d.v_scale[h / (d.hq / d.hk)] : 1.0f);
    if (tid < d.d) store1(d.out, d.out_dtype, row.x * d.out_stride + (long)h * d.d + tid, v * by, d.out_inv_scale);
    if (tid == 0 && d.lse) d.lse[bh] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <typename C, typename T, int DP, int W>
static void launch_paged(const PagedArgs& a, int blocks, bool own, hipStream_t s)
{
    if (own && a.d.out_dtype != NM_DT_F32) queue_kernel(paged_attention_kernel<C, T, DP, 1, 2, W>, dim3(blocks), dim3(64 * W), 0, s, a);
    else queue_kernel(paged_attention_kernel<C, T, DP, 3, 3, W>, dim3(blocks), dim3(64 * W), 0, s, a);
}
// Positions that a request may have.
static long longest_of(const nm_paged_desc& d, int shift)
{
    const long longest = (long)d.max_pages << shift;
    return d.window && d.window < longest ? d.window : longest;
}
// One term of a query where the matrix instructions' type is its own, and two of the weights where the result has 16 bits or fewer.
template <typename C, typename T>
static void launch_paged(const PagedArgs& a, int blocks, hipStream_t s)
{
    const bool own = a.d.q_dtype == (std::is_same<T, f16>::value ? NM_DT_F16 : NM_DT_BF16);
    const bool wide = !a.workers && blocks <= 256 && longest_of(a.d, a.shift) > kUnit;   // eight wavefronts to a row
    const int width = paged_width(a.pack * a.d.d);
    if (width == 64) wide ? launch_paged<C, T, 64, 2 * kPagedWaves>(a, blocks, own, s) : launch_paged<C, T, 64, kPagedWaves>(a, blocks, own, s);
    else if (width == 128) launch_paged<C, T, 128, kPagedWaves>(a, blocks, own, s);
    else launch_paged<C, T, 256, kPagedWaves>(a, blocks, own, s);
}

// What does not depend on pointers: shapes, types, and how the work is shared.
static int32_t plan_paged(const nm_paged_desc* d, PagedArgs* a, size_t* bytes, long* blocks, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    if (d->B < 0 || d->hq < 1 || d->hk < 1 || d->hq % d->hk || d->d < 1 || d->max_pages < 0 || d->num_pages < 0 || d->window < 0)
        return fail(NM_ERR_INVALID_ARG, "%s: bad shape", what);
    if (!float_dtype(d->q_dtype)) return fail(NM_ERR_INVALID_ARG, "%s: bad q_dtype", what);
    if (d->cache_dtype != NM_DT_BF16 && d->cache_dtype != NM_DT_F16 && d->cache_dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "%s: bad cache_dtype", what);
    if (!float_dtype(d->out_dtype) && d->out_dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "%s: bad out_dtype", what);
    if (d->d % 16 || d->d > 256) return fail(NM_ERR_UNSUPPORTED, "%s: d %d is no multiple of 16 up to 256", what, d->d);
    const int shift = page_shift(d->page_size);
    if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "%s: page_size %d is no power of two up to 65536", what, d->page_size);
    if ((int64_t)d->num_pages << shift > 0x7fffffffLL || (int64_t)d->max_pages << shift > 0x3fffffffLL)
        return fail(NM_ERR_UNSUPPORTED, "%s: num_pages * page_size >= 2^31 or max_pages * page_size >= 2^30", what);
    // distances into a cache are held in 16 bytes, in 31 bits (the strides are not negative: checked before any launch)
    if ((double)d->num_pages * (double)d->page_stride + (double)d->page_size * (double)d->slot_stride >= 2147483648.0 * 16 / dtype_bytes(d->cache_dtype))
        return fail(NM_ERR_UNSUPPORTED, "%s: a cache of more than 32 GiB", what);
    if ((int64_t)d->B * d->hq >= 1 << 23) return fail(NM_ERR_UNSUPPORTED, "%s: B * hq >= 2^23", what);
    *a = PagedArgs{};
    a->d = *d;
    a->shift = shift;
    static_cast<PagedSplit&>(*a) = paged_split({d->B, d->hq, d->hk, d->d, dtype_bytes(d->cache_dtype), d->slot_stride, d->head_stride, longest_of(*d, shift)});
    a->extra = 2;
    const long teams = ((a->workers ? a->workers : paged_sets(d->B, d->hk, *a)) + 7) / 8 * 8;   // every XCD has as many
    *blocks = teams * a->share;
    const size_t parts = (size_t)a->share * a->workers * 2 * 16;
    *bytes = parts * (sizeof(float2) + d->d * sizeof(float)) + parts / 32 * sizeof(int4);
    return NM_OK;
}

int32_t check_paged_shape(const nm_paged_desc* d, bool* divided, const char* what)
{
    PagedArgs a;
    long blocks;
    size_t n;
    const int32_t rc = plan_paged(d, &a, &n, &blocks, what);
    *divided = !rc && a.workers;
    return rc;
}

// What a call checks of its pointers and strides (plan_paged has looked at its shapes and types).
int32_t check_paged(const nm_paged_desc* d, const char* what)
{
    const int64_t row = (int64_t)d->hq * d->d;
    if (d->q_stride < row || d->out_stride < row || d->table_stride < d->max_pages) return fail(NM_ERR_INVALID_ARG, "%s: a stride is shorter than a row", what);
    if (d->page_stride < 0 || d->slot_stride < 0 || d->head_stride < 0) return fail(NM_ERR_INVALID_ARG, "%s: negative stride of the cache", what);
    if (!(d->scale == d->scale) || __builtin_isinf(d->scale)) return fail(NM_ERR_INVALID_ARG, "%s: scale must be finite", what);
    if (d->B == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->q || !d->lens || !d->out) return fail(NM_ERR_INVALID_ARG, "%s: q, lens or out is NULL", what);
    if (d->out == d->q && (d->out_dtype != d->q_dtype || d->out_stride != d->q_stride)) return fail(NM_ERR_INVALID_ARG, "%s: in place with another type or stride", what);
    const std::initializer_list<const void*> read = {d->k_cache, d->v_cache, d->k_scale, d->v_scale, d->block_table, d->lens};
    if (begins_as(d->out, read) || begins_as(d->lse, read) || begins_as(d->lse, {d->q, d->out}))
        return fail(NM_ERR_INVALID_ARG, "%s: out or lse is an input, or lse is out", what);
    if ((d->max_pages && !d->block_table) || (d->max_pages && d->num_pages && (!d->k_cache || !d->v_cache)))
        return fail(NM_ERR_INVALID_ARG, "%s: block_table or a cache is NULL", what);
    if (d->cache_dtype == NM_DT_I8 && (!d->k_scale || !d->v_scale)) return fail(NM_ERR_INVALID_ARG, "%s: int8 cache without scales", what);
    const int per16 = 16 / dtype_bytes(d->cache_dtype);
    if (!aligned(d->k_cache, 16) || !aligned(d->v_cache, 16) || d->page_stride % per16 || d->slot_stride % per16 || d->head_stride % per16)
        return fail(NM_ERR_UNSUPPORTED, "%s: the cache's addresses and strides must be multiples of 16 bytes", what);
    return NM_OK;
}

}  // namespace nm

using namespace nm;

extern "C" {

int32_t nm_paged_attention_workspace(const nm_paged_desc* d, size_t* bytes)
{
    PagedArgs a;
    long blocks;
    size_t n;
    const int32_t rc = plan_paged(d, &a, &n, &blocks, "nm_paged_attention_workspace");
    if (rc) return rc;
    if (!bytes) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention_workspace: bytes is NULL");
    *bytes = n;
    return NM_OK;
}

int32_t nm_paged_attention(const nm_paged_desc* d, void* ws, size_t ws_bytes, void* stream)
{
    PagedArgs a;
    long blocks;
    size_t need;
    const int32_t rc = plan_paged(d, &a, &need, &blocks, "nm_paged_attention");
    if (rc) return rc;
    if (const int32_t bad = check_paged(d, "nm_paged_attention")) return bad;
    if (d->B == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (need) {
        if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_paged_attention: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
        if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_paged_attention: workspace must be 256-byte aligned");
        const size_t runs = (size_t)a.share * a.workers;
        a.joined = static_cast<int4*>(ws);
        a.part_ml = reinterpret_cast<float2*>(a.joined + runs);
        a.part_o = reinterpret_cast<float*>(a.part_ml + runs * 2 * 16);
    }
    if (d->cache_dtype == NM_DT_BF16) launch_paged<bf16, bf16>(a, (int)blocks, (hipStream_t)stream);
    else if (d->cache_dtype == NM_DT_F16) launch_paged<f16, f16>(a, (int)blocks, (hipStream_t)stream);
    else if (d->q_dtype == NM_DT_F16) launch_paged<int8_t, f16>(a, (int)blocks, (hipStream_t)stream);
    else launch_paged<int8_t, bf16>(a, (int)blocks, (hipStream_t)stream);
    if (need) {
        const int32_t err = check_hip(hipGetLastError(), "nm_paged_attention launch");
        if (err) return err;
        queue_kernel(paged_join_kernel, dim3(a.share * a.workers, a.group < 16 ? a.group : 16), dim3(kPagedThreads), 0, (hipStream_t)stream, a);
    }
    return check_hip(hipGetLastError(), "nm_paged_attention launch");
}

}  // extern "C"
