// Attention of one new token per row over a paged cache, where groups of rows share a prefix (nm_shared_attention).
//
// Each row's own positions are nm_paged_attention's work: every key and value once, bound by memory.  A group's prefix is read once for all its
// rows: for one key head the queries of all of them, rows times heads, are as many columns of the same matrix products.  Softmax over both: each piece
// of work, a range of positions, leaves its maximum, sum and output, and a last kernel joins what a query has.
//   A first kernel of one workgroup makes three lists, by a range's queries.  Up to 16, which the rows' own are: as nm_paged_attention takes them, each of
// a workgroup's four wavefronts has tiles of 32 positions of its own.  More: 128 positions at a time are in LDS for all wavefronts, each of which has 32
// queries in registers (16 where they are three terms), and, where there are fewer queries than that, only some of the positions.  Up to 64 queries (32),
// in the first list's launch, four wavefronts; more, in a launch of their own, eight wavefronts and 256 queries (128 of heads of more than 128 elements, and of
// heads of more than 64 where queries are three terms) to a CU, which has registers for the operands of one product while another runs, and LDS for the next positions beside these.  (With four wavefronts of 64 queries each, one to a
// SIMD, nothing ran under a wavefront's own waits: 18 us for 128 positions, 7 so.)  A fixed number of workgroups shares each list evenly, whatever the lengths
// are (the first two lists' by their cost; a range costs its units of 128 positions and two, however many queries its tile has, so that tiles of the third list that
// are not full, 128 of 256 queries for one, take less time than they count for); a run's first and last piece may be parts of a range.  Tiles, operand layouts and precision are nm_paged_attention's, but that a
// running maximum is only moved when it is passed by a factor of 32.
//   bf16, 32 query and 8 key heads of 128, GPU time: 64 rows behind 32768 common positions (190 MB, 35 GFLOP) 107 us: 7 the lists, 23 the rows' own, 66 the
// prefix (39 % of the cycles in matrix instructions, 44 % in vector instructions, which one after the other would fill them: the weights' two terms are both
// double the second product and half of the vector instructions), 11 the joining of 36 pieces a query.  96 rows behind 4096, each with up to 4096 of its own (671 MB) 180: 130 the own
// positions, at a copy's rate.  int8, 16 heads of 64, two as one, 16 groups of 8 rows behind up to 8192 (134 MB) 64: 45 for 3500 units of 128 positions and a thousand ranges of one
// or two, whose beginning and end cost as much as two more.
//   Registers: the first two lists' kernel has those that the second list's code takes, for the rows' own positions too: heads of 128 of 16-bit caches 256, and 28 to 36 bytes of scratch
// a lane; of 64 about 180, two workgroups to a CU where nm_paged_attention has three.  Heads of 256 with queries of three terms spill 90 registers in the third list's kernel (270 to 290 bytes).
#include "nm_paged_parts.h"

namespace nm {

constexpr int kSharedMost = NM_PLAN_MAX_REQUESTS;     // rows, groups
// Shorter prefixes are every row's own.  (256 rows of 32 heads of 128 in groups of 2 to 64 behind up to 512, 1024 and 2048 positions: 128, 256 and 512 within 3 % of one
// another, 768 up to 12 % longer; all of them their own, 16 rows to a group: 70, 102 and 143 us, shared 70, 106 and 112.)
constexpr int kSharePrefix = kUnit;
constexpr int kPlanners = 1024;
// Units of all rows up to which nm_paged_attention takes them, two to each of its workgroups or fewer: 4 rows of 640 positions, 12 heads of 64, 13.9 us,
// 20.8 by the lists.
constexpr long kFewUnits = 1024;
constexpr int kLists = 3;

// Wavefronts of a list's workgroups; sixteens of queries that one has of a range, by the heads' size and the terms of a query; and queries of a range.
constexpr int shared_waves(int list) { return list == 2 ? 2 * kPagedWaves : kPagedWaves; }
constexpr int shared_sets(int list, int dp, int terms) { return list == 0 ? 1 : terms == 1 ? (dp <= 128 ? 2 : 1) : list == 2 && dp <= 64 ? 2 : 1; }
constexpr int shared_tile(int list, int dp, int terms) { return list == 0 ? 16 : (list == 1 ? 2 : shared_waves(2)) * 16 * shared_sets(list, dp, terms); }

// Quotients of numbers that are not negative: a division of 32 bits takes a tenth of one of 64.
__device__ __forceinline__ long divided(long n, long by) { return (n | by) >> 31 ? n / by : (long)((unsigned)n / (unsigned)by); }
// As Shares, by these.
struct Portions {
    long each, more;
    __device__ __forceinline__ Portions(long all, long workers) : each(divided(all, workers)), more(all - each * workers) {}
    __device__ __forceinline__ Portions(long e, long m, int) : each(e), more(m) {}
    __device__ __forceinline__ long begin(long w) const { return each * w + min(w, more); }
    __device__ __forceinline__ long owner(long x) const
    {
        const long longer = (each + 1) * more;
        return x < longer ? divided(x, each + 1) : more + divided(x - longer, each);
    }
};

struct SharedHead { long each[kLists], more[kLists]; int workers[kLists]; };   // how a list's cost is divided
struct SharedArgs {
    nm_paged_desc d;
    int G;
    const int32_t* group_start;
    const int32_t* shared;
    int shift, own;              // log2 of page_size, query heads of a key head
    // Neighbouring key heads of int8 may be taken as one, whose queries are zero but in their own head's part (codes are finite): how many there are then, their
    // elements and query heads, and how many are one.
    int heads, width, group, pack;
    int tile[kLists];            // log2 of the queries of a range
    FastDiv by_group;
    int workers, last;           // of the first two lists, and of the third
    int whole_queries;           // 8 elements of a query may be read at once
    SharedHead* head;
    int4* ent;                   // [G + B]: a group: first row, rows, the row whose table it goes by, positions; a row: itself, 1, its own first position, its length
    int* lead;                   // [B]: first row of the group whose prefix the row shares, -1: none
    long* before;                // [kLists, workers]: cost of the entities in front of a worker's first
    int* first;                  // [kLists, workers]: a worker's first entity
    int4* info;                  // [2, B, hq], by a range's first query: how many pieces it has (0: none, -1: the result is there), where the first's part is (-1:
                                 // whole), where the second's is, and how far apart those behind it are
    float2* part_ml;             // [workers, 2, tile] of each list: maximum (of scores in units of log 2) and sum
    float* part_o;               // [likewise, d]: not yet divided by the sum
    float2* whole_ml;            // [2, B, hq]: prefixes, own positions
    float* whole_o;              // [2, B, hq, d]
};

// What an entity is, which list it is on, and what it costs.
struct Entity {
    int row0, table, k0, k1, queries, list, tile, tiles, units, extra;
    __device__ __forceinline__ Entity(const SharedArgs& a, int e)
    {
        const int4 x = a.ent[e];
        const bool prefix = e < a.G;
        row0 = x.x;
        table = prefix ? x.z : x.x;
        k0 = prefix ? 0 : x.z;
        k1 = x.w;
        queries = prefix && k1 <= 0 ? 0 : x.y * a.group;
        list = !prefix || queries <= 1 << a.tile[0] ? 0 : queries <= 1 << a.tile[1] ? 1 : 2;
        const int shift = list == 0 ? a.tile[0] : list == 1 ? a.tile[1] : a.tile[2];
        tile = 1 << shift;
        tiles = (queries + tile - 1) >> shift;
        units = (k1 - k0 + kUnit - 1) / kUnit;
        extra = 2;                                            // beginning and ending a range, in units
    }
    __device__ __forceinline__ long cost() const { return units + extra; }                             // of a key head's tile, in units
    __device__ __forceinline__ long all(const SharedArgs& a) const { return cost() * a.heads * tiles; }
};

__global__ __launch_bounds__(kPlanners) void shared_plan_kernel(SharedArgs a)
{
    // the groups' starts and first rows that take part; then, of each list, the cost of the entities in front of each (rows are on the first alone)
    __shared__ union {
        struct { int start[kSharedMost + 1], lead[kSharedMost]; } g;
        struct { long rows[2 * kSharedMost + 1], groups[kLists - 1][kSharedMost + 1]; } before;
    } s;
    __shared__ long s_wave[kLists][kPlanners / 64];
    int (&s_start)[kSharedMost + 1] = s.g.start, (&s_lead)[kSharedMost] = s.g.lead;
    const int tid = threadIdx.x, B = a.d.B, lane = tid & 63;
    bool good = true;
    for (int g = tid; g <= a.G; g += kPlanners) s_start[g] = a.G ? a.group_start[g] : 0;
    __syncthreads();
    for (int g = tid; g < a.G; g += kPlanners) {
        s_lead[g] = B;
        good &= s_start[g] >= 0 && s_start[g] <= s_start[g + 1] && s_start[g + 1] <= B;
    }
    good = __syncthreads_and(good);
    const int G = good ? a.G : 0;
    const long cap = (long)a.d.max_pages << a.shift;
    for (int b = tid; b < B; b += kPlanners) {
        const int n = (int)min((long)max(a.d.lens[b], 0), cap);
        int own = 0, lead = -1;
        if (G && b >= s_start[0] && b < s_start[G]) {
            int lo = 0, hi = G;                        // the group is in [lo, hi)
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (s_start[mid] <= b) lo = mid; else hi = mid;
            }
            const int p = (int)min((long)max(a.shared[lo], 0), cap);
            if (p >= kSharePrefix && n >= p && s_start[lo + 1] - s_start[lo] > 1) {
                own = p;
                lead = s_start[lo];
                atomicMin(&s_lead[lo], b);
            }
        }
        a.lead[b] = lead;
        a.ent[a.G + b] = make_int4(b, 1, own, n);
    }
    __syncthreads();
    for (int g = tid; g < a.G; g += kPlanners) {
        const bool shares = good && s_lead[g] < B;
        a.ent[g] = make_int4(s_start[g], shares ? s_start[g + 1] - s_start[g] : 0, shares ? s_lead[g] : 0, shares ? (int)min((long)a.shared[g], cap) : 0);
    }
    __syncthreads();
    // a thread's run of entities, then the threads' (an entity costs nothing on the lists that it is not on)
    const int n = a.G + B, per = (n + kPlanners - 1) / kPlanners, e0 = min(tid * per, n), e1 = min(e0 + per, n);
    long mine[kLists], in[kLists], front[kLists], cost[kLists];
#pragma unroll
    for (int list = 0; list < kLists; ++list) mine[list] = 0;
    for (int e = e0; e < e1; ++e) {
        const Entity x(a, e);
        const long all = x.all(a);
#pragma unroll
        for (int list = 0; list < kLists; ++list) mine[list] += x.list == list ? all : 0;
    }
#pragma unroll
    for (int list = 0; list < kLists; ++list) in[list] = mine[list];
#pragma unroll
    for (int step = 1; step < 64; step <<= 1)
#pragma unroll
        for (int list = 0; list < kLists; ++list) {
            const long t = __shfl_up(in[list], step);
            if (lane >= step) in[list] += t;
        }
#pragma unroll
    for (int list = 0; list < kLists; ++list)
        if (lane == 63) s_wave[list][tid >> 6] = in[list];
    __syncthreads();
#pragma unroll
    for (int list = 0; list < kLists; ++list) {
        front[list] = in[list] - mine[list];
        cost[list] = 0;
#pragma unroll
        for (int w = 0; w < kPlanners / 64; ++w) {
            const long t = s_wave[list][w];
            front[list] += w < tid >> 6 ? t : 0;
            cost[list] += t;
        }
    }
    for (int e = e0; e < e1; ++e) {
        s.before.rows[e] = front[0];
        if (e < a.G) s.before.groups[0][e] = front[1], s.before.groups[1][e] = front[2];
        const Entity x(a, e);
        const long all = x.all(a);
#pragma unroll
        for (int list = 0; list < kLists; ++list) front[list] += x.list == list ? all : 0;
    }
    if (tid == 0) s.before.rows[n] = cost[0], s.before.groups[0][a.G] = cost[1], s.before.groups[1][a.G] = cost[2];
    // the first two lists' workers by their cost
    const long both = cost[0] + cost[1];
    const long second = cost[1] ? min(max(1l, (long)((double)a.workers * (double)cost[1] / (double)both + 0.5)), (long)a.workers - (cost[0] > 0)) : 0;
    const long workers[kLists] = {min((long)a.workers - second, cost[0]), min(second, cost[1]), min((long)a.last, cost[2])};
    __syncthreads();
    for (long i = tid; i < workers[0] + workers[1] + workers[2]; i += kPlanners) {
        const int list = i < workers[0] ? 0 : i < workers[0] + workers[1] ? 1 : 2;
        const long w = i - (list > 0 ? workers[0] : 0) - (list > 1 ? workers[1] : 0);
        const Portions shares(list == 0 ? cost[0] : list == 1 ? cost[1] : cost[2], list == 0 ? workers[0] : list == 1 ? workers[1] : workers[2]);
        if (w == 0) {
            a.head->each[list] = shares.each;
            a.head->more[list] = shares.more;
        }
        const long x = shares.begin(w);
        const long* before = list == 0 ? s.before.rows : s.before.groups[list - 1];
        int lo = 0, hi = list == 0 ? n : a.G;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (before[mid] <= x) lo = mid; else hi = mid;
        }
        a.first[list * a.workers + w] = lo;
        a.before[list * a.workers + w] = before[lo];
    }
    if (tid < kLists) a.head->workers[tid] = (int)(tid == 0 ? workers[0] : tid == 1 ? workers[1] : workers[2]);
}

// What a workgroup has of a range: positions [k0, k1) by the table of row `table` (-1: none) for key head g and the n queries from number i0 on of the rows from
// row0 on; slot: where its part goes, -1 where it is the whole range; prefix: of a group; done: its result is the query's.
struct SharedPiece { int table, row0, g, i0, n, k0, k1, slot, prefix, done; };

// A worker's run through its list.
struct Run {
    Portions shares;
    long first, u, u1, before;
    int e, list, worker;
    __device__ __forceinline__ Run(const SharedArgs& a, const SharedHead& head, int list, int worker)
        : shares(head.each[list], head.more[list], 0), first(shares.begin(worker)), u(first), u1(shares.begin(worker + 1)),
          before(a.before[list * a.workers + worker]), e(a.first[list * a.workers + worker]), list(list), worker(worker) {}
    // Number of the first query's part of a worker's slot.
    static __device__ __forceinline__ long part_of(const SharedArgs& a, int list, long worker, int slot)
    {
        return (list > 0 ? (2l * a.workers) << a.tile[0] : 0l) + (list > 1 ? (2l * a.workers) << a.tile[1] : 0l) + ((worker * 2 + slot) << (list == 0 ? a.tile[0] : list == 1 ? a.tile[1] : a.tile[2]));
    }
    __device__ __forceinline__ SharedPiece next(const SharedArgs& a)
    {
        while (u < u1) {
            const Entity x(a, e);
            const long cost = x.cost(), all = x.list == list ? x.all(a) : 0;
            if (u >= before + all) {                          // the next entity
                before += all;
                ++e;
                continue;
            }
            const int r = (int)divided(u - before, cost);
            const long begin = before + r * cost, end = min(u1, begin + cost);
            // a range's cost comes first, then its units
            const int from = (int)max(u - begin - x.extra, 0l), to = (int)max(end - begin - x.extra, 0l);
            const bool starts = u == begin;
            u = end;
            if (x.units ? from == to : !starts) continue;     // another workgroup has what there is of it
            SharedPiece n;
            n.table = x.table;
            n.row0 = x.row0;
            n.g = x.tiles == 1 ? r : r / x.tiles;
            n.i0 = (r - n.g * x.tiles) * x.tile;
            n.n = min(x.queries - n.i0, x.tile);
            n.k0 = x.k0 + from * kUnit;
            n.k1 = (int)min((long)x.k0 + (long)to * kUnit, (long)x.k1);
            n.slot = from == 0 && to == x.units ? -1 : begin > first;
            n.prefix = e < a.G;
            n.done = !n.prefix && x.k0 == 0 && n.slot < 0;
            if (from == 0 && threadIdx.x == 0) {
                const int count = n.done ? -1 : x.units ? (int)(shares.owner(begin + x.extra + x.units - 1) - worker) + 1 : 0;
                const int row = (int)quotient(n.i0, a.by_group);
                a.info[((long)!n.prefix * a.d.B + x.row0 + row) * a.d.hq + n.g * a.group + n.i0 - row * a.group] =
                    make_int4(count, n.slot < 0 ? -1 : (int)part_of(a, list, worker, n.slot), (int)part_of(a, list, worker + 1, 0), 2 * x.tile);
            }
            return n;
        }
        return SharedPiece{-1, 0, 0, 0, 0, 0, 0, -1, 0, 0};
    }
};

// What both lists' code needs of a cache with elements C, for matrix instructions of T and heads of up to DP elements.
template <typename C, typename T, int DP>
struct Tiles {
    static constexpr int kRowPieces = DP * (int)sizeof(C) / 16;      // 16-byte pieces of a row: lanes to a row
    static constexpr int kPer16 = 16 / (int)sizeof(C);               // elements of one
    static constexpr int kRowsAtOnce = 64 / kRowPieces, kLoads = kTile / kRowsAtOnce;
    static constexpr int kStride = DP + 8;                           // elements between rows in LDS
    static constexpr int kSteps = DP / 32, kBlocks = DP / 16;
    static constexpr float kLift = std::is_same<T, f16>::value ? 10.0f : 0.0f;   // fp16 weights are held times 2^10, where small ones have more bits
    static constexpr bool kPairs = kRowPieces == 4;

    const SharedArgs& a;
    int lane, column, j, row_piece, row_first, my_position, lane_bytes;
    bool in_row;
    static __device__ __forceinline__ int position_of(int group, int i) { return kPairs ? (group >> 1) * 2 * kLoads + 2 * i + (group & 1) : group * kLoads + i; }
    __device__ __forceinline__ Tiles(const SharedArgs& a) : a(a)
    {
        lane = threadIdx.x & 63;
        column = lane & 15;                                   // query (and row of an operand)
        j = lane >> 4;                                        // lane group
        row_piece = lane % kRowPieces;
        row_first = lane / kRowPieces;
        my_position = position_of(row_first, lane % kLoads);
        in_row = row_piece * kPer16 < a.width;
        lane_bytes = in_row ? row_piece * 16 : 0;
    }
    // A tile's places: a lane has one position's distance into the cache in 16 bytes, 0 where it takes no part.  Loads are not
    // conditional: a lane of no part reads the first page, and zeros are put in the place of what it read.
    __device__ __forceinline__ int entry_of(const SharedPiece& n, int t0) const
    {
        const bool some = n.table >= 0 && n.k1 > 0;
        const int* table = a.d.max_pages && some ? a.d.block_table + n.table * a.d.table_stride : reinterpret_cast<const int*>(g_zero_line);
        return table[some ? min(t0 + my_position, n.k1 - 1) >> a.shift : 0];
    }
    __device__ __forceinline__ unsigned place_of(const SharedPiece& n, int t0, int entry, unsigned long& valid) const
    {
        const int k = t0 + my_position;
        const bool ok = k < n.k1 && entry >= 0 && entry < a.d.num_pages;
        valid = __ballot(ok);
        return ok ? (unsigned)(((long)entry * a.d.page_stride + (long)(k & (a.d.page_size - 1)) * a.d.slot_stride) / kPer16) : 0u;
    }
    __device__ __forceinline__ void fetch(const void* cache, const SharedPiece& n, unsigned place, v4u (&to)[kLoads]) const
    {
        const char* base = a.d.num_pages ? static_cast<const char*>(cache) + (long)n.g * (a.pack * a.d.head_stride) * sizeof(C) + lane_bytes : reinterpret_cast<const char*>(g_zero_line);
        fetch_rows<kLoads>(base, place, to, std::make_integer_sequence<int, kLoads>{});
        __builtin_amdgcn_sched_barrier(0);                    // the order of the loads is what is waited for
    }
    __device__ __forceinline__ void stage(short* tile, const v4u (&from)[kLoads], unsigned long valid) const
    {
        constexpr int kRow = (kPairs ? 2 : 1) * kStride;
        short* to = tile + position_of(row_first, 0) * kStride + row_piece * kPer16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) put<C, T>(to + i * kRow, from[i]);
        if (valid != ~0ul || a.width != DP) {
#pragma unroll 1
            for (int i = 0; i < kLoads; ++i)
                if (!in_row || !(valid >> (lane - row_piece + i) & 1)) {
#pragma unroll
                    for (int c = 0; c < kPer16; c += 8) *reinterpret_cast<v4u*>(to + i * kRow + c) = v4u{};
                }
        }
    }
    // whether the lane's score number i, of position i / 4 * 16 + j * 4 + i % 4, takes part
    static __device__ __forceinline__ bool scored(int i, int j, unsigned long valid)
    {
        const int at = i / 4 * 16 + j * 4 + i % 4;
        const int group = kPairs ? at / (2 * kLoads) * 2 + (at & 1) : at / kLoads, nth = kPairs ? at % (2 * kLoads) / 2 : at % kLoads;
        return valid >> (group * kRowPieces + nth) & 1;
    }
    __device__ __forceinline__ v8s keys_of(const short* tile, int blk, int step) const { return *reinterpret_cast<const v8s*>(tile + (blk * 16 + column) * kStride + step * 32 + j * 8); }
    __device__ __forceinline__ v8s values_of(const short* tile, int blk) const
    {
        const short* at = tile + (j * 4 + column / 4) * kStride + blk * 16 + column % 4 * 4;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 16 * kStride));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // A tile's scores of S sixteens of queries into weights of kP terms; the queries' sums and outputs so far go along.  m is what is subtracted: a maximum, or up
    // to kSlack less (a weight of up to 2^5 has as many bits, and with fp16's lift stays below 2^16), so that few tiles change it.
    static constexpr float kSlack = 5.0f;
    template <int S, int kP>
    __device__ __forceinline__ void weigh(v4f (&sc)[S][2], unsigned long valid, const float (&factor)[S], float (&m)[S], float (&l)[S], v8s (&p)[S][kP], v4f (&o)[S][kBlocks]) const
    {
        if (valid != ~0ul) {                                  // a branch: few tiles need it, and nothing of it is to be held in registers
            int group = j;
            asm volatile("" : "+v"(group));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = scored(i, group, valid);
#pragma unroll
                for (int t = 0; t < S; ++t) sc[t][i / 4][i % 4] = in ? sc[t][i / 4][i % 4] : -INFINITY;
            }
        }
        float top[S];
        bool over = false;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            top[t] = sc[t][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top[t] = fmaxf(top[t], sc[t][i / 4][i % 4]);
            top[t] *= factor[t];
            over |= top[t] > m[t] + kSlack;
        }
        if (__any(over)) {                                    // few tiles need it
#pragma unroll
            for (int t = 0; t < S; ++t) {
                const float most = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(top[t]), MaxF32{}), MaxF32{}));
                const float next = most > m[t] + kSlack ? most : m[t];
                const float shrink = __builtin_amdgcn_exp2f(m[t] - (next == -INFINITY ? 0.0f : next));
                m[t] = next;
                l[t] *= shrink;
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][blk][i] *= shrink;
            }
        }
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const float lifted = kLift - (m[t] == -INFINITY ? 0.0f : m[t]);
            typedef float Pair __attribute__((ext_vector_type(2)));
            typedef T Term __attribute__((ext_vector_type(2)));
            Pair sum = {0, 0};
            v4u words[kP];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {                  // by two: one conversion
                Pair w;
#pragma unroll
                for (int k = 0; k < 2; ++k) w[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][(i + k) / 4][(i + k) % 4], factor[t], lifted));
                sum += w;
#pragma unroll
                for (int q = 0; q < kP; ++q) {
                    const Term v = __builtin_convertvector(w, Term);
                    if (q + 1 < kP) w -= __builtin_convertvector(v, Pair);   // exact
                    words[q][i / 2] = __builtin_bit_cast(unsigned, v);
                }
            }
#pragma unroll
            for (int q = 0; q < kP; ++q) p[t][q] = __builtin_bit_cast(v8s, words[q]);
            l[t] += sum[0] + sum[1];
        }
    }
    // Calls use(Q{}) with the queries' type: that of the matrix instructions where they are of one term.  (One branch in front of all loads: a branch at
    // each has every one wait for the one before.)
    template <int kQ, typename Use>
    __device__ __forceinline__ void typed(Use use) const
    {
        if constexpr (kQ == 1) use(T{});
        else if (a.d.q_dtype == NM_DT_F32) use(0.0f);
        else if (a.d.q_dtype == NM_DT_BF16) use(bf16{});
        else use(f16{});
    }
    // Number of a query's first element.
    __device__ __forceinline__ long query_of(const SharedPiece& n, int row) const
    {
        const int i = n.i0 + row, b = (int)quotient(i, a.by_group);
        return (long)(n.row0 + b) * a.d.q_stride + (long)(n.g * a.group + i - b * a.group) * a.d.d;
    }
    // Of a range's query number `row`: which of the heads taken as one is its own, and what its scores are multiplied by, but for its own scale; the sign goes with
    // the query.
    __device__ __forceinline__ int part_of(const SharedPiece& n, int row) const { return sizeof(C) == 1 && a.pack > 1 ? (n.i0 + row) % a.group / a.own : 0; }
    __device__ __forceinline__ float scale_of(const SharedPiece& n, int row) const
    {
        return a.d.scale * 1.44269504088896340736f * (sizeof(C) == 1 ? a.d.k_scale[n.g * a.pack + part_of(n, row)] : 1.0f);
    }
    // Powers of two that bring a query of three terms below 4, and back.
    static __device__ __forceinline__ void level(float top, float& down, float& up)
    {
        const int exponent = max(-126, min((int)(__float_as_uint(top) >> 23) - 127, 126));
        down = __uint_as_float((unsigned)(127 - exponent) << 23);
        up = __uint_as_float((unsigned)(127 + exponent) << 23);
    }
    // Writes a query's part or result, its maximum and sum: elements(put) calls put(c, y) for the lane's runs of four elements, from c on.
    template <typename Elements>
    __device__ __forceinline__ void leave(const SharedPiece& n, int row, long part, Elements elements, float top, float sum) const
    {
        const nm_paged_desc& d = a.d;
        const int i = n.i0 + row, nth = (int)quotient(i, a.by_group), b = n.row0 + nth, h = n.g * a.group + i - nth * a.group;
        if (!n.done) {
            const long at = n.slot < 0 ? ((long)!n.prefix * d.B + b) * d.hq + h : part + row;
            float* to = (n.slot < 0 ? a.whole_o : a.part_o) + at * d.d;
            elements([&](int c, v4f y) {
                if (c == 0) (n.slot < 0 ? a.whole_ml : a.part_ml)[at] = make_float2(top, sum);
                *reinterpret_cast<v4f*>(to + c) = y;
            });
            return;
        }
        const float over = (sum == 0.0f ? 0.0f : 1.0f / sum) * (sizeof(C) == 1 ? d.v_scale[h / a.own] : 1.0f);
        elements([&](int c, v4f y) {
            if (c == 0 && d.lse) d.lse[(long)b * d.hq + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
#pragma unroll
            for (int k = 0; k < 4; ++k) store1(d.out, d.out_dtype, b * d.out_stride + (long)h * d.d + c + k, y[k] * over, d.out_inv_scale);
        });
    }
};

// Memory of a workgroup.
template <int DP, int kQ, int W>
struct SharedLds {
    static constexpr int kBuffers = W > kPagedWaves && DP <= 128 ? 2 : 1;   // eight wavefronts have a CU's memory for themselves
    union {
        struct { short q[kQ][16 * (DP + 8)], tile[kPagedWaves][kTile * (DP + 8)]; } few;
        struct { short k[kPagedWaves][kTile * (DP + 8)], v[kPagedWaves][kTile * (DP + 8)]; } many[kBuffers];
        float o[W][16][DP];
    };
    float m[W][16], l[W][16], q_scale[16];
    unsigned long valid[kBuffers][kPagedWaves];
};

// A run through the first list: ranges of up to 16 queries, tiles of a wavefront's own.  What the first tile of a piece needs is requested while the
// piece before is under way.
template <typename C, typename T, int DP, int kQ, int kP>
__device__ __forceinline__ void run_few(const SharedArgs& a, Run run, SharedLds<DP, kQ, kPagedWaves>& s)
{
    using X = Tiles<C, T, DP>;
    constexpr int W = kPagedWaves, kStep = kTile * W, kStride = X::kStride;
    const X x(a);
    const int tid = threadIdx.x, wave = tid >> 6, qrow = tid >> 4, qc = tid & 15;
    short* tile = s.few.tile[wave];
    SharedPiece now = run.next(a);
    if (now.table < 0) return;
    int t0 = now.k0 + wave * kTile;
    int entry = x.entry_of(now, t0), entry2 = x.entry_of(now, t0 + kStep);
    v4u kr[X::kLoads], vr[X::kLoads];
    unsigned long valid;
    {
        const unsigned place = x.place_of(now, t0, entry, valid);
        x.fetch(a.d.k_cache, now, place, kr);
        x.fetch(a.d.v_cache, now, place, vr);
    }
    while (true) {
        const SharedPiece then = run.next(a);
        const int then_t0 = then.k0 + wave * kTile;
        const int then_entry = x.entry_of(then, then_t0), then_entry2 = x.entry_of(then, then_t0 + kStep);
        entry = entry2;
        const int k1 = now.k1, mine = min(qrow, now.n - 1), part = x.part_of(now, mine);   // this thread's query's
        const float by = x.scale_of(now, mine);
        __syncthreads();                                      // the piece before is done with LDS
        {
            const long at = x.query_of(now, mine);
            const int c0 = qc - part * a.d.d;                  // the thread's first element of its own head
            float y[DP / 16], top = 0.0f, down = 1.0f, up = 1.0f;
            x.template typed<kQ>([&](auto type) {
                using Q = decltype(type);
                Q raw[DP / 16];
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) raw[c] = static_cast<const Q*>(a.d.q)[at + min(max(c0 + 16 * c, 0), a.d.d - 1)];
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) y[c] = qrow < now.n && (unsigned)(c0 + 16 * c) < (unsigned)a.d.d ? (float)raw[c] : 0.0f;
            });
            if (kQ > 1) {
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) top = fmaxf(top, fabsf(y[c]));
                X::level(__int_as_float(group_reduce<16>(__float_as_int(top), MaxF32{})), down, up);
            }
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                float rest = copysignf(down, by) * y[c];
#pragma unroll
                for (int q = 0; q < kQ; ++q) {
                    const T v = (T)rest;
                    rest -= (float)v;
                    s.few.q[q][qrow * kStride + qc + 16 * c] = __builtin_bit_cast(short, v);
                }
            }
            if (qc == 0) s.q_scale[qrow] = fabsf(by) * up;
        }
        __syncthreads();
        // never 0, so that it takes a masked score, minus infinity, for what it is
        const float factor[1] = {fmaxf(s.q_scale[x.column], 1.17549435e-38f)};
        if (t0 >= k1) {                                       // no tile for this wavefront
            const unsigned place = x.place_of(then, then_t0, then_entry, valid);
            x.fetch(a.d.k_cache, then, place, kr);
            x.fetch(a.d.v_cache, then, place, vr);
        }
        v4f o[1][X::kBlocks];
#pragma unroll
        for (int i = 0; i < X::kBlocks; ++i) o[0][i] = v4f{0, 0, 0, 0};
        float m[1] = {-INFINITY}, l[1] = {0.0f};
        for (; t0 < k1; t0 += kStep) {
            unsigned long next_valid;
            const bool more = t0 + kStep < k1;
            const SharedPiece& of = more ? now : then;
            const unsigned next = x.place_of(of, more ? t0 + kStep : then_t0, more ? entry : then_entry, next_valid);
            entry = x.entry_of(now, t0 + 2 * kStep);
            x.stage(tile, kr, valid);
            x.fetch(a.d.k_cache, of, next, kr);
            v4f sc[1][2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                sc[0][blk] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int step = 0; step < X::kSteps; ++step) {
                    const v8s ka = x.keys_of(tile, blk, step);
#pragma unroll
                    for (int q = kQ - 1; q >= 0; --q) sc[0][blk] = Mma<T>::mma(ka, *reinterpret_cast<const v8s*>(s.few.q[q] + x.column * kStride + step * 32 + x.j * 8), sc[0][blk]);
                }
            }
            v8s p[1][kP];
            x.template weigh<1, kP>(sc, valid, factor, m, l, p, o);
            x.stage(tile, vr, valid);
            x.fetch(a.d.v_cache, of, next, vr);
#pragma unroll
            for (int blk = 0; blk < X::kBlocks; ++blk) {
                const v8s va = x.values_of(tile, blk);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q) o[0][blk] = Mma<T>::mma(va, p[0][q], o[0][blk]);
            }
            valid = next_valid;
        }
        // the wavefronts' results as one
        l[0] = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l[0]), AddF32{}), AddF32{}));
        if (x.j == 0) { s.m[wave][x.column] = m[0]; s.l[wave][x.column] = l[0]; }
        __syncthreads();                                      // also: no tile is read any more
        {
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s.m[w][x.column]);
            const float mine = __builtin_amdgcn_exp2f(m[0] - (top == -INFINITY ? 0.0f : top) - X::kLift);
#pragma unroll
            for (int blk = 0; blk < X::kBlocks; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) s.o[wave][x.column][blk * 16 + x.j * 4 + i] = o[0][blk][i] * mine;
        }
        __syncthreads();
        if (qrow < now.n) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s.m[w][qrow]);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += s.l[w][qrow] * __builtin_amdgcn_exp2f(s.m[w][qrow] - base - X::kLift);
            x.leave(now, qrow, Run::part_of(a, 0, run.worker, max(now.slot, 0)), [&](auto put) {
                for (int c = qc * 4; c < a.d.d; c += 64) {
                    v4f y{0, 0, 0, 0};
#pragma unroll
                    for (int w = 0; w < W; ++w) y += *reinterpret_cast<const v4f*>(&s.o[w][qrow][part * a.d.d + c]);
                    put(c, y);
                }
            }, top, sum);
        }
        if (then.table < 0) break;
        now = then;
        t0 = then_t0;
        entry2 = then_entry2;
    }
}

// A run through another list: 128 positions at a time in LDS, for all wavefronts' queries.  S: sixteens of a wavefront; W: wavefronts (eight: four bring
// keys and four values).
template <typename C, typename T, int DP, int kQ, int kP, int S, int W>
__device__ __forceinline__ void run_many(const SharedArgs& a, Run run, SharedLds<DP, kQ, W>& s)
{
    using X = Tiles<C, T, DP>;
    constexpr bool kBoth = W == kPagedWaves;
    const X x(a);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qrow = tid / 16 % 16, qc = tid & 15;
    for (SharedPiece now = run.next(a); now.table >= 0; now = run.next(a)) {
        const int k1 = now.k1;
        // wavefronts that have queries of their own, and which of them (and which part of the positions) this one has
        const int apart = now.n <= 16 * S ? 1 : now.n <= 32 * S ? 2 : W == 4 || now.n <= 64 * S ? 4 : W, mine = wave % apart, part = wave / apart, parts = W / apart;
        const int brings = wave % kPagedWaves;
        const bool keys = wave < kPagedWaves;
        int t0 = now.k0 + brings * kTile;
        int entry = x.entry_of(now, t0), entry2 = x.entry_of(now, t0 + kUnit);
        v4u kr[X::kLoads], vr[kBoth ? X::kLoads : 1];
        unsigned long valid;
        auto fetch = [&](unsigned place) {
            x.fetch(keys ? a.d.k_cache : a.d.v_cache, now, place, kr);
            if constexpr (kBoth) x.fetch(a.d.v_cache, now, place, vr);
        };
        fetch(x.place_of(now, t0, entry, valid));
        // queries, as operands: a lane has those of column `column`, 8 elements of each step
        v8s qb[S][kQ][X::kSteps];
        float factor[S];
        x.template typed<kQ>([&](auto type) {
            using Q = decltype(type);
            typedef Q Run8 __attribute__((ext_vector_type(8)));
            // d is a multiple of 16: 8 elements are there, or none
            Run8 raw[S][X::kSteps];
            auto each = [&](auto load) {
#pragma unroll
                for (int t = 0; t < S; ++t) {
                    const int row = (mine * S + t) * 16 + x.column;
                    const Q* from = static_cast<const Q*>(a.d.q) + x.query_of(now, min(row, now.n - 1));
                    const int c0 = x.j * 8 - x.part_of(now, min(row, now.n - 1)) * a.d.d;   // the lane's first element of its own head
#pragma unroll
                    for (int step = 0; step < X::kSteps; ++step) {
                        const int c = c0 + step * 32;
                        load(t, step, from + min(max(c, 0), a.d.d - 8), row < now.n && (unsigned)c < (unsigned)a.d.d);
                    }
                }
            };
            if (a.whole_queries) each([&](int t, int step, const Q* from, bool) { raw[t][step] = *reinterpret_cast<const Run8*>(from); });
            else each([&](int t, int step, const Q* from, bool) {
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[t][step][e] = from[e];
            });
            each([&](int t, int step, const Q*, bool there) {
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[t][step][e] = there ? raw[t][step][e] : (Q)0.0f;
            });
#pragma unroll
            for (int t = 0; t < S; ++t) {
                const float by = x.scale_of(now, min((mine * S + t) * 16 + x.column, now.n - 1));
                float top = 0.0f, down = 1.0f, up = 1.0f;
                if constexpr (kQ > 1) {
#pragma unroll
                    for (int step = 0; step < X::kSteps; ++step)
#pragma unroll
                        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)raw[t][step][e]));
                    X::level(__int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(top), MaxF32{}), MaxF32{})), down, up);
                }
                const float signed_down = copysignf(down, by);
#pragma unroll
                for (int step = 0; step < X::kSteps; ++step)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float rest = signed_down * (float)raw[t][step][e];
#pragma unroll
                        for (int q = 0; q < kQ; ++q) {
                            const T v = (T)rest;
                            rest -= (float)v;
                            qb[t][q][step][e] = __builtin_bit_cast(short, v);
                        }
                    }
                factor[t] = fmaxf(fabsf(by) * up, 1.17549435e-38f);   // never 0, so that it takes a masked score, minus infinity, for what it is
            }
        });
        v4f o[S][X::kBlocks];
        float m[S], l[S];
#pragma unroll
        for (int t = 0; t < S; ++t) {
#pragma unroll
            for (int i = 0; i < X::kBlocks; ++i) o[t][i] = v4f{0, 0, 0, 0};
            m[t] = -INFINITY;
            l[t] = 0.0f;
        }
        // 128 positions from registers into a buffer, and the next ones on their way
        auto bring = [&](auto& to, unsigned long (&there)[kPagedWaves]) {
            x.stage(keys ? to.k[brings] : to.v[brings], kr, valid);
            if constexpr (kBoth) x.stage(to.v[brings], vr, valid);
            if (keys && x.lane == 0) there[brings] = valid;
            const unsigned place = x.place_of(now, t0 + kUnit, entry2, valid);
            t0 += kUnit;
            entry2 = x.entry_of(now, t0 + kUnit);
            fetch(place);                                     // (behind the last: the first page)
        };
        constexpr bool kTwo = SharedLds<DP, kQ, W>::kBuffers > 1;
        if (kTwo) {
            __syncthreads();                                  // the piece before is done with LDS
            bring(s.many[0], s.valid[0]);
        }
        int buffer = 0;
        for (int u0 = now.k0; u0 < k1; u0 += kUnit, buffer ^= kTwo) {
            __syncthreads();                                  // the positions before are done with, and (of two buffers) these are there
            if (!kTwo) {
                bring(s.many[0], s.valid[0]);
                __syncthreads();
            } else if (u0 + kUnit < k1) {
                bring(s.many[buffer ^ 1], s.valid[buffer ^ 1]);
            }
            const auto& many = s.many[buffer];
            const int tiles = min((k1 - u0 + kTile - 1) / kTile, kPagedWaves);
#pragma unroll 1
            for (int n = part; n < tiles; n += parts) {
                const unsigned long bits = s.valid[buffer][n];         // uniform, which the compiler cannot know
                const unsigned long there = (unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)bits);
                v4f sc[S][2];
#pragma unroll
                for (int t = 0; t < S; ++t) sc[t][0] = sc[t][1] = v4f{0, 0, 0, 0};
                // reads run ahead of the products that use them, which the compiler by itself puts next to one another
                constexpr int kFrags = 2 * X::kSteps, kAhead = 3;
                v8s ka[kFrags];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) ka[i] = x.keys_of(many.k[n], i % 2, i / 2);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < kFrags; ++i) {
                    if (i + kAhead < kFrags) ka[i + kAhead] = x.keys_of(many.k[n], (i + kAhead) % 2, (i + kAhead) / 2);
#pragma unroll
                    for (int t = 0; t < S; ++t)
#pragma unroll
                        for (int q = kQ - 1; q >= 0; --q) sc[t][i % 2] = Mma<T>::mma(ka[i], qb[t][q][i / 2], sc[t][i % 2]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                v8s p[S][kP];
                x.template weigh<S, kP>(sc, there, factor, m, l, p, o);
                constexpr int kBehind = 2;
                v8s va[X::kBlocks];
#pragma unroll
                for (int blk = 0; blk < kBehind; ++blk) va[blk] = x.values_of(many.v[n], blk);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int blk = 0; blk < X::kBlocks; ++blk) {
                    if (blk + kBehind < X::kBlocks) va[blk + kBehind] = x.values_of(many.v[n], blk + kBehind);
#pragma unroll
                    for (int q = kP - 1; q >= 0; --q)
#pragma unroll
                        for (int t = 0; t < S; ++t) o[t][blk] = Mma<T>::mma(va[blk], p[t][q], o[t][blk]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        // the wavefronts' results as one, sixteen queries of each at a time
        const long at = Run::part_of(a, run.list, run.worker, max(now.slot, 0));
        if (parts == 1) {                                     // each has its own: a lane has four elements of each block of its query
#pragma unroll
            for (int t = 0; t < S; ++t) {
                const float sum = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l[t]), AddF32{}), AddF32{})), down = __builtin_amdgcn_exp2f(-X::kLift);
                const int row = (mine * S + t) * 16 + x.column;
                if (row < now.n) {
                    const int own = x.part_of(now, row) * a.d.d;
                    x.leave(now, row, at, [&](auto put) {
#pragma unroll
                        for (int blk = 0; blk < X::kBlocks; ++blk)
                            if ((unsigned)(blk * 16 - own) < (unsigned)a.d.d) put(blk * 16 - own + x.j * 4, o[t][blk] * down);
                    }, m[t], sum * down);
                }
            }
            continue;
        }
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const float sum_l = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l[t]), AddF32{}), AddF32{}));
            __syncthreads();
            if (x.j == 0) { s.m[wave][x.column] = m[t]; s.l[wave][x.column] = sum_l; }
            __syncthreads();
            float top = -INFINITY;
            for (int w = mine; w < W; w += apart) top = fmaxf(top, s.m[w][x.column]);
            const float shrink = __builtin_amdgcn_exp2f(m[t] - (top == -INFINITY ? 0.0f : top) - X::kLift);
#pragma unroll
            for (int blk = 0; blk < X::kBlocks; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) s.o[wave][x.column][blk * 16 + x.j * 4 + i] = o[t][blk][i] * shrink;
            __syncthreads();
            for (int of = tid / 256; of < apart; of += W / 4) {   // sixteen queries are 256 threads' work
                const int row = (of * S + t) * 16 + qrow;
                if (row >= now.n) break;
                float top = -INFINITY, sum = 0.0f;
                for (int w = of; w < W; w += apart) top = fmaxf(top, s.m[w][qrow]);
                const float base = top == -INFINITY ? 0.0f : top;
                for (int w = of; w < W; w += apart) sum += s.l[w][qrow] * __builtin_amdgcn_exp2f(s.m[w][qrow] - base - X::kLift);
                const int own = x.part_of(now, row) * a.d.d;
                x.leave(now, row, at, [&](auto put) {
                    for (int c = qc * 4; c < a.d.d; c += 64) {
                        v4f y{0, 0, 0, 0};
                        for (int w = of; w < W; w += apart) y += *reinterpret_cast<const v4f*>(&s.o[w][qrow][own + c]);
                        put(c, y);
                    }
                }, top, sum);
            }
        }
    }
}

// The first two lists.  C, T, DP, kQ, kP: as in nm_paged_attention.
template <typename C, typename T, int DP, int kQ, int kP>
__global__ __launch_bounds__(kPagedThreads, DP <= 128 ? 2 : 1) void shared_attention_kernel(SharedArgs a)
{
    __shared__ __attribute__((aligned(16))) SharedLds<DP, kQ, kPagedWaves> s;
    // workgroup i runs on XCD i mod 8: neighbouring runs are one XCD's, and each XCD has its share of either list
    const SharedHead head = *a.head;
    const int xcd = blockIdx.x % 8, i = blockIdx.x / 8, second = (head.workers[1] + 7) / 8, first = (head.workers[0] + 7) / 8;
    if (i < second) {
        const int worker = xcd * second + i;
        if (worker < head.workers[1]) run_many<C, T, DP, kQ, kP, shared_sets(1, DP, kQ), kPagedWaves>(a, Run(a, head, 1, worker), s);
    } else if (i - second < first) {
        const int worker = xcd * first + i - second;
        if (worker < head.workers[0]) run_few<C, T, DP, kQ, kP>(a, Run(a, head, 0, worker), s);
    }
}

// The third: a workgroup of eight wavefronts to a CU.  (Launched wherever a group could be that large: 4.5 us where none is.)
template <typename C, typename T, int DP, int kQ, int kP>
__global__ __launch_bounds__(64 * shared_waves(2), 2) void shared_prefix_kernel(SharedArgs a)
{
    __shared__ __attribute__((aligned(16))) SharedLds<DP, kQ, shared_waves(2)> s;
    const SharedHead head = *a.head;
    const int each = (head.workers[2] + 7) / 8, worker = (int)(blockIdx.x % 8) * each + (int)(blockIdx.x / 8);
    if ((int)(blockIdx.x / 8) < each && worker < head.workers[2]) run_many<C, T, DP, kQ, kP, shared_sets(2, DP, kQ), shared_waves(2)>(a, Run(a, head, 2, worker), s);
}

// Joins what a query has: its group's prefix and its row's own positions, each whole or in pieces.  A workgroup to a query: a thread to a piece finds the piece's
// place and weight, then lanes of four elements add every so-manieth piece's output, whose first loads are under way before the weights are there.  2048 queries
// of 128 of 36 pieces (47 MB fetched, at 4.4 TB/s) 10.7 us, 96 rows of 32 heads, of 8 pieces, 11.0; where threads found the weights of their pieces as they added them 10.7 and 12.6.
__global__ __launch_bounds__(kPagedThreads) void shared_join_kernel(SharedArgs a)
{
    constexpr int kAhead = 4;
    __shared__ __attribute__((aligned(16))) float s_o[kPagedThreads * 4];
    __shared__ const float* s_from[kPagedThreads];
    __shared__ float s_by[kPagedThreads], s_top[kPagedWaves], s_sum[kPagedWaves];
    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, b = blockIdx.y, h = blockIdx.x, g = (int)quotient(h, a.by_group), in_group = h - g * a.group;
    const int lead = a.lead[b];
    const long bh = (long)b * d.hq + h, all = (long)d.B * d.hq;
    // [0] the prefix, [1] the row's own positions; and the query's number in the range
    int4 info[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
    int nth[2] = {0, in_group & ((1 << a.tile[0]) - 1)};
    info[1] = a.info[all + bh - nth[1]];
    if (info[1].x < 0) return;
    if (lead >= 0) {
        const int i = (b - lead) * a.group + in_group;
        nth[0] = i & ((1 << a.tile[2]) - 1);
        const int i0 = i - nth[0], row = (int)quotient(i0, a.by_group);
        info[0] = a.info[(long)(lead + row) * d.hq + g * a.group + i0 - row * a.group];
    }
    const int used = info[0].x + info[1].x;
    const int lanes = d.d / 4, at_once = kPagedThreads / lanes, mine = tid / lanes, c = tid % lanes * 4;
    float m = -INFINITY, l = 0.0f;
    v4f x{0, 0, 0, 0};
    for (int k0 = 0; k0 < used; k0 += kPagedThreads) {
        const int n = min(used - k0, kPagedThreads), k = k0 + tid;
        float2 ml{-INFINITY, 0.0f};
        if (tid < n) {
            const bool own = k >= info[0].x;
            const int4 of = own ? info[1] : info[0];
            const int i = own ? k - info[0].x : k;
            const bool whole = of.y < 0;
            const long part = whole ? own * all + bh : (i ? of.z + (long)(i - 1) * of.w : of.y) + (own ? nth[1] : nth[0]);
            ml = (whole ? a.whole_ml : a.part_ml)[part];
            s_from[tid] = (whole ? a.whole_o : a.part_o) + part * d.d;
        }
        const float most = __int_as_float(group_reduce<64>(__float_as_int(ml.x), MaxF32{}));
        if (tid % 64 == 0) s_top[tid / 64] = most;
        __syncthreads();
        v4f y[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (mine < at_once && mine + e * at_once < n) y[e] = *reinterpret_cast<const v4f*>(s_from[mine + e * at_once] + c);
        float top = m;
        for (int i = 0; i < kPagedWaves; ++i) top = fmaxf(top, s_top[i]);
        const float base = top == -INFINITY ? 0.0f : top, shrink = __builtin_amdgcn_exp2f(m - base), by = __builtin_amdgcn_exp2f(ml.x - base);
        l = l * shrink + ml.y * by;
        s_by[tid] = by;
        m = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= shrink;
        if (mine < at_once)
            for (int j = mine;;) {
#pragma unroll
                for (int e = 0; e < kAhead; ++e)
                    if (j + e * at_once < n)
                        for (int i = 0; i < 4; ++i) x[i] += y[e][i] * s_by[j + e * at_once];
                j += kAhead * at_once;
                if (j >= n) break;
#pragma unroll
                for (int e = 0; e < kAhead; ++e)
                    if (j + e * at_once < n) y[e] = *reinterpret_cast<const v4f*>(s_from[j + e * at_once] + c);
            }
        if (k0 + kPagedThreads < used) __syncthreads();
    }
    const float part_sum = group_sum<64>(l);
    if (tid % 64 == 0) s_sum[tid / 64] = part_sum;
    if (mine < at_once) *reinterpret_cast<v4f*>(&s_o[mine * d.d + c]) = x;
    __syncthreads();
    const float top = m;
    float sum = 0.0f, v = 0.0f;
    for (int i = 0; i < kPagedWaves; ++i) sum += s_sum[i];
    if (tid < d.d)
        for (int i = 0; i < at_once; ++i) v += s_o[i * d.d + tid];
    const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * (d.cache_dtype == NM_DT_I8 ? d.v_scale[h / a.own] : 1.0f);
    if (tid < d.d) store1(d.out, d.out_dtype, b * d.out_stride + (long)h * d.d + tid, v * by, d.out_inv_scale);
    if (tid == 0 && d.lse) d.lse[bh] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <typename C, typename T, int DP, int kQ, int kP>
static void launch_shared(const SharedArgs& a, hipStream_t s)
{
    // either list's workers rounded up to one for every XCD
    queue_kernel(shared_attention_kernel<C, T, DP, kQ, kP>, dim3((a.workers + 7) / 8 * 8 + 8), dim3(kPagedThreads), 0, s, a);
    if (a.G && (long)a.d.B * a.group > 1 << a.tile[1]) queue_kernel(shared_prefix_kernel<C, T, DP, kQ, kP>, dim3(a.last), dim3(64 * shared_waves(2)), 0, s, a);
}
template <typename C, typename T, int DP>
static void launch_shared(const SharedArgs& a, bool own, hipStream_t s)
{
    own ? launch_shared<C, T, DP, 1, 2>(a, s) : launch_shared<C, T, DP, 3, 3>(a, s);
}
// One term of a query where the matrix instructions' type is its own, and two of the weights where the result has 16 bits or fewer.
static bool one_term(const nm_paged_desc& d)
{
    const bool f16_cache = d.cache_dtype == NM_DT_F16 || (d.cache_dtype == NM_DT_I8 && d.q_dtype == NM_DT_F16);
    return d.q_dtype == (f16_cache ? NM_DT_F16 : NM_DT_BF16) && d.out_dtype != NM_DT_F32;
}
template <typename C, typename T>
static void launch_shared(const SharedArgs& a, hipStream_t s)
{
    const bool own = one_term(a.d);
    const int width = paged_width(a.width);
    if (width == 64) launch_shared<C, T, 64>(a, own, s);
    else if (width == 128) launch_shared<C, T, 128>(a, own, s);
    else launch_shared<C, T, 256>(a, own, s);
}

// Takes bytes of the workspace in turn; with a NULL base it counts.
struct Carve {
    char* base;
    size_t used = 0;
    template <typename P> void take(P*& p, size_t n)
    {
        used = (used + 15) / 16 * 16;
        p = base ? reinterpret_cast<P*>(base + used) : nullptr;
        used += n * sizeof(P);
    }
};

// What does not depend on pointers.  *alone: no row is long enough to be divided, and nm_paged_attention takes them one by one.
static int32_t plan_shared(const nm_shared_desc* d, SharedArgs* a, void* ws, size_t* bytes, bool* alone, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    bool divided;
    const int32_t rc = check_paged_shape(&d->p, &divided, what);
    if (rc) return rc;
    if (d->G < 0) return fail(NM_ERR_INVALID_ARG, "%s: G is negative", what);
    if (d->p.window) return fail(NM_ERR_UNSUPPORTED, "%s: a window", what);
    if (d->p.B > kSharedMost || d->G > kSharedMost) return fail(NM_ERR_UNSUPPORTED, "%s: B %d or G %d > %d", what, d->p.B, d->G, kSharedMost);
    // rows that are not divided, no groups, or few units in all
    const long most = (long)d->p.B * d->p.hk * ((((long)d->p.max_pages << page_shift(d->p.page_size)) + kUnit - 1) / kUnit);
    *alone = !divided || d->G == 0 || most <= kFewUnits;
    *a = SharedArgs{};
    a->d = d->p;
    a->G = d->G;
    a->group_start = d->group_start;
    a->shared = d->shared;
    a->shift = page_shift(d->p.page_size);
    a->own = d->p.hq / d->p.hk;
    // Heads of int8 as one, whole lines of 128 bytes, where their queries, of a group's rows (of so many as the groups have among them), are still few
    // (16 groups of 8 rows, 16 heads of 64: 64 us, 78.6 apart); more would double the products.
    a->pack = 1;
    if (d->p.cache_dtype == NM_DT_I8 && d->p.head_stride == d->p.d)
        while (2 * a->pack * d->p.d <= 128 && d->p.hk % (2 * a->pack) == 0 && (d->G ? (d->p.B + d->G - 1) / d->G : 1) * a->own * 2 * a->pack <= shared_tile(0, 128, 1)) a->pack *= 2;
    a->heads = d->p.hk / a->pack;
    a->width = d->p.d * a->pack;
    a->group = a->own * a->pack;
    a->by_group = fast_div(a->group);
    const int width = paged_width(a->width);
    for (int list = 0; list < kLists; ++list) a->tile[list] = __builtin_ctz(shared_tile(list, width, one_term(d->p) ? 1 : 3));   // powers of two
    a->workers = 256 * (width <= 128 ? 2 : 1);
    a->whole_queries = aligned_rows(d->p.q, d->p.q_stride, d->p.q_dtype, 8);
    a->last = 256;
    const size_t parts = (size_t)a->workers * 2 * ((1 << a->tile[0]) + (1 << a->tile[1])) + ((size_t)a->last * 2 << a->tile[2]), queries = (size_t)d->p.B * d->p.hq;
    Carve c{static_cast<char*>(ws)};
    c.take(a->head, 1);
    c.take(a->ent, (size_t)d->G + d->p.B);
    c.take(a->info, 2 * queries);
    c.take(a->before, kLists * a->workers);
    c.take(a->first, kLists * a->workers);
    c.take(a->lead, d->p.B);
    c.take(a->part_ml, parts);
    c.take(a->whole_ml, 2 * queries);
    c.take(a->part_o, parts * d->p.d);
    c.take(a->whole_o, 2 * queries * d->p.d);
    *bytes = c.used;
    return *alone ? nm_paged_attention_workspace(&d->p, bytes) : NM_OK;
}

}  // namespace nm

using namespace nm;

extern "C" {

int32_t nm_shared_attention_workspace(const nm_shared_desc* d, size_t* bytes)
{
    SharedArgs a;
    size_t n;
    bool alone;
    const int32_t rc = plan_shared(d, &a, nullptr, &n, &alone, "nm_shared_attention_workspace");
    if (rc) return rc;
    if (!bytes) return fail(NM_ERR_INVALID_ARG, "nm_shared_attention_workspace: bytes is NULL");
    *bytes = n;
    return NM_OK;
}

int32_t nm_shared_attention(const nm_shared_desc* desc, void* ws, size_t ws_bytes, void* stream)
{
    SharedArgs a;
    size_t need;
    bool alone;
    int32_t rc = plan_shared(desc, &a, ws, &need, &alone, "nm_shared_attention");
    if (rc) return rc;
    const nm_paged_desc& d = desc->p;
    if ((rc = check_paged(&d, "nm_shared_attention"))) return rc;
    if (d.B == 0) return NM_OK;
    if (desc->G && (!desc->group_start || !desc->shared)) return fail(NM_ERR_INVALID_ARG, "nm_shared_attention: group_start or shared is NULL");
    if (begins_as(d.out, {desc->group_start, desc->shared}) || begins_as(d.lse, {desc->group_start, desc->shared}))
        return fail(NM_ERR_INVALID_ARG, "nm_shared_attention: out or lse is group_start or shared");
    if (alone && !need) return nm_paged_attention(&d, nullptr, 0, stream);
    if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_shared_attention: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_shared_attention: workspace must be 256-byte aligned");
    if (alone) return nm_paged_attention(&d, ws, ws_bytes, stream);
    const hipStream_t s = (hipStream_t)stream;
    queue_kernel(shared_plan_kernel, dim3(1), dim3(kPlanners), 0, s, a);
    if (d.cache_dtype == NM_DT_BF16) launch_shared<bf16, bf16>(a, s);
    else if (d.cache_dtype == NM_DT_F16) launch_shared<f16, f16>(a, s);
    else if (d.q_dtype == NM_DT_F16) launch_shared<int8_t, f16>(a, s);
    else launch_shared<int8_t, bf16>(a, s);
    if ((rc = check_hip(hipGetLastError(), "nm_shared_attention launch"))) return rc;
    queue_kernel(shared_join_kernel, dim3(d.hq, d.B), dim3(kPagedThreads), 0, s, a);
    return check_hip(hipGetLastError(), "nm_shared_attention launch");
}

}  // extern "C"
