// Attention of one new token per row over a paged cache, where groups of rows share a prefix (nm_shared_attention).
//
// The rows' own positions are nm_paged_attention's work: every key and value once, bound by memory.  A group's prefix is read once for all its
// rows: for one key head the queries of all of them, rows times heads, are as many columns of the same matrix products.  A piece
// of work is a range of positions with up to kQueries columns; a group with more goes over its prefix again, side by side on one XCD, so
// that its L2 serves the others.  Softmax over both ranges: each piece leaves its maximum, sum and output, and a last kernel joins a row's.
//   A first kernel of one workgroup makes the list: of each group (its prefix, all its rows' queries) and each row (its own positions, its queries) the
// cost, and where in their sequence each workgroup of the second begins.  As in nm_paged_attention a fixed number of workgroups share all of it evenly, whatever
// the lengths are, and a run's first and last piece may be parts of a range.  Tiles, operand layouts and precision are that kernel's too.
#include "nm_paged_parts.h"

namespace nm {

constexpr int kSharedMost = NM_PLAN_MAX_REQUESTS;     // rows, groups
constexpr int kSharePrefix = kUnit;                   // shorter prefixes are every row's own
constexpr int kPlanners = 1024;

// Columns of a piece in sixteens.
constexpr int shared_sets(int dp) { return dp <= 128 ? 2 : 1; }

struct SharedHead { long each, more; int workers, pad; };   // how the cost is divided
struct SharedArgs {
    nm_paged_desc d;
    int G;
    const int32_t* group_start;
    const int32_t* shared;
    int shift, group, sets;      // log2 of page_size, query heads of a key head, sixteens of columns of a piece
    int workers;                 // at most
    SharedHead* head;
    int4* ent;                   // [G + B]: a group: first row, rows, the row whose table it goes by, positions; a row: itself, 1, its own first position, its length
    int* lead;                   // [B]: first row of the group whose prefix the row shares, -1: none
    long* before;                // [workers]: cost of the entities in front of a worker's first
    int* first;                  // [workers]: a worker's first entity
    int4* info;                  // [2, B, hq], by a tile's first query: how many pieces it has (0: none, -1: the result is there), the first's worker and slot (-1: whole)
    float2* part_ml;             // [workers, 2, 16 sets]: maximum (of scores in units of log 2) and sum
    float* part_o;               // [workers, 2, 16 sets, d]: not yet divided by the sum
    float2* whole_ml;            // [2, B, hq]
    float* whole_o;              // [2, B, hq, d]
};

// What an entity is, and what it costs.
struct Entity {
    int row0, table, k0, k1, queries, tiles, units, unit, extra;
    __device__ __forceinline__ Entity(const SharedArgs& a, int e)
    {
        const int4 x = a.ent[e];
        const bool prefix = e < a.G;
        row0 = x.x;
        table = prefix ? x.z : x.x;
        k0 = prefix ? 0 : x.z;
        k1 = x.w;
        queries = prefix && k1 <= 0 ? 0 : x.y * a.group;
        tiles = (queries + 16 * a.sets - 1) / (16 * a.sets);
        units = (k1 - k0 + kUnit - 1) / kUnit;
        // a unit's keys and values, and its columns; beginning and ending a range
        unit = 4 + min((queries + 15) / 16, a.sets);
        extra = 2 * unit;
    }
    __device__ __forceinline__ long cost() const { return (long)units * unit + extra; }               // of a key head's tile
    __device__ __forceinline__ long all(const SharedArgs& a) const { return cost() * a.d.hk * tiles; }
};
__device__ __forceinline__ int most_unit(const SharedArgs& a) { return 4 + a.sets; }

__global__ __launch_bounds__(kPlanners) void shared_plan_kernel(SharedArgs a)
{
    __shared__ long s_before[2 * kSharedMost + 1], s_wave[kPlanners / 64];
    __shared__ int s_start[kSharedMost + 1], s_lead[kSharedMost];
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
    __threadfence_block();
    __syncthreads();
    // a thread's run of entities, then the threads'
    const int n = a.G + B, per = (n + kPlanners - 1) / kPlanners, e0 = min(tid * per, n), e1 = min(e0 + per, n);
    long mine = 0;
    for (int e = e0; e < e1; ++e) mine += Entity(a, e).all(a);
    long in = mine;
    for (int step = 1; step < 64; step <<= 1) {
        const long t = __shfl_up(in, step);
        if (lane >= step) in += t;
    }
    if (lane == 63) s_wave[tid >> 6] = in;
    __syncthreads();
    long front = in - mine, all = 0;
    for (int w = 0; w < kPlanners / 64; ++w) {
        if (w < tid >> 6) front += s_wave[w];
        all += s_wave[w];
    }
    for (int e = e0; e < e1; ++e) {
        s_before[e] = front;
        front += Entity(a, e).all(a);
    }
    if (tid == 0) s_before[n] = all;
    __syncthreads();
    // no share is smaller than a unit, so that every worker between a range's first and last has some of it
    const int workers = (int)max(1l, min((long)a.workers, all / most_unit(a)));
    const Shares shares(all, workers);
    if (tid == 0) *a.head = SharedHead{shares.each, shares.more, workers, 0};
    for (int w = tid; w < workers; w += kPlanners) {
        const long x = shares.begin(w);
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (s_before[mid] <= x) lo = mid; else hi = mid;
        }
        a.first[w] = lo;
        a.before[w] = s_before[lo];
    }
}

// What a workgroup has of a range: positions [k0, k1) by the table of row `table` (-1: none) for key head g and the n queries from number i0 on of the rows from
// row0 on; slot: where its part goes, -1 where it is the whole range; prefix: of a group.
struct SharedPiece { int table, row0, g, i0, n, k0, k1, slot, prefix, done; };

// C, T, DP, kQ, kP: as in nm_paged_attention; N: sixteens of columns.
template <typename C, typename T, int DP, int kQ, int kP, int N>
__global__ __launch_bounds__(kPagedThreads, DP <= 128 ? 2 : 1) void shared_attention_kernel(SharedArgs a)
{
    constexpr int W = kPagedWaves;
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
    __shared__ __attribute__((aligned(16))) short s_q[kQ][16 * N * kStride];
    __shared__ float s_qscale[16 * N], s_m[W][16], s_l[W][16];

    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int column = lane & 15, j = lane >> 4;              // head (and row of an operand), lane group
    const int row_piece = lane % kRowPieces, row_first = lane / kRowPieces;
    constexpr bool kPairs = kRowPieces == 4;
    auto position_of = [](int group, int i) { return kPairs ? (group >> 1) * 2 * kLoads + 2 * i + (group & 1) : group * kLoads + i; };
    const int my_position = position_of(row_first, lane % kLoads);
    short* tile = s.tile[wave];
    const bool in_row = row_piece * kPer16 < d.d;

    // workgroup i runs on XCD i mod 8: neighbouring runs are one XCD's
    const SharedHead head = *a.head;
    const int each_xcd = (head.workers + 7) / 8, worker = (int)(blockIdx.x % 8) * each_xcd + (int)(blockIdx.x / 8);
    if ((int)(blockIdx.x / 8) >= each_xcd || worker >= head.workers) return;
    const Shares shares(head.each, head.more, 0);
    const long first = shares.begin(worker), u1 = shares.begin(worker + 1);
    long u = first, before = a.before[worker];
    int e = a.first[worker];

    auto advance = [&]() -> SharedPiece {
        while (u < u1) {
            const Entity x(a, e);
            const long cost = x.cost(), all = x.all(a);
            if (u >= before + all) {                          // the next entity
                before += all;
                ++e;
                continue;
            }
            const int r = (int)((u - before) / cost);
            const long begin = before + r * cost, end = min(u1, begin + cost);
            // a range's cost comes first, then its units
            auto units_at = [&](long at) { return (int)min((max(at - begin - x.extra, 0l) + x.unit - 1) / x.unit, (long)x.units); };
            const int from = units_at(u), to = units_at(end);
            const bool starts = u == begin;
            u = end;
            if (x.units ? from == to : !starts) continue;     // another workgroup has what there is of it
            SharedPiece n;
            n.table = x.table;
            n.row0 = x.row0;
            n.g = r / x.tiles;
            n.i0 = r % x.tiles * 16 * N;
            n.n = min(x.queries - n.i0, 16 * N);
            n.k0 = x.k0 + from * kUnit;
            n.k1 = (int)min((long)x.k0 + (long)to * kUnit, (long)x.k1);
            n.slot = from == 0 && to == x.units ? -1 : begin > first;
            n.prefix = e < a.G;
            n.done = !n.prefix && x.k0 == 0 && n.slot < 0;
            if (from == 0 && tid == 0) {
                const int count = n.done ? -1 : x.units ? (int)(shares.owner(begin + x.extra + (long)(x.units - 1) * x.unit) - worker) + 1 : 0;
                a.info[((long)!n.prefix * d.B + x.row0 + n.i0 / a.group) * d.hq + n.g * a.group + n.i0 % a.group] = make_int4(count, worker, n.slot, 0);
            }
            return n;
        }
        return SharedPiece{-1, 0, 0, 0, 0, 0, 0, -1, 0, 0};
    };
    // A tile's places: a lane has one position's distance into the cache in 16 bytes, 0 where it takes no part.  Loads are not
    // conditional: a lane of no part reads the first page, and zeros are put in the place of what it read.
    auto entry_of = [&](const SharedPiece& n, int t0) {
        const bool some = n.table >= 0 && n.k1 > 0;
        const int* table = d.max_pages && some ? d.block_table + n.table * d.table_stride : reinterpret_cast<const int*>(g_zero_line);
        return table[some ? min(t0 + my_position, n.k1 - 1) >> a.shift : 0];
    };
    auto place_of = [&](const SharedPiece& n, int t0, int entry, unsigned long& valid) -> unsigned {
        const int k = t0 + my_position;
        const bool ok = k < n.k1 && entry >= 0 && entry < d.num_pages;
        valid = __ballot(ok);
        return ok ? (unsigned)(((long)entry * d.page_stride + (long)(k & (d.page_size - 1)) * d.slot_stride) / kPer16) : 0u;
    };
    const int lane_bytes = in_row ? row_piece * 16 : 0;
    auto fetch = [&](const void* cache, const SharedPiece& n, unsigned place, v4u (&to)[kLoads]) {
        const char* base = d.num_pages ? static_cast<const char*>(cache) + (long)n.g * d.head_stride * sizeof(C) + lane_bytes : reinterpret_cast<const char*>(g_zero_line);
        fetch_rows<kLoads>(base, place, to, std::make_integer_sequence<int, kLoads>{});
        __builtin_amdgcn_sched_barrier(0);                    // the order of the loads is what is waited for
    };
    auto stage = [&](const v4u (&from)[kLoads], unsigned long valid) {
        constexpr int kRow = (kPairs ? 2 : 1) * kStride;
        short* to = tile + position_of(row_first, 0) * kStride + row_piece * kPer16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) put<C, T>(to + i * kRow, from[i]);
        if (valid != ~0ul || d.d != DP) {
#pragma unroll 1
            for (int i = 0; i < kLoads; ++i)
                if (!in_row || !(valid >> (lane - row_piece + i) & 1)) {
#pragma unroll
                    for (int c = 0; c < kPer16; c += 8) *reinterpret_cast<v4u*>(to + i * kRow + c) = v4u{};
                }
        }
    };
    // whether the lane's score number i, of position i / 4 * 16 + j * 4 + i % 4, takes part
    auto scored = [&](int i, unsigned long valid) {
        const int at = i / 4 * 16 + j * 4 + i % 4;
        const int group = kPairs ? at / (2 * kLoads) * 2 + (at & 1) : at / kLoads, nth = kPairs ? at % (2 * kLoads) / 2 : at % kLoads;
        return valid >> (group * kRowPieces + nth) & 1;
    };

    const int qrow = tid >> 4, qc = tid & 15;                 // 16 queries at a time, 16 lanes each

    // What the first tile of a piece needs is requested while the piece before is under way.
    SharedPiece now = advance();
    if (now.table < 0) return;
    int t0 = now.k0 + wave * kTile;
    int entry = entry_of(now, t0), entry2 = entry_of(now, t0 + kStep);
    v4u kr[kLoads], vr[kLoads];
    unsigned long valid;
    {
        const unsigned place = place_of(now, t0, entry, valid);
        fetch(d.k_cache, now, place, kr);
        fetch(d.v_cache, now, place, vr);
    }
    while (true) {
        const SharedPiece then = advance();
        const int then_t0 = then.k0 + wave * kTile;
        const int then_entry = entry_of(then, then_t0), then_entry2 = entry_of(then, then_t0 + kStep);
        entry = entry2;
        const int g = now.g, k1 = now.k1, sets = (now.n + 15) / 16;
        // the sign of the scale goes with the queries
        const float by = d.scale * 1.44269504088896340736f * (sizeof(C) == 1 ? d.k_scale[g] : 1.0f);
        __syncthreads();                                      // the piece before is done with LDS
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (t >= sets) continue;
            const int i = now.i0 + t * 16 + qrow;
            const bool mine = t * 16 + qrow < now.n;
            const long at = (long)(now.row0 + i / a.group) * d.q_stride + (long)(g * a.group + i % a.group) * d.d;
            float x[DP / 16], top_q = 0.0f, down = 1.0f, up = 1.0f;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                const int col = qc + 16 * c;
                const bool there = mine && col < d.d;
                x[c] = !there ? 0.0f : d.q_dtype == NM_DT_F32 ? static_cast<const float*>(d.q)[at + col]
                              : d.q_dtype == NM_DT_BF16 ? (float)static_cast<const bf16*>(d.q)[at + col] : (float)static_cast<const f16*>(d.q)[at + col];
            }
            if (kQ > 1) {
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) top_q = fmaxf(top_q, fabsf(x[c]));
                top_q = __int_as_float(group_reduce<16>(__float_as_int(top_q), MaxF32{}));
                const int exponent = max(-126, min((int)(__float_as_uint(top_q) >> 23) - 127, 126));   // the row goes below 4
                down = __uint_as_float((unsigned)(127 - exponent) << 23);
                up = __uint_as_float((unsigned)(127 + exponent) << 23);
            }
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                float rest = copysignf(down, by) * x[c];
#pragma unroll
                for (int q = 0; q < kQ; ++q) {
                    const T v = (T)rest;
                    rest -= (float)v;
                    s_q[q][(t * 16 + qrow) * kStride + qc + 16 * c] = __builtin_bit_cast(short, v);
                }
            }
            if (qc == 0) s_qscale[t * 16 + qrow] = up;
        }
        __syncthreads();
        if (t0 >= k1) {                                       // no tile for this wavefront
            const unsigned place = place_of(then, then_t0, then_entry, valid);
            fetch(d.k_cache, then, place, kr);
            fetch(d.v_cache, then, place, vr);
        }
        v4f o[N][kBlocks];
        float m[N], l[N], factor[N];
#pragma unroll
        for (int t = 0; t < N; ++t) {
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) o[t][i] = v4f{0, 0, 0, 0};
            m[t] = -INFINITY;
            l[t] = 0.0f;
            // never 0, so that it takes a masked score, minus infinity, for what it is
            factor[t] = t < sets ? fmaxf(fabsf(by) * s_qscale[t * 16 + column], 1.17549435e-38f) : 1.0f;
        }
        for (; t0 < k1; t0 += kStep) {
            unsigned long next_valid;
            const bool more = t0 + kStep < k1;
            const SharedPiece& of = more ? now : then;
            const unsigned next = place_of(of, more ? t0 + kStep : then_t0, more ? entry : then_entry, next_valid);
            entry = entry_of(now, t0 + 2 * kStep);
            // scores
            stage(kr, valid);
            fetch(d.k_cache, of, next, kr);
            v4f sc[N][2];
#pragma unroll
            for (int t = 0; t < N; ++t) sc[t][0] = sc[t][1] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                v8s ka[2];
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) ka[blk] = *reinterpret_cast<const v8s*>(tile + (blk * 16 + column) * kStride + step * 32 + j * 8);
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    if (t >= sets) continue;
#pragma unroll
                    for (int q = kQ - 1; q >= 0; --q) {
                        const v8s qb = *reinterpret_cast<const v8s*>(s_q[q] + (t * 16 + column) * kStride + step * 32 + j * 8);
#pragma unroll
                        for (int blk = 0; blk < 2; ++blk) sc[t][blk] = Mma<T>::mma(ka[blk], qb, sc[t][blk]);
                    }
                }
            }
            v8s p[N][kP];
#pragma unroll
            for (int t = 0; t < N; ++t) {
                if (t >= sets) continue;
                if (valid != ~0ul) {
                    asm volatile("");                         // a branch: few tiles need it
#pragma unroll
                    for (int i = 0; i < 8; ++i) sc[t][i / 4][i % 4] = scored(i, valid) ? sc[t][i / 4][i % 4] : -INFINITY;
                }
                float top = sc[t][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[t][i / 4][i % 4]);
                top = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(top), MaxF32{}), MaxF32{}));
                top = fmaxf(m[t], top == -INFINITY ? top : top * factor[t]);
                const float base = top == -INFINITY ? 0.0f : top;
                const float shrink = __builtin_amdgcn_exp2f(m[t] - base);
                m[t] = top;
                l[t] *= shrink;
                const float lifted = kLift - base;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i / 4][i % 4], factor[t], lifted));
                    l[t] += w;
#pragma unroll
                    for (int q = 0; q < kP; ++q) {
                        const T v = (T)w;
                        w = __builtin_fmaf((float)v, -1.0f, w);
                        p[t][q][i] = __builtin_bit_cast(short, v);
                    }
                }
                if (__any(shrink != 1.0f)) {
#pragma unroll
                    for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[t][blk][i] *= shrink;
                }
            }
            // values
            stage(vr, valid);
            fetch(d.v_cache, of, next, vr);
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk) {
                const short* at = tile + (j * 4 + column / 4) * kStride + blk * 16 + column % 4 * 4;
                const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at));
                const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 16 * kStride));
                const v8s va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    if (t >= sets) continue;
#pragma unroll
                    for (int q = kP - 1; q >= 0; --q) o[t][blk] = Mma<T>::mma(va, p[t][q], o[t][blk]);
                }
            }
            valid = next_valid;
        }

        // the wavefronts' results as one, sixteen columns at a time
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if (t >= sets) continue;
            const float sum_l = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l[t]), AddF32{}), AddF32{}));
            __syncthreads();                                  // no tile, and no columns before these, are read any more
            if (j == 0) { s_m[wave][column] = m[t]; s_l[wave][column] = sum_l; }
            __syncthreads();
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s_m[w][column]);
            const float mine = __builtin_amdgcn_exp2f(m[t] - (top == -INFINITY ? 0.0f : top) - kLift);
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) s.o[wave][column][blk * 16 + j * 4 + i] = o[t][blk][i] * mine;
            __syncthreads();
            const int row = t * 16 + qrow;
            if (row < now.n) {
                const int i = now.i0 + row, b = now.row0 + i / a.group, h = g * a.group + i % a.group;
                float top = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) top = fmaxf(top, s_m[w][qrow]);
                const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int w = 0; w < W; ++w) sum += s_l[w][qrow] * __builtin_amdgcn_exp2f(s_m[w][qrow] - base - kLift);
                const long part = now.slot < 0 ? ((long)!now.prefix * d.B + b) * d.hq + h : ((long)worker * 2 + now.slot) * 16 * N + row;
                if (qc == 0) {
                    if (!now.done) (now.slot < 0 ? a.whole_ml : a.part_ml)[part] = make_float2(top, sum);
                    else if (d.lse) d.lse[(long)b * d.hq + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
                }
                const float over = (sum == 0.0f ? 0.0f : 1.0f / sum) * (sizeof(C) == 1 ? d.v_scale[g] : 1.0f);
                float* to = (now.slot < 0 ? a.whole_o : a.part_o) + part * d.d;
                for (int c = qc * 4; c < d.d; c += 64) {
                    v4f y{0, 0, 0, 0};
#pragma unroll
                    for (int w = 0; w < W; ++w) y += *reinterpret_cast<const v4f*>(&s.o[w][qrow][c]);
                    if (!now.done) {
                        *reinterpret_cast<v4f*>(to + c) = y;
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) store1(d.out, d.out_dtype, b * d.out_stride + (long)h * d.d + c + k, y[k] * over, d.out_inv_scale);
                    }
                }
            }
        }
        if (then.table < 0) break;
        now = then;
        t0 = then_t0;
        entry2 = then_entry2;
    }
}

// Joins what a query has: its group's prefix and its row's own positions, each whole or in pieces.  A workgroup to a query; lanes of four elements read every
// so-manieth piece's output and join them as they come; their results are joined through LDS.
__global__ __launch_bounds__(kPagedThreads) void shared_join_kernel(SharedArgs a)
{
    __shared__ __attribute__((aligned(16))) float s_o[kPagedThreads * 4];
    __shared__ float s_m[kPagedThreads / 4], s_l[kPagedThreads / 4];
    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, b = blockIdx.x / d.hq, h = blockIdx.x % d.hq, g = h / a.group, set = 16 * a.sets;
    const int lead = a.lead[b];
    const long bh = (long)b * d.hq + h, all = (long)d.B * d.hq;
    // [0] the prefix, [1] the row's own: pieces, the first's worker and slot, the query's number among the piece's
    int4 info[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
    int nth[2];
    {
        const int i = h % a.group;
        nth[1] = i % set;
        info[1] = a.info[all + (long)b * d.hq + g * a.group + i - nth[1]];
    }
    if (info[1].x < 0) return;
    if (lead >= 0) {
        const int i = (b - lead) * a.group + h % a.group;
        nth[0] = i % set;
        const int i0 = i - nth[0];
        info[0] = a.info[(long)(lead + i0 / a.group) * d.hq + g * a.group + i0 % a.group];
    }
    const int used = info[0].x + info[1].x;
    const int lanes = d.d / 4, at_once = kPagedThreads / lanes, mine = tid / lanes, c = tid % lanes * 4;
    float m = -INFINITY, l = 0.0f;
    v4f x{0, 0, 0, 0};
    if (mine < at_once) {
#pragma unroll 4
        for (int k = mine; k < used; k += at_once) {
            const int own = k >= info[0].x, i = own ? k - info[0].x : k;
            const int4 of = info[own];
            const long part = of.z < 0 ? own * all + bh : ((long)(of.y + i) * 2 + (i == 0 ? of.z : 0)) * set + nth[own];
            const float2 ml = (of.z < 0 ? a.whole_ml : a.part_ml)[part];
            const v4f y = *reinterpret_cast<const v4f*>((of.z < 0 ? a.whole_o : a.part_o) + part * d.d + c);
            const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
            const float shrink = __builtin_amdgcn_exp2f(m - base), by = __builtin_amdgcn_exp2f(ml.x - base);
            l = l * shrink + ml.y * by;
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = x[k] * shrink + y[k] * by;
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
    const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * (d.cache_dtype == NM_DT_I8 ? d.v_scale[g] : 1.0f);
    if (tid < d.d) store1(d.out, d.out_dtype, b * d.out_stride + (long)h * d.d + tid, v * by, d.out_inv_scale);
    if (tid == 0 && d.lse) d.lse[bh] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <typename C, typename T, int DP>
static void launch_shared(const SharedArgs& a, bool own, hipStream_t s)
{
    if (own) queue_kernel(shared_attention_kernel<C, T, DP, 1, 2, shared_sets(DP)>, dim3((a.workers + 7) / 8 * 8), dim3(kPagedThreads), 0, s, a);
    else queue_kernel(shared_attention_kernel<C, T, DP, 3, 3, shared_sets(DP)>, dim3((a.workers + 7) / 8 * 8), dim3(kPagedThreads), 0, s, a);
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
    const int width = paged_width(a.d.d);
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
    *alone = !divided;
    *a = SharedArgs{};
    a->d = d->p;
    a->G = d->G;
    a->group_start = d->group_start;
    a->shared = d->shared;
    a->shift = page_shift(d->p.page_size);
    a->group = d->p.hq / d->p.hk;
    const int width = paged_width(d->p.d);
    a->sets = shared_sets(width);
    a->workers = 256 * (width <= 128 ? 2 : 1);
    const size_t parts = (size_t)a->workers * 2 * 16 * a->sets, queries = (size_t)d->p.B * d->p.hq;
    Carve c{static_cast<char*>(ws)};
    c.take(a->head, 1);
    c.take(a->ent, (size_t)d->G + d->p.B);
    c.take(a->info, 2 * queries);
    c.take(a->before, a->workers);
    c.take(a->first, a->workers);
    c.take(a->lead, d->p.B);
    c.take(a->part_ml, parts);
    c.take(a->whole_ml, 2 * queries);
    c.take(a->part_o, parts * d->p.d);
    c.take(a->whole_o, 2 * queries * d->p.d);
    *bytes = *alone ? 0 : c.used;
    return NM_OK;
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
    if (alone) return nm_paged_attention(&d, nullptr, 0, stream);
    if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_shared_attention: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_shared_attention: workspace must be 256-byte aligned");
    const hipStream_t s = (hipStream_t)stream;
    queue_kernel(shared_plan_kernel, dim3(1), dim3(kPlanners), 0, s, a);
    if (d.cache_dtype == NM_DT_BF16) launch_shared<bf16, bf16>(a, s);
    else if (d.cache_dtype == NM_DT_F16) launch_shared<f16, f16>(a, s);
    else if (d.q_dtype == NM_DT_F16) launch_shared<int8_t, f16>(a, s);
    else launch_shared<int8_t, bf16>(a, s);
    if ((rc = check_hip(hipGetLastError(), "nm_shared_attention launch"))) return rc;
    queue_kernel(shared_join_kernel, dim3(d.B * d.hq), dim3(kPagedThreads), 0, s, a);
    return check_hip(hipGetLastError(), "nm_shared_attention launch");
}

}  // extern "C"
