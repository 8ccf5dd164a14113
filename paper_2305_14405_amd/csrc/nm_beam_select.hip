// The best continuations of every request's hypotheses (nm_beam_select).
//
// One pass over the logits makes both of what is needed of a row: its sum of exponentials, and its K best logits.  (Within a row the order of
// candidates is that of the logits, so nothing but K of a row can be among the request's K.)  A workgroup goes over a chunk of a row, every lane with a
// maximum and a sum of its own.  Each wavefront sorts its lanes' maxima; the K-th of one wavefront, and the least of the wavefronts' K/4-th, are values that at least
// K logits of the chunk reach.  The lanes that hold such logits, K and a few more, are few: of what they went over, the tiles whose
// largest logit (kept in LDS) reaches the value are read again, the logits that reach the value are collected in LDS, and each counts how many are better: that is its place.  A candidate is one 64-bit number, the logit's bits in the order
// of their values above the complement of the token, so that comparing it settles ties too.  Where more than LDS takes reach the value (many
// equal logits, or all large ones in a few lanes), they are put one by one into lists, sorted, an entry to a lane.
//   A second kernel has a workgroup to a request: it joins the chunks' sums, forms the candidates' log-probabilities in 64 bits, and chooses among
// them in the same way; short histories it copies itself.
//   Bound by latency at few rows: one request of 4 hypotheses, 32000 fp32 logits, 5.3 + 4.4 us, chains of loads, a sort of 21 steps, barriers.  32 of 8, 131072
// bf16 (67 MB, 13 us at a copy's rate): 18.1 + 5.2, 3.7 TB/s in the first: two workgroups to a CU, vector instructions 47 % of the cycles, and 3 us of the
// same chain behind the last logits.  Half of the tokens masked, by -inf or a finite number: the same (22.9, 35.5 where a lane's sum began from a logit of 0, so that low first
// ones had the chunk read twice).  Chunks of nothing but one finite number, three quarters of a row: 97, for all of their logits are equal, and go through the lists, one
// by one; of -inf: 22.5.  (All of a lane's logits read again, where only some of its tiles are wanted: 20.6.  Lists of K kept by every wavefront as it goes:
// 83 in all.)
#include <algorithm>

#include "nm_decode.h"

namespace nm {

constexpr int kBeamWaves = 4, kBeamThreads = 64 * kBeamWaves;   // of the first kernel
constexpr int kJoinWaves = 8, kJoinThreads = 64 * kJoinWaves;   // of the second
// Groups of 16 bytes that a lane asks for at a time: with 4 the code, which is fetched as it first runs, is longer (one request of 4 over 32000 9.6 us, 9.1 with
// 2; 24 of 6 over 50001 16.9 and 15.9; 32 of 8 over 131072 22.8 either way), with 1 too little is under way (16.5, 25.3).
constexpr int kBeamStep = 2;
constexpr int kBeamMost = 512;                                 // candidates that are ranked at once
constexpr int kRecords = 32;                                   // maxima that a lane of the first kernel keeps of its logits

struct BeamArgs {
    nm_beam_desc d;
    int chunks, chunk;               // of a row, and their length, a number of kBeamStep groups of 16 bytes for every lane
    FastDiv each;                    // candidates of a row: chunks K
    int rows;                        // of this launch of the first kernel
    int histories;                   // the second kernel copies them
    unsigned long* part_key;         // [R W, chunks, K], best first, 0: none
    double* part_sum;                // [R W, chunks]: sum of exp(x - max)
    float* part_max;                 // [R W, chunks], -inf: no logits
};

typedef unsigned long Key;

// A logit and its token as one number: greater is better.  -inf is not among them.
__device__ __forceinline__ Key key_of(float x, int v)
{
    const unsigned u = __float_as_uint(x + 0.0f);              // -0 is 0
    return (Key)(u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) << 32 | (unsigned)~v;
}
__device__ __forceinline__ float logit_of(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int token_of(Key k) { return (int)~(unsigned)k; }

__device__ __forceinline__ Key lane_key(Key k, int lane)       // of a uniform lane
{
    return (Key)(unsigned)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)k, lane);
}
// The wavefront's list, entry i in lane i, with one more; what falls behind lane 63 is gone.
__device__ __forceinline__ Key insert(Key list, Key key, int lane)
{
    const int at = __popcll(__ballot(list > key));
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)list, 0x138, 0xf, 0xf, false);          // from the lane in front (wave_shr:1)
    const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(list >> 32), 0x138, 0xf, 0xf, false);
    return lane < at ? list : lane == at ? key : (Key)hi << 32 | lo;
}
// Those of a wavefront's keys (one to a lane, 0: none) that belong into the list's first K.
__device__ __forceinline__ Key insert_all(Key list, Key mine, int K, int lane)
{
    Key least = lane_key(list, K - 1);
    unsigned long left = __ballot(mine > least);
    while (left) {
        const int from = __ffsll((long long)left) - 1;
        list = insert(list, lane_key(mine, from), lane);
        least = lane_key(list, K - 1);
        left &= left - 1;
        left &= __ballot(mine > least);
    }
    return list;
}

// The value of lane ^ MASK.
struct Second { __device__ __forceinline__ int operator()(int, int b) const { return b; } };
struct Differ { __device__ __forceinline__ int operator()(int a, int b) const { return a ^ b; } };
template <int MASK>
__device__ __forceinline__ int across(int v)
{
    return MASK < 16 ? butterfly_step<MASK>(v, Second{}) : butterfly_step<MASK>(v, Differ{}) ^ v;
}
template <int MASK>
__device__ __forceinline__ double across(double v)
{
    const long u = __double_as_longlong(v);
    return __longlong_as_double((long)across<MASK>((int)(u >> 32)) << 32 | (unsigned)across<MASK>((int)u));
}
__device__ __forceinline__ double wave_sum(double v)
{
    v += across<32>(v);
    v += across<16>(v);
    v += across<8>(v);
    v += across<4>(v);
    v += across<2>(v);
    return v + across<1>(v);
}
__device__ __forceinline__ float wave_max(float v) { return __int_as_float(group_reduce<64>(__float_as_int(v), MaxF32{})); }

// Sorts a wavefront's numbers, the largest into lane 0 (Batcher's bitonic order: runs of SIZE, merged over distances STEP).
template <int SIZE, int STEP>
__device__ __forceinline__ float sort_step(float v, int lane)
{
    const float other = __int_as_float(across<STEP>(__float_as_int(v)));
    v = ((lane & STEP) == 0) == ((lane & SIZE) == 0) ? fmaxf(v, other) : fminf(v, other);
    if constexpr (STEP > 1) v = sort_step<SIZE, STEP / 2>(v, lane);
    return v;
}
__device__ __forceinline__ float sorted(float v, int lane)
{
    v = sort_step<2, 1>(v, lane);
    v = sort_step<4, 2>(v, lane);
    v = sort_step<8, 4>(v, lane);
    v = sort_step<16, 8>(v, lane);
    v = sort_step<32, 16>(v, lane);
    return sort_step<64, 32>(v, lane);
}

// A value that at least K of the numbers whose maxima over disjoint sets the workgroup's threads have reach (-inf: there may be fewer).  s: LDS.
template <int W>
__device__ __forceinline__ float reached(float top, int K, float (&s)[2][W])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int order = __float_as_int(sorted(top, lane));
    // with every lane active: of one that is not, a copy of the register need not have the value
    const float last = __int_as_float(__builtin_amdgcn_readlane(order, K - 1)), share = __int_as_float(__builtin_amdgcn_readlane(order, (K - 1) / W));
    if (lane == 0) {
        s[0][wave] = last;
        s[1][wave] = share;
    }
    __syncthreads();
    float most = s[0][0], least = s[1][0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
        most = fmaxf(most, s[0][w]);
        least = fminf(least, s[1][w]);
    }
    return fmaxf(most, least);
}

constexpr float kLog2e = 1.44269504088896340736f;
// Largest logits of a row, of either sign, whose products with log2(e) a rounding moves by 64 at most, half a step of numbers below 2^31: powers of two of what it leaves, and
// of its opposite, are far from exp2's ends.  (Of 2092843776 it leaves -127.3: the power is flushed to 0, its inverse is no infinity, and the sum would be 0.)
constexpr float kFarLogit = 1073741824.0f;

// NaN: -inf, +inf: the largest number.  (A median of three with -inf as a bound is folded into a minimum, which passes the number in place of a NaN.)
__device__ __forceinline__ float logit(float x) { return x == x ? fminf(x, 3.40282346638528859812e38f) : -INFINITY; }

// Whether the row's logits matter: its hypothesis goes on from a score and a weight that are numbers.
__device__ __forceinline__ bool offers(const nm_beam_desc& d, long row)
{
    const float s = d.scores[row], w = d.weight ? d.weight[row] : 1.0f;
    return __builtin_fabsf(s) < INFINITY && w > 0.0f && w < INFINITY;
}

// The largest of three; a NaN is passed over, or left for the sum to show.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float v;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(v) : "v"(a), "v"(b), "v"(c));
    return v;
}

// Calls use(i, how many of n numbers are better than number i) for each of them, L lanes to a number.
template <int L, int kThreads, typename Better, typename Use>
__device__ __forceinline__ void places(int n, Better better, Use use)
{
    for (int i0 = 0; i0 < n; i0 += kThreads / L) {
        const int i = i0 + (int)threadIdx.x / L, mine = min(i, n - 1);
        int place = 0;
#pragma unroll 2
        for (int k = threadIdx.x % L; k < n; k += L) place += better(k, mine);
        place = group_reduce<L>(place, AddI32{});
        if (i < n && threadIdx.x % L == 0) use(i, place);
    }
}

template <typename T>
__global__ __launch_bounds__(kBeamThreads) void beam_rows_kernel(BeamArgs a)
{
    constexpr int kGroup = 16 / (int)sizeof(T), kApart = kBeamThreads * kGroup, kTile = kBeamStep * kApart;
    constexpr int kEach = kBeamStep * kGroup;                  // logits of a lane at a time
    typedef T Vec __attribute__((ext_vector_type(kGroup)));
    __shared__ Key s_key[kBeamMost];
    __shared__ float s_max[kBeamWaves], s_reached[2][kBeamWaves];
    __shared__ double s_sum[kBeamWaves];
    __shared__ float s_record[kRecords][kBeamThreads];        // largest logits of a lane's tiles, `span` tiles to a number
    __shared__ unsigned s_count, s_hits, s_hit[kBeamMost];
    const nm_beam_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = d.K;
    const long row = blockIdx.y;
    const T* x = static_cast<const T*>(d.logits) + row * d.logits_stride;
    // groups of 16 bytes begin `ahead` elements in front of the row
    const int ahead = (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
    const int begin = (int)blockIdx.x * a.chunk - ahead, end = min(begin + a.chunk, d.V);
    // a group of the row: a logit in front of it or behind is none.  What lies between the first row's begin and the last one's end may be read.
    const long front = -row * d.logits_stride, behind = (a.rows - 1 - row) * d.logits_stride + d.V;
    auto group = [&](int v) -> Vec {
        Vec w;
        if (v >= front && v + kGroup <= behind) {
            w = *reinterpret_cast<const Vec*>(x + v);
#pragma unroll
            for (int e = 0; e < kGroup; ++e) w[e] = (unsigned)(v + e) < (unsigned)d.V ? w[e] : (T)-INFINITY;
        } else {
#pragma unroll 1
            for (int e = 0; e < kGroup; ++e) w[e] = (unsigned)(v + e) < (unsigned)d.V ? x[v + e] : (T)-INFINITY;
        }
        return w;
    };
    auto ask = [&](int t, Vec (&w)[kBeamStep]) {
        const int v = t + tid * kGroup;
        if (t >= 0 && t + kTile <= d.V) {                      // uniform
#pragma unroll
            for (int i = 0; i < kBeamStep; ++i) w[i] = *reinterpret_cast<const Vec*>(x + v + i * kApart);
        } else {
#pragma unroll
            for (int i = 0; i < kBeamStep; ++i) w[i] = group(v + i * kApart);
        }
    };
    // the first are asked for before it is known whether the row matters
    Vec w[kBeamStep];
    ask(begin, w);
    if (!offers(d, row) || (d.done && d.done[row])) return;    // uniform
    if (tid == 0) s_count = s_hits = 0;
    const int span = (a.chunk / kTile + kRecords - 1) / kRecords;
    int records;

    // Logits as they are (of numbers that mask tokens, such as -1e9 or a type's lowest, the powers are 0); where +inf or a NaN turns up in the maximum or the sum, or the maximum of the
    // chunk is far from 0, once more with what they count as, by differences.
    float top, least, mine;
    double sum;
    auto sweep = [&](auto special) {
        mine = -INFINITY;
        sum = 0;
        records = 0;
        int left = span;
        // off: what is subtracted from x log2(e); from the lowest on, so that a sum of nothing is never multiplied by an infinity
        float record = -INFINITY, off = -kFarLogit * kLog2e;
        for (int t = begin; t < end; t += kTile) {
            float y[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) y[i] = special ? logit((float)w[i / kGroup][i % kGroup]) : (float)w[i / kGroup][i % kGroup];
            if (t + kTile < end) ask(t + kTile, w);
            float tile = y[0];
#pragma unroll
            for (int i = 1; i + 1 < kEach; i += 2) tile = max3(tile, y[i], y[i + 1]);
            record = max3(record, tile, y[kEach - 1]);
            const float now = fmaxf(mine, record);
            if (--left == 0) {                                 // uniform
                s_record[records++][tid] = record;
                record = -INFINITY;
                left = span;
            }
            float part[4] = {0, 0, 0, 0};
            if (!special) {
                // exp(x - m) as a power of two of x log2(e) - m log2(e), rounded once (what the second product's rounding leaves is made up for behind)
                const float next = fmaxf(now, -kFarLogit) * kLog2e;
#pragma unroll
                for (int i = 0; i < kEach; ++i) part[i % 4] += __builtin_amdgcn_exp2f(__builtin_fmaf(y[i], kLog2e, -next));
                sum *= (double)__builtin_amdgcn_exp2f(off - next);
                off = next;
            } else {
                const float base = now == -INFINITY ? 0.0f : now;
#pragma unroll
                for (int i = 0; i < kEach; ++i) part[i % 4] += __builtin_amdgcn_exp2f((y[i] - base) * kLog2e);
                sum *= (double)__builtin_amdgcn_exp2f((mine - base) * kLog2e);
            }
            sum += (double)((part[0] + part[1]) + (part[2] + part[3]));
            mine = now;
        }
        if (left < span) s_record[records++][tid] = record;
        top = wave_max(mine);
        if (lane == 0) s_max[wave] = top;
        least = reached(mine, K, s_reached);                   // synchronises
#pragma unroll
        for (int i = 0; i < kBeamWaves; ++i) top = fmaxf(top, s_max[i]);
        const float base = top == -INFINITY ? 0.0f : top;
        const float from = special ? mine : fmaxf(mine, -kFarLogit);
        float by = __builtin_amdgcn_exp2f((from - base) * kLog2e);
        if (!special) by *= __builtin_amdgcn_exp2f(-__builtin_fmaf(from, kLog2e, -off));
        sum = wave_sum(sum * (double)by);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = 0;
#pragma unroll
        for (int i = 0; i < kBeamWaves; ++i) sum += s_sum[i];
    };
    sweep(std::false_type{});
    if (!((__builtin_fabsf(top) <= kFarLogit || top == -INFINITY) && sum < INFINITY)) {   // uniform; NaNs too
        __syncthreads();
        ask(begin, w);
        sweep(std::true_type{});
    }
    const long out = row * a.chunks + blockIdx.x;
    if (tid == 0) {
        a.part_max[out] = top;
        a.part_sum[out] = sum;
    }

    // The tiles of lanes that hold any of those are read once more, by all lanes.  (Code for what few lanes come to is fetched for all.)
    if (mine >= least && mine > -INFINITY)
#pragma unroll 1
        for (int i = tid; i < records * kBeamThreads; i += kBeamThreads) {
            const float record = s_record[i / kBeamThreads][i % kBeamThreads];
            if (record >= least && record > -INFINITY) {
                const unsigned at = atomicAdd(&s_hits, 1u);
                if (at < kBeamMost) s_hit[at] = i;
            }
        }
    __syncthreads();
    const unsigned hits = s_hits, all = a.chunk / kGroup, each = span * kBeamStep, groups = hits <= kBeamMost ? hits * each : 0;
    auto number = [&](unsigned i) {
        const unsigned hit = s_hit[i % hits];
        return begin + (int)((hit / kBeamThreads * each + i / hits) * kApart + hit % kBeamThreads * kGroup);
    };
    for (unsigned i = tid; i < groups; i += kBeamThreads) {
        const int v = number(i);
        if (v >= begin + a.chunk) continue;                    // the last number's tiles may be fewer
        const Vec y = group(v);
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
            const float z = logit((float)y[e]);
            if (z >= least && z > -INFINITY) {
                const unsigned at = atomicAdd(&s_count, 1u);
                if (at < kBeamMost) s_key[at] = key_of(z, v + e);
            }
        }
    }
    __syncthreads();
    const int n = (int)(hits <= kBeamMost ? s_count : hits);          // each of them has a logit of those
    Key* best = a.part_key + out * K;
    if (n <= kBeamMost) {
        if (tid >= n && tid < K) best[tid] = 0;
        places<8, kBeamThreads>(n, [&](int k, int i) { return (int)(s_key[k] > s_key[i]); }, [&](int i, int place) {
            if (place < K) best[place] = s_key[i];
        });
        return;
    }
    __syncthreads();
    Key list = 0;
    for (unsigned i0 = 0; i0 < all; i0 += kBeamThreads) {      // every lane of a wavefront comes along
        const unsigned i = i0 + tid;
#pragma unroll 1
        for (int e = 0; e < kGroup; ++e) {
            const int v = i < all ? begin + (int)(i * kGroup) + e : -1;
            const float z = v >= 0 && v < d.V ? logit((float)x[v]) : -INFINITY;
            list = insert_all(list, z >= least && z > -INFINITY ? key_of(z, v) : 0, K, lane);
        }
    }
    s_key[tid] = list;
    __syncthreads();
    if (wave) return;
#pragma unroll 1
    for (int i = 1; i < kBeamWaves; ++i) list = insert_all(list, lane < K ? s_key[i * 64 + lane] : 0, K, lane);
    if (lane < K) best[lane] = list;
}

constexpr int kFollow = 8;

// A row's history behind its choice: tokens [first, ...) of those that it takes over, every `step`-th; and the new one.
__device__ __forceinline__ void follow(const nm_beam_desc& d, long row, int parent, int token, int first, int step)
{
    const int held = parent < 0 ? 0 : min(max(d.history_lens[parent], 0), d.max_history);
    const bool grows = parent >= 0 && held < d.max_history && !(d.done && d.done[parent]);
    int* to = d.history_out + row * d.history_out_stride;
    const int* from = d.history + (long)max(parent, 0) * d.history_stride;
    for (int i = first; i < held; i += kFollow * step) {       // that many under way
        int x[kFollow];
#pragma unroll
        for (int k = 0; k < kFollow; ++k) x[k] = from[min(i + k * step, held - 1)];
#pragma unroll
        for (int k = 0; k < kFollow; ++k)
            if (i + k * step < held) to[i + k * step] = x[k];
    }
    if (first == 0) {
        if (grows) to[held] = token;
        d.history_lens_out[row] = held + grows;
    }
}

// A workgroup to a request.
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a)
{
    // of a hypothesis: its largest logit, what is added to a logit's difference from that, and its weight; kind 0: offers nothing, 1: its tokens, 2: its end
    __shared__ float s_top[NM_BEAM_MAX];
    __shared__ double s_add[NM_BEAM_MAX], s_weight[NM_BEAM_MAX], s_rank[kBeamMost];
    __shared__ Key s_key[kBeamMost];
    __shared__ int s_kind[NM_BEAM_MAX], s_of[kBeamMost], s_count, s_parent[NM_BEAM_MAX], s_token[NM_BEAM_MAX];
    __shared__ float s_reached[2][kJoinWaves];
    const nm_beam_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = d.K, W = d.W, r = blockIdx.x;
    const long row0 = (long)r * W;
    const int each = a.chunks * K, all = W * each;
    const Key* keys = a.part_key + row0 * each;
    // The first candidate is asked for before anything else (of a hypothesis that turns out to offer none, it is not looked at).
    const Key ahead = keys[min(tid, all - 1)];
    for (int w = wave; w < W; w += kJoinWaves) {
        const long row = row0 + w, part = row * a.chunks;
        const float m0 = a.part_max[part + min(lane, a.chunks - 1)];
        const double l0 = a.part_sum[part + min(lane, a.chunks - 1)];
        const int kind = !offers(d, row) ? 0 : d.done && d.done[row] ? 2 : 1;
        float top = -INFINITY;
        double sum = 0;
        if (kind == 1) {
            if (lane < a.chunks) top = m0;
            for (int c = lane + 64; c < a.chunks; c += 64) top = fmaxf(top, a.part_max[part + c]);
            top = wave_max(top);
            const float base = top == -INFINITY ? 0.0f : top;
            if (lane < a.chunks) sum = l0 * (double)__builtin_amdgcn_exp2f((m0 - base) * kLog2e);
            for (int c = lane + 64; c < a.chunks; c += 64) sum += a.part_sum[part + c] * (double)__builtin_amdgcn_exp2f((a.part_max[part + c] - base) * kLog2e);
            sum = wave_sum(sum);
        }
        if (lane == 0) {
            s_top[w] = top;
            s_add[w] = (double)d.scores[row] - (kind == 1 ? log(sum) : 0.0);
            s_weight[w] = d.weight ? (double)d.weight[row] : 1.0;
            s_kind[w] = kind;
        }
    }
    if (tid == 0) s_count = 0;
    for (int k = tid; k < K; k += kJoinThreads) s_parent[k] = s_token[k] = -1;
    __syncthreads();

    // The candidates one after the other: hypothesis, key (an end's is 1), and what it is ranked by.
    auto candidates = [&](auto&& use) {
#pragma unroll 1
        for (int i = tid; i < all; i += kJoinThreads) {
            const int w = (int)quotient(i, a.each), kind = s_kind[w];
            const Key key = kind == 1 ? (i == tid ? ahead : keys[i]) : (Key)(kind == 2 && i == w * each);
            if (key) use(w, key, (kind == 2 ? s_add[w] : ((double)logit_of(key) - (double)s_top[w]) + s_add[w]) * s_weight[w]);
        }
    };
    float least = -INFINITY;                                   // all of few
    if (all > 64) {
        float top = -INFINITY;
        candidates([&](int, Key, double rank) { top = fmaxf(top, (float)rank); });   // (rounding keeps the order)
        least = reached(top, K, s_reached);
    }
    candidates([&](int w, Key key, double rank) {
        if ((float)rank >= least) {
            const int at = atomicAdd(&s_count, 1);
            if (at < kBeamMost) {
                s_rank[at] = rank;
                s_key[at] = key;
                s_of[at] = w;
            }
        }
    });
    __syncthreads();
    const int n = s_count;
    auto put = [&](int k, int w, Key key) {
        const long out = (long)r * K + k;
        const int kind = s_kind[w], token = kind == 2 ? d.end_token : token_of(key);
        d.parents[out] = s_parent[k] = (int)row0 + w;
        d.tokens[out] = s_token[k] = token;
        d.scores_out[out] = (float)(kind == 2 ? s_add[w] : ((double)logit_of(key) - (double)s_top[w]) + s_add[w]);
        if (d.done_out) d.done_out[out] = kind == 2 || token == d.end_token;
    };
    if (n <= kBeamMost) {
        places<4, kJoinThreads>(n, [&](int k, int i) {
            const double other = s_rank[k], rank = s_rank[i];
            const int w = s_of[k], v = s_of[i];
            return (int)(other > rank) | ((int)(other == rank) & ((int)(w < v) | ((int)(w == v) & (int)(s_key[k] > s_key[i]))));
        }, [&](int i, int place) {
            if (place < K) put(place, s_of[i], s_key[i]);
        });
    } else {
        // one list after the other: the best by their place among those in front, an entry to a lane
        __syncthreads();
        if (wave == 0) {
            double list_rank = -INFINITY;
            int list_w = 0;
            Key list_key = 0;
            for (int w = 0; w < W; ++w) {
                if (!s_kind[w]) continue;
                Key row = 0;                                   // the hypothesis' own, by key
                if (s_kind[w] == 2) row = lane == 0;
                else
                    for (int c = 0; c < a.chunks; ++c) row = insert_all(row, lane < K ? a.part_key[((row0 + w) * a.chunks + c) * K + lane] : 0, K, lane);
                for (int i = 0; i < K; ++i) {
                    const Key key = lane_key(row, i);
                    if (!key) break;
                    const double rank = (s_kind[w] == 2 ? s_add[w] : ((double)logit_of(key) - (double)s_top[w]) + s_add[w]) * s_weight[w];
                    const int at = __popcll(__ballot(list_key && list_rank >= rank));   // those in front are of lower hypotheses, or better
                    if (at >= K) break;
                    const double up_rank = __shfl_up(list_rank, 1);
                    const int up_w = __shfl_up(list_w, 1);
                    const Key up_key = __shfl_up(list_key, 1);
                    if (lane == at) { list_rank = rank; list_w = w; list_key = key; }
                    else if (lane > at) { list_rank = up_rank; list_w = up_w; list_key = up_key; }
                }
            }
            if (lane < K && list_key) put(lane, list_w, list_key);
        }
    }
    __syncthreads();
    for (int k = tid; k < K; k += kJoinThreads)
        if (s_parent[k] < 0) {
            const long out = (long)r * K + k;
            d.parents[out] = d.tokens[out] = -1;
            d.scores_out[out] = -INFINITY;
            if (d.done_out) d.done_out[out] = 0;
        }
    if (a.histories)
        for (int k = wave; k < K; k += kJoinWaves) follow(d, (long)r * K + k, s_parent[k], s_token[k], lane, 64);
}

// Long histories: a few workgroups to a row.
__global__ __launch_bounds__(kBeamThreads) void beam_history_kernel(nm_beam_desc d)
{
    const long row = blockIdx.x;
    follow(d, row, d.parents[row], d.tokens[row], blockIdx.y * kBeamThreads + threadIdx.x, gridDim.y * kBeamThreads);
}

// Workgroups of the first kernel, about: 512 22.8 us for 32 requests of 8 over 131072, 768 23.2; 24 of 6 over 50001 with twice as many 2 us longer.
constexpr long kBeamGroups = 512;
// Tokens that a history, and a request's histories, have room for up to which its workgroup of the second kernel copies them, a wavefront to a history; more go to a
// kernel of their own.  (There and by a kernel: 4 of 1000 12.1 and 13.2 us, of 4000 14.3 and 13.3; 16 requests of 8 of 2000 16.0 and 16.2; 300 of 2 of 4000 24.4 and 23.4.)
constexpr int kHistory = 2048;
constexpr long kHistories = 16384;

static int32_t plan_beam(const nm_beam_desc* d, BeamArgs* a, size_t* bytes, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    if (d->R < 0 || d->W < 1 || d->K < 1 || d->V < 1) return fail(NM_ERR_INVALID_ARG, "%s: bad shape", what);
    if (!float_dtype(d->logits_dtype)) return fail(NM_ERR_INVALID_ARG, "%s: bad logits_dtype", what);
    if (d->W > NM_BEAM_MAX || d->K > NM_BEAM_MAX) return fail(NM_ERR_UNSUPPORTED, "%s: W %d or K %d > %d", what, d->W, d->K, NM_BEAM_MAX);
    if ((int64_t)d->R * d->W > 1 << 20 || (int64_t)d->R * d->K > 1 << 23 || d->V > 1 << 26)   // 2^24 workgroups of 256 are more than a launch takes
        return fail(NM_ERR_UNSUPPORTED, "%s: R * W > 2^20, R * K > 2^23 or V > 2^26", what);
    if (d->history && d->max_history > 1 << 30) return fail(NM_ERR_UNSUPPORTED, "%s: max_history > 2^30", what);
    *a = BeamArgs{};
    a->d = *d;
    // chunks of one tile where there are few rows, and as many as give every CU two workgroups
    const long rows = (long)d->R * d->W, tile = kBeamStep * kBeamThreads * 16 / dtype_bytes(d->logits_dtype);
    const long tiles = ((long)d->V + 15 + tile - 1) / tile;    // a row's first group of 16 bytes may begin in front of it
    const long wanted = rows ? std::min(std::max(1l, kBeamGroups / rows), tiles) : 1;
    a->chunk = (int)((tiles + wanted - 1) / wanted * tile);
    a->chunks = (int)((tiles * tile + a->chunk - 1) / a->chunk);
    a->each = fast_div(a->chunks * d->K);
    a->histories = d->history && d->max_history <= kHistory && (long)d->K * d->max_history <= kHistories;
    const size_t parts = (size_t)rows * a->chunks;
    *bytes = parts * (d->K * sizeof(Key) + sizeof(double) + sizeof(float));
    return NM_OK;
}

}  // namespace nm

using namespace nm;

extern "C" {

int32_t nm_beam_select_workspace(const nm_beam_desc* d, size_t* bytes)
{
    BeamArgs a;
    size_t n;
    const int32_t rc = plan_beam(d, &a, &n, "nm_beam_select_workspace");
    if (rc) return rc;
    if (!bytes) return fail(NM_ERR_INVALID_ARG, "nm_beam_select_workspace: bytes is NULL");
    *bytes = n;
    return NM_OK;
}

int32_t nm_beam_select(const nm_beam_desc* d, void* ws, size_t ws_bytes, void* stream)
{
    BeamArgs a;
    size_t need;
    const int32_t rc = plan_beam(d, &a, &need, "nm_beam_select");
    if (rc) return rc;
    if (d->end_token < -1 || d->end_token >= d->V) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: end_token %d is no token", d->end_token);
    if (d->end_token < 0 && d->done) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: done without an end_token");
    if (d->logits_stride < d->V) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: logits_stride is shorter than a row");
    if (d->history ? d->max_history < 1 || d->history_stride < d->max_history || d->history_out_stride < d->max_history : false)
        return fail(NM_ERR_INVALID_ARG, "nm_beam_select: max_history < 1, or a stride of the histories is shorter");
    if (d->R == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->logits || !d->scores || !d->parents || !d->tokens || !d->scores_out) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: logits, scores, parents, tokens or scores_out is NULL");
    if (d->history ? !d->history_lens || !d->history_out || !d->history_lens_out : d->history_lens || d->history_out || d->history_lens_out)
        return fail(NM_ERR_INVALID_ARG, "nm_beam_select: history, history_lens, history_out and history_lens_out belong together");
    const void* in[] = {d->logits, d->scores, d->weight, d->done, d->history, d->history_lens};
    const void* out[] = {d->parents, d->tokens, d->scores_out, d->done_out, d->history_out, d->history_lens_out};
    for (const void*& q : out) {
        for (const void* p : in)
            if (p && p == q) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: an output is an input");
        for (const void*& p : out)
            if (&p != &q && p && p == q) return fail(NM_ERR_INVALID_ARG, "nm_beam_select: two outputs are one");
    }
    if (!aligned(d->logits, dtype_bytes(d->logits_dtype))) return fail(NM_ERR_UNSUPPORTED, "nm_beam_select: logits are not aligned to their elements");
    if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_beam_select: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_beam_select: workspace must be 256-byte aligned");
    const int rows = d->R * d->W;
    const size_t parts = (size_t)rows * a.chunks;
    a.part_key = static_cast<Key*>(ws);
    a.part_sum = reinterpret_cast<double*>(a.part_key + parts * d->K);
    a.part_max = reinterpret_cast<float*>(a.part_sum + parts);
    const hipStream_t s = (hipStream_t)stream;
    // rows are the grid's second dimension, of at most 2^16 - 1 workgroups: more go in pieces
    for (int first = 0; first < rows; first += 65535) {
        BeamArgs b = a;
        const int n = std::min(rows - first, 65535);
        b.rows = n;
        b.d.logits = static_cast<const char*>(d->logits) + first * d->logits_stride * dtype_bytes(d->logits_dtype);
        b.d.scores += first;
        if (b.d.weight) b.d.weight += first;
        if (b.d.done) b.d.done += first;
        b.part_key += (size_t)first * a.chunks * d->K;
        b.part_sum += (size_t)first * a.chunks;
        b.part_max += (size_t)first * a.chunks;
        const dim3 grid(a.chunks, n);
        if (d->logits_dtype == NM_DT_F32) queue_kernel(beam_rows_kernel<float>, grid, dim3(kBeamThreads), 0, s, b);
        else if (d->logits_dtype == NM_DT_BF16) queue_kernel(beam_rows_kernel<bf16>, grid, dim3(kBeamThreads), 0, s, b);
        else queue_kernel(beam_rows_kernel<f16>, grid, dim3(kBeamThreads), 0, s, b);
        const int32_t err = check_hip(hipGetLastError(), "nm_beam_select launch");
        if (err) return err;
    }
    queue_kernel(beam_join_kernel, dim3(d->R), dim3(kJoinThreads), 0, s, a);
    if (d->history && !a.histories) {
        const int32_t err = check_hip(hipGetLastError(), "nm_beam_select launch");
        if (err) return err;
        queue_kernel(beam_history_kernel, dim3(d->R * d->K, std::min((d->max_history + kFollow * kBeamThreads - 1) / (kFollow * kBeamThreads), 64)), dim3(kBeamThreads), 0, s, *d);
    }
    return check_hip(hipGetLastError(), "nm_beam_select launch");
}

}  // extern "C"
