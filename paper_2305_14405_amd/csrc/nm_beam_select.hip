// The best continuations of every request's hypotheses (nm_beam_select).
//
// One pass over the logits makes both of what is needed of a row: its sum of exponentials, and its K best logits.  (Within a row the order of
// candidates is that of the logits, so nothing but K of a row can be among the request's K.)  A wavefront takes 2048 logits at a time into
// registers; each lane has a running maximum and sum of its own, and the wavefront one list, sorted, an entry to a lane: an entry is one 64-bit number, the
// logit's bits in the order of their values above the complement of the token, so that comparing it settles ties too.  Logits above the K-th
// entry are found by a ballot and put in one by one, which few are after the first thousands.  Rows are split into chunks where there are few of them.  A
// second kernel has a workgroup to a request: it merges the chunks' lists and sums, forms the candidates' log-probabilities in 64 bits, and
// merges the rows' lists, W heads at a time.
#include <algorithm>

#include "nm_decode.h"

namespace nm {

constexpr int kBeamWaves = 4, kBeamThreads = 64 * kBeamWaves;
constexpr int kBeamLane = 32, kBeamTile = 64 * kBeamLane;      // logits of a lane, of a wavefront
constexpr int kBeamChunks = 64;                                // of a row at most: a lane of the second kernel to each

struct BeamArgs {
    nm_beam_desc d;
    int chunks, chunk;               // of a row, and their length
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

// exp(a) for a <= 0, by the hardware's power of two.
__device__ __forceinline__ float exp_of(float a) { return __builtin_amdgcn_exp2f(a * 1.44269504088896340736f); }

// NaN: -inf, +inf: the largest number.  (A median of three with -inf as a bound is folded into a minimum, which passes the number in place of a NaN.)
__device__ __forceinline__ float logit(float x) { return x == x ? fminf(x, 3.40282346638528859812e38f) : -INFINITY; }

// Whether the row's logits matter: its hypothesis goes on from a score and a weight that are numbers.
__device__ __forceinline__ bool offers(const nm_beam_desc& d, long row)
{
    const float s = d.scores[row], w = d.weight ? d.weight[row] : 1.0f;
    return __builtin_fabsf(s) < INFINITY && w > 0.0f && w < INFINITY;
}

template <typename T>
__global__ __launch_bounds__(kBeamThreads) void beam_rows_kernel(BeamArgs a)
{
    constexpr int kGroup = 16 / (int)sizeof(T), kGroups = kBeamLane / kGroup;
    typedef T Vec __attribute__((ext_vector_type(kGroup)));
    __shared__ Key s_list[kBeamWaves][64];
    __shared__ float s_max[kBeamWaves];
    __shared__ double s_sum[kBeamWaves];
    const nm_beam_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = d.K;
    const long row = blockIdx.y;
    if (!offers(d, row) || (d.done && d.done[row])) return;   // uniform
    const T* x = static_cast<const T*>(d.logits) + row * d.logits_stride;
    // groups of 16 bytes begin `ahead` elements in front of the row
    const int ahead = (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
    const int v_end = (int)min((long)d.V, (long)(blockIdx.x + 1) * a.chunk - ahead), v_begin = max((int)blockIdx.x * a.chunk - ahead, 0);

    Key list = 0;
    float top = -INFINITY;
    double sum = 0;
    for (long t = (long)blockIdx.x * a.chunk - ahead + wave * kBeamTile; t < v_end; t += kBeamTile * kBeamWaves) {
        float y[kBeamLane];
        const int first = (int)t + lane * kGroup;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const int v = first + i * 64 * kGroup;
            if (v >= v_begin && v + kGroup <= v_end) {
                const Vec w = *reinterpret_cast<const Vec*>(x + v);
#pragma unroll
                for (int e = 0; e < kGroup; ++e) y[i * kGroup + e] = logit((float)w[e]);
            } else {
#pragma unroll
                for (int e = 0; e < kGroup; ++e) y[i * kGroup + e] = v + e >= v_begin && v + e < v_end ? logit((float)x[v + e]) : -INFINITY;
            }
        }
        float m = y[0];
#pragma unroll
        for (int i = 1; i < kBeamLane; ++i) m = fmaxf(m, y[i]);
        const float now = fmaxf(m, top), base = now == -INFINITY ? 0.0f : now;
        float part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kBeamLane; ++i) part[i % 4] += exp_of(y[i] - base);
        sum = sum * (double)exp_of(top - base) + (double)((part[0] + part[1]) + (part[2] + part[3]));
        top = now;
        const Key last = lane_key(list, K - 1);
        if (__any(m > -INFINITY && (!last || m >= logit_of(last)))) {
#pragma unroll
            for (int i = 0; i < kBeamLane; ++i) {
                const int v = first + i / kGroup * 64 * kGroup + i % kGroup;
                list = insert_all(list, y[i] > -INFINITY ? key_of(y[i], v) : 0, K, lane);
            }
        }
    }
    // the lanes' sums, then the wavefronts'
    float m = top;
    for (int step = 32; step; step >>= 1) m = fmaxf(m, __shfl_xor(m, step));
    sum *= (double)exp_of(top - (m == -INFINITY ? 0.0f : m));
    for (int step = 32; step; step >>= 1) sum += __shfl_xor(sum, step);
    s_list[wave][lane] = list;
    if (lane == 0) { s_max[wave] = m; s_sum[wave] = sum; }
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < kBeamWaves; ++w) list = insert_all(list, lane < K ? s_list[w][lane] : 0, K, lane);
    const long part = row * a.chunks + blockIdx.x;
    if (lane < K) a.part_key[part * K + lane] = list;
    if (lane == 0) {
        float all = s_max[0];
        for (int w = 1; w < kBeamWaves; ++w) all = fmaxf(all, s_max[w]);
        double total = 0;
        for (int w = 0; w < kBeamWaves; ++w) total += s_sum[w] * (double)exp_of(s_max[w] - (all == -INFINITY ? 0.0f : all));
        a.part_max[part] = all;
        a.part_sum[part] = total;
    }
}

// A workgroup to a request.
__global__ __launch_bounds__(kBeamThreads) void beam_join_kernel(BeamArgs a)
{
    __shared__ double s_rank[NM_BEAM_MAX][NM_BEAM_MAX], s_total[NM_BEAM_MAX][NM_BEAM_MAX];   // [hypothesis][its candidates]
    __shared__ int s_token[NM_BEAM_MAX][NM_BEAM_MAX];
    const nm_beam_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = d.K, r = blockIdx.x;
    for (int w = wave; w < d.W; w += kBeamWaves) {
        const long row = (long)r * d.W + w;
        double total = -INFINITY;
        int token = -1;
        if (offers(d, row)) {
            if (d.done && d.done[row]) {
                if (lane == 0) { total = d.scores[row]; token = d.end_token; }
            } else {
                const long part = row * a.chunks;
                const float m = lane < a.chunks ? a.part_max[part + lane] : -INFINITY;
                float top = m;
                for (int step = 32; step; step >>= 1) top = fmaxf(top, __shfl_xor(top, step));
                double sum = lane < a.chunks ? a.part_sum[part + lane] * exp((double)m - (double)(top == -INFINITY ? 0.0f : top)) : 0.0;
                for (int step = 32; step; step >>= 1) sum += __shfl_xor(sum, step);
                Key list = 0;
                for (int c = 0; c < a.chunks; ++c) list = insert_all(list, lane < K ? a.part_key[(part + c) * K + lane] : 0, K, lane);
                if (list && lane < K) {
                    total = (double)d.scores[row] + (((double)logit_of(list) - (double)top) - log(sum));
                    token = token_of(list);
                }
            }
        }
        s_total[w][lane] = total;
        s_rank[w][lane] = total == -INFINITY ? total : (d.weight ? (double)d.weight[row] : 1.0) * total;
        s_token[w][lane] = token;
    }
    __syncthreads();
    if (wave) return;
    // lane w has the best candidate of hypothesis w that is left
    int at = 0;
    double head = lane < d.W ? s_rank[lane][0] : -INFINITY;
    for (int k = 0; k < K; ++k) {
        double best = head;
        for (int step = 32; step; step >>= 1) best = fmax(best, __shfl_xor(best, step));
        const int w = __ffsll((long long)__ballot(head == best)) - 1;
        const long out = (long)r * K + k;
        if (best == -INFINITY) {
            if (lane == 0) {
                d.parents[out] = d.tokens[out] = -1;
                d.scores_out[out] = -INFINITY;
                if (d.done_out) d.done_out[out] = 0;
            }
        } else if (lane == w) {
            const long row = (long)r * d.W + w;
            d.parents[out] = (int)row;
            d.tokens[out] = s_token[w][at];
            d.scores_out[out] = (float)s_total[w][at];
            if (d.done_out) d.done_out[out] = (d.done && d.done[row]) || s_token[w][at] == d.end_token;
            ++at;
            head = at < K ? s_rank[w][at] : -INFINITY;
        }
    }
}

// Histories: a few workgroups to a row.
__global__ __launch_bounds__(kBeamThreads) void beam_history_kernel(nm_beam_desc d)
{
    const long row = blockIdx.x;
    const int parent = d.parents[row];
    const int held = parent < 0 ? 0 : min(max(d.history_lens[parent], 0), d.max_history);
    const bool grows = parent >= 0 && held < d.max_history && !(d.done && d.done[parent]);
    int* to = d.history_out + row * d.history_out_stride;
    const int* from = d.history + (long)max(parent, 0) * d.history_stride;
    for (int i = blockIdx.y * kBeamThreads + threadIdx.x; i < held; i += gridDim.y * kBeamThreads) to[i] = from[i];
    if (blockIdx.y == 0 && threadIdx.x == 0) {
        if (grows) to[held] = d.tokens[row];
        d.history_lens_out[row] = held + grows;
    }
}

static int32_t plan_beam(const nm_beam_desc* d, BeamArgs* a, size_t* bytes, const char* what)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "%s: desc is NULL", what);
    if (d->R < 0 || d->W < 1 || d->K < 1 || d->V < 1) return fail(NM_ERR_INVALID_ARG, "%s: bad shape", what);
    if (!float_dtype(d->logits_dtype)) return fail(NM_ERR_INVALID_ARG, "%s: bad logits_dtype", what);
    if (d->W > NM_BEAM_MAX || d->K > NM_BEAM_MAX) return fail(NM_ERR_UNSUPPORTED, "%s: W %d or K %d > %d", what, d->W, d->K, NM_BEAM_MAX);
    if ((int64_t)d->R * d->W > 1 << 20 || d->V > 1 << 26) return fail(NM_ERR_UNSUPPORTED, "%s: R * W > 2^20 or V > 2^26", what);
    *a = BeamArgs{};
    a->d = *d;
    const long rows = (long)d->R * d->W, most = ((long)d->V + 16 + kBeamTile * kBeamWaves - 1) / (kBeamTile * kBeamWaves);
    const long wanted = rows ? (2048 + rows - 1) / rows : 1;
    long chunks = std::min(std::min(most, wanted), (long)kBeamChunks);
    const long step = kBeamTile * kBeamWaves;
    a->chunk = (int)((((long)d->V + 16 + chunks - 1) / chunks + step - 1) / step * step);
    a->chunks = (int)(((long)d->V + 16 + a->chunk - 1) / a->chunk);
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
    queue_kernel(beam_join_kernel, dim3(d->R), dim3(kBeamThreads), 0, s, a);
    if (d->history) {
        const int32_t err = check_hip(hipGetLastError(), "nm_beam_select launch");
        if (err) return err;
        queue_kernel(beam_history_kernel, dim3(d->R * d->K, std::min((d->max_history + 4 * kBeamThreads - 1) / (4 * kBeamThreads), 64)), dim3(kBeamThreads), 0, s, *d);
    }
    return check_hip(hipGetLastError(), "nm_beam_select launch");
}

}  // extern "C"
