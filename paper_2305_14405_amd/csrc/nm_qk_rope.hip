// Norms and rotation of a step's queries and keys, which leave for the cache with the values (nm_qk_norm_rope).
//
// Bound by memory: every element is read once and written once, with some ten operations on it.  A head's elements lie in the registers of
// G lanes, two groups of neighbours to a lane (16 bytes each where sizes and addresses allow) that are each other's partners in the
// rotation, or hold whole pairs: the sum of squares is a butterfly over G lanes, and no element crosses lanes.  The angles belong to the
// token: a workgroup has up to eight tokens, a thread makes the sine and cosine of one of their angles while the first loads are
// under way, and all heads read them from LDS.  An angle is reduced in 64 bits (position * frequency reaches 10^6
// radians, where 32 bits would leave 0.06 of error) and its sine taken in 32.
//   16397 tokens of 32 + 8 + 8 bf16 heads of 128 (403 MB): 93 us, 4.3 TB/s, 80 us at a copy's 5.06 TB/s; vector instructions are issued in 46 %
// of the cycles.  8 bytes of either half at a time and one token to a workgroup took 114.  One token of 36 heads: 3.5 us, a launch and three dependent loads.
#include "nm_decode.h"

namespace nm {

constexpr int kRopeThreads = 256;

constexpr int kRopeTokens = 8;

struct QkArgs {
    nm_qk_desc d;
    int shift;          // log2 of page_size
    int heads;          // heads a token has here: hq + hk, and hk more of values where there is a cache
    int tokens;         // of a workgroup, up to kRopeTokens
    int per_block;      // heads of each that a workgroup goes through
    FastDiv by_heads;   // by that
    unsigned slots;     // num_pages * page_size
    float inv_d;
};

// cos and sin of position * inv_freq: whole turns are taken off in binary64.
__device__ __forceinline__ float2 turn(int position, float inv_freq)
{
    double a = (double)position * (double)inv_freq * 0.15915494309189533577;   // turns
    a -= rint(a);
    float s, c;
    sincospif((float)(a * 2.0), &s, &c);
    return make_float2(c, s);
}

// Where head h of token t lies, and what is to be done with it.
template <typename T>
struct Head {
    const T* in;
    int kind;           // 0 query, 1 key, 2 value
    int h;              // among its kind
    __device__ Head(const nm_qk_desc& d, int t, int head)
    {
        kind = head < d.hq ? 0 : head < d.hq + d.hk ? 1 : 2;
        h = head - (kind == 0 ? 0 : kind == 1 ? d.hq : d.hq + d.hk);
        const void* base = kind == 0 ? d.q : kind == 1 ? d.k : d.v;
        const long stride = kind == 0 ? d.q_stride : kind == 1 ? d.k_stride : d.v_stride;
        in = static_cast<const T*>(base) + t * stride + (long)h * d.d;
    }
};

__device__ __forceinline__ long cache_at(const nm_qk_desc& d, int shift, int slot, int h)
{
    return (long)(slot >> shift) * d.page_stride + (long)(slot & (d.page_size - 1)) * d.slot_stride + (long)h * d.head_stride;
}

// E neighbours at once: d and rot multiples of 2 E.
template <typename T, int E, int G, bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_kernel(QkArgs a)
{
    typedef T Vec __attribute__((ext_vector_type(E)));
    const nm_qk_desc& d = a.d;
    __shared__ float2 s_cs[kRopeTokens][128];
    __shared__ int s_slot[kRopeTokens];
    const int tid = threadIdx.x, t0 = blockIdx.x * a.tokens, tokens = min(a.tokens, d.T - t0);
    const int l = tid % G, half = d.rot / 2, rest = (d.d - d.rot) / 2;
    const bool mine = l < d.d / (2 * E);
    // the lane's two groups: of either half of the head (interleaved), of the rotated part, or of what is behind it
    const bool turned = l * 2 * E < d.rot;
    const int e0 = kInterleaved ? l * E : turned ? l * E : d.rot + l * E - half, e1 = e0 + (kInterleaved ? d.d / 2 : turned ? half : rest);
    const int first = blockIdx.y * a.per_block, per = min(a.per_block, a.heads - first), all = tokens * a.per_block;

    // item i: head first + i % per_block of token i / per_block (the last block of heads may be shorter: its items are skipped)
    struct Item { int t, head; bool there; };
    auto item_of = [&](int i) {
        const int t = (int)quotient((unsigned)i, a.by_heads), head = i - t * a.per_block;
        return Item{t, first + head, t < tokens && head < per};
    };
    auto load = [&](const Item& it, Vec& x0, Vec& x1) {
        const int t = min(it.t, tokens - 1), head = min(it.head, first + per - 1);
        const Head<T> at(d, t0 + t, head);
        const T* from = at.in;
        x0 = *reinterpret_cast<const Vec*>(from + (mine ? e0 : 0));
        x1 = *reinterpret_cast<const Vec*>(from + (mine ? e1 : 0));
    };
    int i = tid / G;
    Item now = item_of(i);
    Vec n0, n1;
    load(now, n0, n1);

    typedef float Gamma __attribute__((ext_vector_type(4), aligned(4)));
    float gq[2][E], gk[2][E];
    if (d.flags & NM_QK_NORM) {
        auto fetch_gamma = [&](const float* gamma, float (&g)[2][E]) {
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const Gamma v = gamma ? *reinterpret_cast<const Gamma*>(gamma + (mine ? (part ? e1 : e0) + e : 0)) : Gamma{1, 1, 1, 1};
#pragma unroll
                    for (int n = 0; n < 4; ++n) g[part][e + n] = v[n];
                }
        };
        fetch_gamma(d.q_gamma, gq);
        fetch_gamma(d.k_gamma, gk);
    }
    for (int p = tid; p < tokens * half; p += kRopeThreads) {
        const int t = p / half, angle = p - t * half;
        s_cs[t][angle] = turn(d.positions[t0 + t], d.inv_freq[angle]);
    }
    if (tid < tokens) s_slot[tid] = d.k_cache ? d.slots[t0 + tid] : -1;
    __syncthreads();

    for (; i - tid / G < all; i += kRopeThreads / G) {
        const Item it = now;
        float x[2][E];
#pragma unroll
        for (int e = 0; e < E; ++e) { x[0][e] = mine ? (float)n0[e] : 0.0f; x[1][e] = mine ? (float)n1[e] : 0.0f; }
        now = item_of(i + kRopeThreads / G);
        load(now, n0, n1);
        if (!it.there) continue;                              // a whole group of lanes, as below
        const Head<T> at(d, t0 + it.t, it.head);
        if (at.kind < 2) {
            if (d.flags & NM_QK_NORM) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) sum = __builtin_fmaf(x[0][e], x[0][e], __builtin_fmaf(x[1][e], x[1][e], sum));
                sum = group_sum<G>(sum);
                const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, a.inv_d, d.eps));
                const bool query = at.kind == 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x[0][e] = x[0][e] * r * (query ? gq[0][e] : gk[0][e]);
                    x[1][e] = x[1][e] * r * (query ? gq[1][e] : gk[1][e]);
                }
            }
            if (kInterleaved) {
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const int angle = ((part ? e1 : e0) + e) / 2;
                        const float2 cs = mine && angle < half ? s_cs[it.t][angle] : make_float2(1.0f, 0.0f);
                        const float p = x[part][e], q = x[part][e + 1];
                        x[part][e] = __builtin_fmaf(p, cs.x, -(q * cs.y));
                        x[part][e + 1] = __builtin_fmaf(q, cs.x, p * cs.y);
                    }
            } else if (turned && mine) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float2 cs = s_cs[it.t][l * E + e];
                    const float p = x[0][e], q = x[1][e];
                    x[0][e] = __builtin_fmaf(p, cs.x, -(q * cs.y));
                    x[1][e] = __builtin_fmaf(q, cs.x, p * cs.y);
                }
            }
        }
        const int slot = s_slot[it.t];
        const bool kept = (unsigned)slot < a.slots;
        if (!mine) continue;
        if (at.kind == 0 || (at.kind == 1 && d.k_out)) {
            void* out = at.kind == 0 ? d.q_out : d.k_out;
            const long to = (t0 + it.t) * (at.kind == 0 ? d.q_out_stride : d.k_out_stride) + (long)at.h * d.d;
            store_run<E>(out, d.out_dtype, to + e0, x[0], 0.0f);
            store_run<E>(out, d.out_dtype, to + e1, x[1], 0.0f);
        }
        if (at.kind > 0 && kept) {
            const long to = cache_at(d, a.shift, slot, at.h);
            void* cache = at.kind == 1 ? d.k_cache : d.v_cache;
            const float inv = d.cache_dtype == NM_DT_I8 ? (at.kind == 1 ? d.k_inv_scale : d.v_inv_scale)[at.h] : 0.0f;
            store_run<E>(cache, d.cache_dtype, to + e0, x[0], inv);
            store_run<E>(cache, d.cache_dtype, to + e1, x[1], inv);
        }
    }
}

// Any head size and alignment: a wavefront to a head, two pairs and four elements behind the rotated ones to a lane.
template <typename T>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_any_kernel(QkArgs a)
{
    const nm_qk_desc& d = a.d;
    const int t = blockIdx.x, lane = threadIdx.x & 63, half = d.rot / 2;
    const bool inter = d.flags & NM_ROPE_INTERLEAVED;
    const int slot = d.k_cache ? d.slots[t] : -1;
    const bool kept = (unsigned)slot < a.slots;
    float2 cs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = lane + 64 * i;
        cs[i] = p < half ? turn(d.positions[t], d.inv_freq[p]) : make_float2(1.0f, 0.0f);
    }
    // element of register i: pairs in 0 .. 3 (first and second of pair lane, then of pair lane + 64), the rest in 4 .. 7; d.d: none
    int e[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = lane + 64 * i;
        e[2 * i] = p < half ? (inter ? 2 * p : p) : d.d;
        e[2 * i + 1] = p < half ? (inter ? 2 * p + 1 : p + half) : d.d;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) e[4 + i] = d.rot + lane + 64 * i;
    for (int head = blockIdx.y * a.per_block + (threadIdx.x >> 6); head < min((int)(blockIdx.y + 1) * a.per_block, a.heads); head += kRopeThreads / 64) {
        const Head<T> at(d, t, head);
        if (at.kind > 0 && !kept && !(at.kind == 1 && d.k_out)) continue;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e[i] < d.d ? (float)at.in[e[i]] : 0.0f;
        if (at.kind < 2 && (d.flags & NM_QK_NORM)) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
            const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(group_sum<64>(sum), a.inv_d, d.eps));
            const float* gamma = at.kind == 0 ? d.q_gamma : d.k_gamma;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (gamma && e[i] < d.d ? gamma[e[i]] : 1.0f);
        }
        if (at.kind < 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float p = x[2 * i], q = x[2 * i + 1];
                x[2 * i] = p * cs[i].x - q * cs[i].y;
                x[2 * i + 1] = q * cs[i].x + p * cs[i].y;
            }
        }
        const bool out = at.kind == 0 || (at.kind == 1 && d.k_out);
        void* to = at.kind == 0 ? d.q_out : d.k_out;
        const long to_at = t * (at.kind == 0 ? d.q_out_stride : d.k_out_stride) + (long)at.h * d.d;
        void* cache = at.kind == 1 ? d.k_cache : d.v_cache;
        const long at_cache = kept ? cache_at(d, a.shift, slot, at.h) : 0;
        const float inv = at.kind > 0 && kept && d.cache_dtype == NM_DT_I8 ? (at.kind == 1 ? d.k_inv_scale : d.v_inv_scale)[at.h] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e[i] < d.d) {
                if (out) store1(to, d.out_dtype, to_at + e[i], x[i], 0.0f);
                if (at.kind > 0 && kept) store1(cache, d.cache_dtype, at_cache + e[i], x[i], inv);
            }
    }
}

template <typename T, int E, int G>
static void launch_qk(const QkArgs& a, dim3 grid, hipStream_t s)
{
    if (a.d.flags & NM_ROPE_INTERLEAVED) queue_kernel(qk_rope_kernel<T, E, G, true>, grid, dim3(kRopeThreads), 0, s, a);
    else queue_kernel(qk_rope_kernel<T, E, G, false>, grid, dim3(kRopeThreads), 0, s, a);
}
template <typename T, int E>
static void launch_qk_groups(QkArgs a, hipStream_t s)
{
    int G = 4;
    while (G < a.d.d / (2 * E)) G *= 2;
    // Few tokens: a workgroup to a round of heads.  More: all heads of a token, of two or four, which share the sines, the gammas and the
    // start of a workgroup.  (40 + 8 heads of 128 in bf16, us by a round / 1 / 2 / 4 / 8 tokens: 256 tokens 4.6 5.3 6.3 9.5 16, 1000 11 8.9 9.6
    // 12 19, 2048 18 14.7 12.1 14 20, 4096 42 34 28 26 34, 16397 158 122 97 93 99.)  And as many tokens as fill a round.
    const int round = kRopeThreads / G;
    a.tokens = a.d.T >= 4096 ? 4 : a.d.T >= 1536 ? 2 : 1;
    if (round / a.heads > a.tokens) a.tokens = round / a.heads < kRopeTokens ? round / a.heads : kRopeTokens;
    a.per_block = a.d.T >= 768 || a.heads < round ? a.heads : round;
    a.by_heads = fast_div(a.per_block);
    const dim3 grid((a.d.T + a.tokens - 1) / a.tokens, (a.heads + a.per_block - 1) / a.per_block);
    if (G == 4) launch_qk<T, E, 4>(a, grid, s);
    else if (G == 8) launch_qk<T, E, 8>(a, grid, s);
    else if (G == 16) launch_qk<T, E, 16>(a, grid, s);
    else if constexpr (E == 4) launch_qk<T, E, 32>(a, grid, s);
}
// run: neighbours that sizes and addresses allow at once, 8 or 4, or 0.
template <typename T>
static void launch_qk_t(QkArgs a, int run, hipStream_t s)
{
    if (sizeof(T) == 2 && run == 8) {
        launch_qk_groups<T, 8>(a, s);
    } else if (run) {
        launch_qk_groups<T, 4>(a, s);
    } else {
        a.per_block = a.d.T >= 1024 ? a.heads : kRopeThreads / 64;
        queue_kernel(qk_rope_any_kernel<T>, dim3(a.d.T, (a.heads + a.per_block - 1) / a.per_block), dim3(kRopeThreads), 0, s, a);
    }
}

}  // namespace nm

using namespace nm;

extern "C" int32_t nm_qk_norm_rope(const nm_qk_desc* d, void* stream)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: desc is NULL");
    if (d->T < 0 || d->hq < 1 || d->hk < 1 || d->d < 1 || d->rot < 0 || d->rot > d->d || d->rot % 2)
        return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: bad shape");
    if (d->d > 256) return fail(NM_ERR_UNSUPPORTED, "nm_qk_norm_rope: d %d > 256", d->d);
    if (d->T > 1 << 23) return fail(NM_ERR_UNSUPPORTED, "nm_qk_norm_rope: T %d > 2^23", d->T);
    if ((int64_t)d->hq + 2 * (int64_t)d->hk > 65535) return fail(NM_ERR_UNSUPPORTED, "nm_qk_norm_rope: more than 65535 heads");
    if (d->flags & ~(NM_QK_NORM | NM_ROPE_INTERLEAVED)) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: unknown flag");
    if (!float_dtype(d->in_dtype) || !float_dtype(d->out_dtype)) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: bad in_dtype or out_dtype");
    if ((d->flags & NM_QK_NORM) && !(d->eps >= 0.0f && d->eps <= 3e38f)) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: eps must be finite and not negative");
    if (!d->k_cache != !d->v_cache) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: one cache without the other");
    const int64_t wq = (int64_t)d->hq * d->d, wk = (int64_t)d->hk * d->d;
    if (d->q_stride < wq || d->k_stride < wk || (d->k_cache && d->v_stride < wk) || d->q_out_stride < wq || (d->k_out && d->k_out_stride < wk))
        return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: a stride is shorter than a token's heads");
    int shift = 0;
    if (d->k_cache) {
        if (!float_dtype(d->cache_dtype) && d->cache_dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: bad cache_dtype");
        shift = page_shift(d->page_size);
        if (shift < 0) return fail(NM_ERR_UNSUPPORTED, "nm_qk_norm_rope: page_size %d is no power of two up to 65536", d->page_size);
        if (d->num_pages < 0 || d->page_stride < 0 || d->slot_stride < 0 || d->head_stride < 0)
            return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: negative size of the cache");
        if ((int64_t)d->num_pages << shift > 0x7fffffffLL) return fail(NM_ERR_UNSUPPORTED, "nm_qk_norm_rope: num_pages * page_size >= 2^31");
        if (d->cache_dtype == NM_DT_I8 && (!d->k_inv_scale || !d->v_inv_scale)) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: int8 cache without scales");
    }
    if (d->T == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->q || !d->k || !d->q_out || (d->k_cache && (!d->v || !d->slots))) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: NULL argument");
    if (d->rot && (!d->positions || !d->inv_freq)) return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: rotation without positions or inv_freq");
    if ((d->q_out == d->q && (d->out_dtype != d->in_dtype || d->q_out_stride != d->q_stride)) ||
        (d->k_out == d->k && (d->out_dtype != d->in_dtype || d->k_out_stride != d->k_stride)))
        return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: in place with another type or stride");
    const void* v = d->k_cache ? d->v : nullptr;              // read only then
    const std::initializer_list<const void*> read = {v, d->q_gamma, d->k_gamma, d->positions, d->inv_freq, d->slots, d->k_inv_scale, d->v_inv_scale};
    if (begins_as(d->q_out, read) || begins_as(d->q_out, {d->k, d->k_out, d->k_cache, d->v_cache}) || begins_as(d->k_out, read) ||
        begins_as(d->k_out, {d->q, d->k_cache, d->v_cache}) || begins_as(d->k_cache, read) || begins_as(d->k_cache, {d->q, d->k, d->v_cache}) ||
        begins_as(d->v_cache, read) || begins_as(d->v_cache, {d->q, d->k}))
        return fail(NM_ERR_INVALID_ARG, "nm_qk_norm_rope: an output is an input or another output");
    QkArgs a{};
    a.d = *d;
    a.shift = shift;
    a.inv_d = 1.0f / (float)d->d;
    a.heads = d->hq + d->hk + (d->k_cache ? d->hk : 0);
    a.slots = (unsigned)((int64_t)d->num_pages << shift);
    auto runs_of = [&](int n) {
        const bool cache = !d->k_cache || (aligned_rows(d->k_cache, d->page_stride, d->cache_dtype, n) && aligned_rows(d->v_cache, d->slot_stride, d->cache_dtype, n) &&
                                           d->head_stride % n == 0 && aligned_rows(d->v, d->v_stride, d->in_dtype, n));
        return d->d % (2 * n) == 0 && d->rot % (2 * n) == 0 && cache && aligned_rows(d->q, d->q_stride, d->in_dtype, n) &&
               aligned_rows(d->k, d->k_stride, d->in_dtype, n) && aligned_rows(d->q_out, d->q_out_stride, d->out_dtype, n) &&
               (!d->k_out || aligned_rows(d->k_out, d->k_out_stride, d->out_dtype, n));
    };
    const int run = d->in_dtype != NM_DT_F32 && runs_of(8) ? 8 : runs_of(4) ? 4 : 0;
    if (d->in_dtype == NM_DT_F32) launch_qk_t<float>(a, run, (hipStream_t)stream);
    else if (d->in_dtype == NM_DT_BF16) launch_qk_t<bf16>(a, run, (hipStream_t)stream);
    else launch_qk_t<f16>(a, run, (hipStream_t)stream);
    return check_hip(hipGetLastError(), "nm_qk_norm_rope launch");
}
