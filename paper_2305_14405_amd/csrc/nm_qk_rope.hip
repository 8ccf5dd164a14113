// Norms and rotation of a step's queries and keys, which leave for the cache with the values (nm_qk_norm_rope).
//
// Bound by memory: every element is read once and written once, with some ten operations on it.  A head's elements lie in the registers of
// G lanes, eight to a lane as two groups of four whose members are each other's partners in the rotation (or neighbours, interleaved): the
// sum of squares is a butterfly over G lanes, and no element crosses lanes.  The angles belong to the token: one
// workgroup has (some of) a token's heads, rot / 2 of its threads make the sines and cosines while the first loads are under way, and all
// heads read them from LDS.  An angle is reduced in 64 bits (position * frequency reaches 10^6 radians, where 32 bits would
// leave 0.06 of error) and its sine taken in 32.
#include "nm_decode.h"

namespace nm {

constexpr int kRopeThreads = 256;

struct QkArgs {
    nm_qk_desc d;
    int shift;          // log2 of page_size
    int heads;          // heads a token has here: hq + hk, and hk more of values where there is a cache
    int per_block;      // heads a workgroup goes through
    unsigned slots;     // num_pages * page_size
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

// Whole groups of elements: d and rot multiples of 8.
template <typename T, int G, bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_kernel(QkArgs a)
{
    const nm_qk_desc& d = a.d;
    __shared__ float2 s_cs[128];
    const int tid = threadIdx.x, t = blockIdx.x;
    const int l = tid % G, lanes = d.d / 8, half = d.rot / 2;
    const bool mine = l < lanes;
    // the lane's two groups of four elements
    const bool turned = l * 8 < d.rot;
    const int e0 = kInterleaved || !turned ? l * 8 : l * 4, e1 = kInterleaved || !turned ? l * 8 + 4 : half + l * 4;
    const int slot = d.k_cache ? d.slots[t] : -1;
    const bool kept = (unsigned)slot < a.slots;
    const int first = blockIdx.y * a.per_block, last = min(first + a.per_block, a.heads);
    auto wanted = [&](int head) { return head < last && mine && (head < d.hq || kept || (head < d.hq + d.hk && d.k_out)); };

    int head = first + tid / G;
    v4f x0{}, x1{};
    if (wanted(head)) {
        const Head<T> at(d, t, head);
        x0 = load4(at.in + e0);
        x1 = load4(at.in + e1);
    }
    if (half) {
        const int position = d.positions[t];
        if (tid < half) s_cs[tid] = turn(position, d.inv_freq[tid]);
        __syncthreads();
    }
    float2 cs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = turned && mine ? s_cs[l * 4 + i] : make_float2(1.0f, 0.0f);

    for (; head - tid / G < last; head += kRopeThreads / G) {
        const Head<T> at(d, t, head);
        v4f n0{}, n1{};
        const int next = head + kRopeThreads / G;
        if (wanted(next)) {
            const Head<T> to(d, t, next);
            n0 = load4(to.in + e0);
            n1 = load4(to.in + e1);
        }
        if (at.kind < 2 && (d.flags & NM_QK_NORM)) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = __builtin_fmaf(x0[i], x0[i], __builtin_fmaf(x1[i], x1[i], sum));
            sum = group_sum<G>(sum);
            const float r = 1.0f / sqrtf(sum / (float)d.d + d.eps);
            const float* gamma = at.kind == 0 ? d.q_gamma : d.k_gamma;
            v4f g0 = {1, 1, 1, 1}, g1 = g0;
            if (gamma && mine) {
#pragma unroll
                for (int i = 0; i < 4; ++i) { g0[i] = gamma[e0 + i]; g1[i] = gamma[e1 + i]; }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { x0[i] = x0[i] * r * g0[i]; x1[i] = x1[i] * r * g1[i]; }
        }
        if (at.kind < 2 && half) {
            if (kInterleaved) {
                const v4f y0 = x0, y1 = x1;
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float2 p = cs[i / 2], q = cs[2 + i / 2];
                    x0[i] = y0[i] * p.x - y0[i + 1] * p.y;
                    x0[i + 1] = y0[i + 1] * p.x + y0[i] * p.y;
                    x1[i] = y1[i] * q.x - y1[i + 1] * q.y;
                    x1[i + 1] = y1[i + 1] * q.x + y1[i] * q.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = x0[i], q = x1[i];
                    x0[i] = p * cs[i].x - q * cs[i].y;
                    x1[i] = q * cs[i].x + p * cs[i].y;
                }
            }
        }
        if (wanted(head)) {
            if (at.kind == 0 || (at.kind == 1 && d.k_out)) {
                void* out = at.kind == 0 ? d.q_out : d.k_out;
                const long to = t * (at.kind == 0 ? d.q_out_stride : d.k_out_stride) + (long)at.h * d.d;
                store4(out, d.out_dtype, to + e0, x0, 0.0f);
                store4(out, d.out_dtype, to + e1, x1, 0.0f);
            }
            if (at.kind > 0 && kept) {
                const long to = cache_at(d, a.shift, slot, at.h);
                void* cache = at.kind == 1 ? d.k_cache : d.v_cache;
                const float inv = d.cache_dtype == NM_DT_I8 ? (at.kind == 1 ? d.k_inv_scale : d.v_inv_scale)[at.h] : 0.0f;
                store4(cache, d.cache_dtype, to + e0, x0, inv);
                store4(cache, d.cache_dtype, to + e1, x1, inv);
            }
        }
        x0 = n0;
        x1 = n1;
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
            const float r = 1.0f / sqrtf(group_sum<64>(sum) / (float)d.d + d.eps);
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

template <typename T, int G>
static void launch_qk(const QkArgs& a, dim3 grid, hipStream_t s)
{
    if (a.d.flags & NM_ROPE_INTERLEAVED) queue_kernel(qk_rope_kernel<T, G, true>, grid, dim3(kRopeThreads), 0, s, a);
    else queue_kernel(qk_rope_kernel<T, G, false>, grid, dim3(kRopeThreads), 0, s, a);
}

template <typename T>
static void launch_qk_t(QkArgs a, bool vec, hipStream_t s)
{
    int G = 64;
    if (vec)
        for (G = 4; G < a.d.d / 8; G *= 2) {}
    // workgroups that go through some heads of a token each: all of them where the tokens alone fill the GPU's 256 CUs a few times over, else
    // one round of heads
    const int round = kRopeThreads / G;
    a.per_block = a.d.T >= 1024 ? a.heads : round;
    const dim3 grid(a.d.T, (a.heads + a.per_block - 1) / a.per_block);
    if (!vec) queue_kernel(qk_rope_any_kernel<T>, grid, dim3(kRopeThreads), 0, s, a);
    else if (G == 4) launch_qk<T, 4>(a, grid, s);
    else if (G == 8) launch_qk<T, 8>(a, grid, s);
    else if (G == 16) launch_qk<T, 16>(a, grid, s);
    else launch_qk<T, 32>(a, grid, s);
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
    QkArgs a{};
    a.d = *d;
    a.shift = shift;
    a.heads = d->hq + d->hk + (d->k_cache ? d->hk : 0);
    a.slots = (unsigned)((int64_t)d->num_pages << shift);
    const bool cache_vec = !d->k_cache || (aligned_rows(d->k_cache, d->page_stride, d->cache_dtype, 4) && aligned_rows(d->v_cache, d->slot_stride, d->cache_dtype, 4) &&
                                           d->head_stride % 4 == 0 && aligned_rows(d->v, d->v_stride, d->in_dtype, 4));
    const bool vec = d->d % 8 == 0 && d->rot % 8 == 0 && cache_vec && aligned_rows(d->q, d->q_stride, d->in_dtype, 4) &&
                     aligned_rows(d->k, d->k_stride, d->in_dtype, 4) && aligned_rows(d->q_out, d->q_out_stride, d->out_dtype, 4) &&
                     (!d->k_out || aligned_rows(d->k_out, d->k_out_stride, d->out_dtype, 4));
    if (d->in_dtype == NM_DT_F32) launch_qk_t<float>(a, vec, (hipStream_t)stream);
    else if (d->in_dtype == NM_DT_BF16) launch_qk_t<bf16>(a, vec, (hipStream_t)stream);
    else launch_qk_t<f16>(a, vec, (hipStream_t)stream);
    return check_hip(hipGetLastError(), "nm_qk_norm_rope launch");
}
