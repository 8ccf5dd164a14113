// Attention of one new token per request over a paged cache (nm_paged_attention).
//
// Bound by memory: every key and value is read once, with 4 * (query heads of its group) operations an element.  A workgroup has one
// request's key head, up to 16 query heads of its group, and a piece of the length; its four wavefronts walk that piece's tiles of 32
// positions in turn, each with a running maximum, sum and output of its own, and are joined at the end through LDS; pieces are joined
// by a second kernel.  One tile's keys and values are on their way into registers while the one before is computed.
//   Scores: keys are the rows of the 16x16x32 matrix instruction, query heads its columns, so a lane has eight positions of one head:
// its maximum and sum are in-lane steps and two across lanes.  Those registers are already the second product's operand: the contraction
// index of a matrix instruction may be permuted, so "row 4 j + i of the first, then of the second 16 keys" is what lane group j contributes, and
// the values are fetched from LDS in that order by the transposing read.  Output: columns are heads again, so the rescaling factor
// is in the lane that needs it.
//   Precision: scores and sums fp32; exp(s - m) goes into the second product as two terms of 16 bits (2^-17 of itself, below what a 16-bit result
// shows; three terms where the result is fp32), queries that are no 16-bit numbers of the cache's type as three terms of theirs, scaled by a power of two
// so that nothing overflows.  The matrix cores have 20 times the time this needs.
#include "nm_decode.h"

namespace nm {

typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
constexpr int kTile = 32;                       // positions a wavefront takes at once
constexpr int kRound = kTile * kPagedWaves;     // and a workgroup

struct PagedArgs {
    nm_paged_desc d;
    int shift;            // log2 of page_size
    int group;            // query heads of a key head
    int groups;           // of up to 16 of them
    int piece;            // positions of a piece of the length
    int pieces;           // of the longest there can be
    float* part_o;        // [B, hq, pieces, d] not yet divided by the sum; null where there is one piece
    float2* part_ml;      // [B, hq, pieces]: maximum (of scores in units of log 2) and sum
};

template <typename C> struct Mfma;
template <> struct Mfma<bf16> {
    typedef bf16 T;
    static __device__ __forceinline__ v4f mma(v8s a, v8s b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0); }
};
template <> struct Mfma<f16> {
    typedef f16 T;
    static __device__ __forceinline__ v4f mma(v8s a, v8s b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0); }
};
template <> struct Mfma<int8_t> : Mfma<bf16> {};   // codes are exact in bf16

// 16 bytes of a cache row as elements of the matrix instructions' type, to LDS.
template <typename C>
__device__ __forceinline__ void put(short* to, v4u w)
{
    *reinterpret_cast<v4u*>(to) = w;
}
template <>
__device__ __forceinline__ void put<int8_t>(short* to, v4u w)
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        v4u o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned x = w[half * 2 + i / 2] >> (i % 2 * 16);
            const unsigned a = __float_as_uint((float)(int8_t)x), b = __float_as_uint((float)(int8_t)(x >> 8));
            o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);   // the upper halves: small integers have no bits below
        }
        *reinterpret_cast<v4u*>(to + half * 8) = o;
    }
}

// C: type of the cache; DP: d rounded up to 64, 128 or 256; kTerms: of the weights (2 or 3); of a query (1 or 3).
template <typename C, int DP, int kQ, int kP>
__global__ __launch_bounds__(kPagedThreads) void paged_attention_kernel(PagedArgs a)
{
    typedef typename Mfma<C>::T T;
    constexpr int kRowPieces = DP * (int)sizeof(C) / 16;      // 16-byte pieces of a row: lanes to a row
    constexpr int kRowsAtOnce = 64 / kRowPieces, kLoads = kTile / kRowsAtOnce;
    constexpr int kStride = DP + 8;                           // elements between rows in LDS
    constexpr int kSteps = DP / 32, kBlocks = DP / 16;
    constexpr float kLift = std::is_same<C, f16>::value ? 10.0f : 0.0f;   // fp16 weights are held times 2^10, where small ones have more bits
    __shared__ __attribute__((aligned(16))) union {
        short tile[kPagedWaves][kTile * kStride];
        float o[kPagedWaves][16][DP];
    } s;
    __shared__ __attribute__((aligned(16))) short s_q[kQ][16 * kStride];
    __shared__ float s_qscale[16], s_m[kPagedWaves][16], s_l[kPagedWaves][16];

    const nm_paged_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int id = blockIdx.x;
    const int sub = id % a.groups; id /= a.groups;
    const int g = id % d.hk; id /= d.hk;
    const int b = id % d.B, piece = id / d.B;

    const long most = (long)d.max_pages << a.shift;
    const int n = (int)min((long)max(d.lens[b], 0), most);
    const int low = d.window ? max(n - d.window, 0) : 0;
    const int k0 = low + piece * a.piece, k1 = min(k0 + a.piece, n);   // piece * a.piece < pieces * a.piece < 2^31
    const int h0 = g * a.group + sub * 16, heads = min(a.group - sub * 16, 16);
    if (k0 >= k1 && !(piece == 0 && !a.part_ml)) return;               // nothing here, and the joining kernel knows it

    // queries: 16 rows (zeros behind the group's), 16 lanes each
    {
        const int row = tid >> 4, c0 = tid & 15;
        float x[DP / 16], top = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int c = c0 + 16 * i;
            const long at = b * d.q_stride + (long)(h0 + row) * d.d + c;
            const bool there = row < heads && c < d.d;
            x[i] = !there ? 0.0f : d.q_dtype == NM_DT_F32 ? static_cast<const float*>(d.q)[at] : d.q_dtype == NM_DT_BF16 ? (float)static_cast<const bf16*>(d.q)[at]
                                                                                                                        : (float)static_cast<const f16*>(d.q)[at];
            top = fmaxf(top, fabsf(x[i]));
        }
        float down = 1.0f, up = 1.0f;
        if (kQ > 1) {
            top = __int_as_float(group_reduce<16>(__float_as_int(top), MaxF32{}));
            const int e = (int)(__float_as_uint(top) >> 23) - 127;     // top in [2^e, 2^(e + 1)): the row goes below 2
            const int by = max(-126, min(e, 126));
            down = __uint_as_float((unsigned)(127 - by) << 23);
            up = __uint_as_float((unsigned)(127 + by) << 23);
        }
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            float rest = x[i] * down;
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
                const T t = (T)rest;
                rest -= (float)t;
                s_q[q][row * kStride + c0 + 16 * i] = __builtin_bit_cast(short, t);
            }
        }
        if (c0 == 0) s_qscale[row] = up;
    }
    __syncthreads();

    const int column = lane & 15, j = lane >> 4;              // head (and row of an operand), lane group
    const float factor = d.scale * 1.44269504088896340736f * s_qscale[column] * (sizeof(C) == 1 ? d.k_scale[g] : 1.0f);
    const int row_piece = lane % kRowPieces, row_first = lane / kRowPieces;
    const bool in_row = row_piece * (16 / (int)sizeof(C)) < d.d;
    const C* kbase = static_cast<const C*>(d.k_cache) + (long)g * d.head_stride + row_piece * (16 / (int)sizeof(C));
    const C* vbase = static_cast<const C*>(d.v_cache) + (long)g * d.head_stride + row_piece * (16 / (int)sizeof(C));
    const int* table = d.block_table + b * d.table_stride;
    short* tile = s.tile[wave];

    // a tile's place: lane l < 32 has position l's offset in the cache (elements), or none
    auto entry_of = [&](int t0) { const int k = t0 + (lane & 31); return k < k1 ? table[k >> a.shift] : -1; };
    auto offset_of = [&](int t0, int entry, unsigned& valid) -> long {
        const int k = t0 + (lane & 31);
        const bool ok = entry >= 0 && entry < d.num_pages;
        valid = (unsigned)__ballot(ok);
        return ok ? (long)entry * d.page_stride + (long)(k & (d.page_size - 1)) * d.slot_stride : 0;
    };
    auto fetch = [&](const C* base, long offset, unsigned valid, v4u (&to)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = i * kRowsAtOnce + row_first;
            const long at = __shfl(offset, row);
            to[i] = v4u{};
            if ((valid >> row & 1) && in_row) to[i] = *reinterpret_cast<const v4u*>(base + at);
        }
    };
    auto stage = [&](const v4u (&from)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) put<C>(tile + (i * kRowsAtOnce + row_first) * kStride + row_piece * (16 / (int)sizeof(C)), from[i]);
    };

    v4f o[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) o[i] = v4f{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    int t0 = k0 + wave * kTile;
    v4u kr[kLoads], vr[kLoads];
    unsigned valid = 0;
    int entry = entry_of(t0);
    {
        const long offset = offset_of(t0, entry, valid);
        fetch(kbase, offset, valid, kr);
        fetch(vbase, offset, valid, vr);
    }
    entry = entry_of(t0 + kRound);
    for (; t0 < k1; t0 += kRound) {
        unsigned next_valid;
        const long next = offset_of(t0 + kRound, entry, next_valid);
        entry = entry_of(t0 + 2 * kRound);
        // scores
        stage(kr);
        fetch(kbase, next, next_valid, kr);
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
                    sc[blk] = Mfma<C>::mma(ka, qb, sc[blk]);
                }
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = sc[i / 4][i % 4] * factor;
            sc[i / 4][i % 4] = (valid >> (i / 4 * 16 + j * 4 + i % 4) & 1) ? x : -INFINITY;
            top = fmaxf(top, sc[i / 4][i % 4]);
        }
        top = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(top), MaxF32{}), MaxF32{}));
        const float base = top == -INFINITY ? 0.0f : top;
        const float shrink = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= shrink;
        v8s p[kP];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float e = __builtin_amdgcn_exp2f(sc[i / 4][i % 4] - (base - kLift));
            l += e;
#pragma unroll
            for (int q = 0; q < kP; ++q) {
                const T t = (T)e;
                e -= (float)t;
                p[q][i] = __builtin_bit_cast(short, t);
            }
        }
        // values
        stage(vr);
        fetch(vbase, next, next_valid, vr);
#pragma unroll
        for (int blk = 0; blk < kBlocks; ++blk) {
            const short* at = tile + (j * 4 + column / 4) * kStride + blk * 16 + column % 4 * 4;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 16 * kStride));
            const v8s va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[blk][i] *= shrink;
#pragma unroll
            for (int q = kP - 1; q >= 0; --q) o[blk] = Mfma<C>::mma(va, p[q], o[blk]);
        }
        valid = next_valid;
    }
    l = __int_as_float(butterfly_step<32>(butterfly_step<16>(__float_as_int(l), AddF32{}), AddF32{}));

    // the four wavefronts' results as one
    if (j == 0) { s_m[wave][column] = m; s_l[wave][column] = l; }
    __syncthreads();                                          // also: no tile is read any more
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, s_m[w][column]);
    const float base = top == -INFINITY ? 0.0f : top;
    const float mine = __builtin_amdgcn_exp2f(m - base - kLift);
#pragma unroll
    for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
        for (int i = 0; i < 4; ++i) s.o[wave][column][blk * 16 + j * 4 + i] = o[blk][i] * mine;
    __syncthreads();
    const float vscale = sizeof(C) == 1 ? d.v_scale[g] : 1.0f;
    for (int row = tid >> 4; row < heads; row += kPagedThreads / 16) {
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, s_m[w][row]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) sum += s_l[w][row] * __builtin_amdgcn_exp2f(s_m[w][row] - base - kLift);
        const long bh = (long)b * d.hq + h0 + row;
        const long part = bh * a.pieces + piece;
        if ((tid & 15) == 0) {
            if (a.part_ml) a.part_ml[part] = make_float2(top, sum);
            else if (d.lse) d.lse[bh] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
        }
        const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * vscale;
        for (int c = (tid & 15) * 4; c < d.d; c += 64) {
            v4f x{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kPagedWaves; ++w) x += *reinterpret_cast<const v4f*>(&s.o[w][row][c]);
            if (a.part_ml) {
                *reinterpret_cast<v4f*>(a.part_o + part * d.d + c) = x;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) store1(d.out, d.out_dtype, b * d.out_stride + (long)(h0 + row) * d.d + c + i, x[i] * by, d.out_inv_scale);
            }
        }
    }
}

// The pieces of one query head as one: a workgroup to a head; 16 lanes read a piece's output, four elements at a time.
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a)
{
    __shared__ float s_o[16][256];
    __shared__ float s_top[4], s_sum[4];
    const nm_paged_desc& d = a.d;
    const int bh = blockIdx.x, b = bh / d.hq, h = bh % d.hq, tid = threadIdx.x;
    const int n = (int)min((long)max(d.lens[b], 0), (long)d.max_pages << a.shift);
    const int span = d.window ? min(n, d.window) : n;
    const int used = (span + a.piece - 1) / a.piece;
    const float2* ml = a.part_ml + (long)bh * a.pieces;
    float top = -INFINITY, sum = 0.0f;
    for (int i = tid; i < used; i += 256) top = fmaxf(top, ml[i].x);
    top = __int_as_float(group_reduce<64>(__float_as_int(top), MaxF32{}));
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    const float base = top == -INFINITY ? 0.0f : top;
    for (int i = tid; i < used; i += 256) sum += ml[i].y * __builtin_amdgcn_exp2f(ml[i].x - base);
    sum = group_sum<64>(sum);
    if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
    __syncthreads();
    sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);

    const int row = tid >> 4;
    for (int c = (tid & 15) * 4; c < d.d; c += 64) {
        v4f x{0, 0, 0, 0};
        for (int i = row; i < used; i += 16) {
            const float by = __builtin_amdgcn_exp2f(ml[i].x - base);
            const v4f y = *reinterpret_cast<const v4f*>(a.part_o + ((long)bh * a.pieces + i) * d.d + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(y[e], by, x[e]);
        }
        *reinterpret_cast<v4f*>(&s_o[row][c]) = x;
    }
    __syncthreads();
    const float vscale = d.cache_dtype == NM_DT_I8 ? d.v_scale[h / a.group] : 1.0f;
    const float by = (sum == 0.0f ? 0.0f : 1.0f / sum) * vscale;
    if (tid < d.d) {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x += s_o[i][tid];
        store1(d.out, d.out_dtype, b * d.out_stride + (long)h * d.d + tid, x * by, d.out_inv_scale);
    }
    if (tid == 0 && d.lse) d.lse[bh] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <typename C, int DP>
static void launch_paged(const PagedArgs& a, int blocks, hipStream_t s)
{
    // one term of a query where the matrix instructions' type is its own, and two of the weights where the result has 16 bits or fewer
    const bool own = a.d.q_dtype == (std::is_same<C, f16>::value ? NM_DT_F16 : NM_DT_BF16);
    if (own && a.d.out_dtype != NM_DT_F32) queue_kernel(paged_attention_kernel<C, DP, 1, 2>, dim3(blocks), dim3(kPagedThreads), 0, s, a);
    else queue_kernel(paged_attention_kernel<C, DP, 3, 3>, dim3(blocks), dim3(kPagedThreads), 0, s, a);
}
template <typename C>
static void launch_paged(const PagedArgs& a, int blocks, hipStream_t s)
{
    if (a.d.d <= 64) launch_paged<C, 64>(a, blocks, s);
    else if (a.d.d <= 128) launch_paged<C, 128>(a, blocks, s);
    else launch_paged<C, 256>(a, blocks, s);
}

// What does not depend on pointers: shapes, types, and how the length is divided.
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
    *a = PagedArgs{};
    a->d = *d;
    a->shift = shift;
    a->group = d->hq / d->hk;
    a->groups = (a->group + 15) / 16;
    long longest = (long)d->max_pages << shift;
    if (d->window && d->window < longest) longest = d->window;
    const long rows = (long)d->B * d->hk * a->groups;
    // pieces: as long as leaves 2048 workgroups (eight to a CU, so that ragged lengths even out), 128 positions at least
    long piece = kRound;
    while (piece < longest && rows * ((longest + 2 * piece - 1) / (2 * piece)) >= 2048) piece *= 2;
    a->piece = (int)piece;
    a->pieces = (int)(longest > 0 ? (longest + piece - 1) / piece : 1);
    *blocks = rows * a->pieces;
    if (*blocks >= 1L << 24 || (long)d->B * d->hq >= 1L << 24) return fail(NM_ERR_UNSUPPORTED, "%s: too many heads and pieces", what);
    const size_t parts = (size_t)d->B * d->hq * a->pieces;
    *bytes = a->pieces > 1 ? (parts * sizeof(float2) + 255) / 256 * 256 + parts * d->d * sizeof(float) : 0;
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
    const int64_t row = (int64_t)d->hq * d->d;
    if (d->q_stride < row || d->out_stride < row || d->table_stride < d->max_pages) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: a stride is shorter than a row");
    if (d->page_stride < 0 || d->slot_stride < 0 || d->head_stride < 0) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: negative stride of the cache");
    if (!(d->scale == d->scale) || __builtin_isinf(d->scale)) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: scale must be finite");
    if (d->B == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->q || !d->lens || !d->out) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: q, lens or out is NULL");
    if ((d->max_pages && !d->block_table) || (d->max_pages && d->num_pages && (!d->k_cache || !d->v_cache)))
        return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: block_table or a cache is NULL");
    if (d->cache_dtype == NM_DT_I8 && (!d->k_scale || !d->v_scale)) return fail(NM_ERR_INVALID_ARG, "nm_paged_attention: int8 cache without scales");
    const int per16 = 16 / dtype_bytes(d->cache_dtype);
    if (!aligned(d->k_cache, 16) || !aligned(d->v_cache, 16) || d->page_stride % per16 || d->slot_stride % per16 || d->head_stride % per16)
        return fail(NM_ERR_UNSUPPORTED, "nm_paged_attention: the cache's addresses and strides must be multiples of 16 bytes");
    if (need) {
        if (!ws || ws_bytes < need) return fail(NM_ERR_WORKSPACE, "nm_paged_attention: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
        if (!aligned(ws, 256)) return fail(NM_ERR_WORKSPACE, "nm_paged_attention: workspace must be 256-byte aligned");
        const size_t parts = (size_t)d->B * d->hq * a.pieces;
        a.part_ml = static_cast<float2*>(ws);
        a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + (parts * sizeof(float2) + 255) / 256 * 256);
    }
    if (d->cache_dtype == NM_DT_BF16) launch_paged<bf16>(a, (int)blocks, (hipStream_t)stream);
    else if (d->cache_dtype == NM_DT_F16) launch_paged<f16>(a, (int)blocks, (hipStream_t)stream);
    else launch_paged<int8_t>(a, (int)blocks, (hipStream_t)stream);
    if (need) {
        const int32_t err = check_hip(hipGetLastError(), "nm_paged_attention launch");
        if (err) return err;
        queue_kernel(paged_join_kernel, dim3(d->B * d->hq), dim3(256), 0, (hipStream_t)stream, a);
    }
    return check_hip(hipGetLastError(), "nm_paged_attention launch");
}

}  // extern "C"
