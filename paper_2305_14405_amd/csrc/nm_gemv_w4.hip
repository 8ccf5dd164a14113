// Products of a few rows with 4-bit weights (nm_gemv_w4).
//
// Bound by memory: N K / 2 bytes of weights, each read once, for 2 M operations a weight.  A workgroup has 16 columns (rows of W) and all
// of K, which its wavefronts share in blocks of 128; their sums are joined through LDS, so that columns alone need not fill the GPU.
//   A lane loads 16 bytes, 32 consecutive weights, of row lane % 16; the four lanes of a row have 64 bytes of it.  The 16x16x32 matrix instruction
// (rows of x its rows, columns its columns) adds over the four lanes, so to add within one run of 32 weights (the smallest group) the
// four lanes exchange words, four half swaps for 16 bytes: then register i of lane group j holds weights 8 j .. 8 j + 7 of run i.
//   int8: (v << 4) & 0xf0f0f0f0 and v & 0xf0f0f0f0 are 16 times the even and the odd weights as int8: three operations for eight
// weights, and exact.  bf16, fp16: u = w + 8 is put under an exponent, 16 + u, exactly, in nine; a second matrix instruction with the constant -24
// in the weights' place takes the offset off again, where it costs nothing (the sum of x it subtracts is at most some 5 times the
// result's size, so fp32 loses two bits of 24).
//   What a group's sum is multiplied by is one number per lane (its column).
#include "nm_decode.h"

namespace nm {

typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int kW4Waves = 8, kW4Threads = 64 * kW4Waves;

struct W4Args {
    nm_w4_desc d;
    DevTable table;
    int blocks;      // of 128 weights in K (the last one may be short)
    FastDiv per;     // blocks to a group of 128 or more
};

__device__ __forceinline__ float load_scale(const void* p, int dtype, long at)
{
    return dtype == NM_DT_F32 ? static_cast<const float*>(p)[at] : dtype == NM_DT_BF16 ? (float)static_cast<const bf16*>(p)[at] : (float)static_cast<const f16*>(p)[at];
}

// Register i of lane group j <-> register j of lane group i.
__device__ __forceinline__ v4u exchange(v4u w)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), e = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return v4u{c[0], c[1], e[0], e[1]};
}

// What differs by the type of x: its eight values of a lane, the sum over them, and eight weights.
template <typename X> struct W4;
template <> struct W4<int8_t> {
    typedef v2u Rows;
    typedef v4i Sum;
    static __device__ __forceinline__ Rows order(v2u x) { return Rows{__builtin_amdgcn_perm(x[1], x[0], 0x06040200u), __builtin_amdgcn_perm(x[1], x[0], 0x07050301u)}; }
    static __device__ __forceinline__ Sum zero() { return Sum{0, 0, 0, 0}; }
    static __device__ __forceinline__ v2u weights(unsigned w) { return v2u{(w << 4) & 0xf0f0f0f0u, w & 0xf0f0f0f0u}; }
    static __device__ __forceinline__ Sum add(Rows x, v2u w, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, x), __builtin_bit_cast(long, w), c, 0, 0, 0); }
    static __device__ __forceinline__ Sum offset(Rows, Sum c) { return c; }
    static constexpr float kUnit = 1.0f / 16.0f;
};
template <typename X> struct W4Half {
    typedef v4u Rows;
    typedef v4f Sum;
    static constexpr bool kBf = std::is_same<X, bf16>::value;
    // eight values in the order in which the weights come out of their word: 0 4 1 5 2 6 3 7
    static __device__ __forceinline__ Rows order(v4u x)
    {
        return Rows{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                    __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
    }
    static __device__ __forceinline__ Sum zero() { return Sum{0, 0, 0, 0}; }
    // 16 + u: u in the upper four bits of the mantissa (7 bits of bf16, 10 of fp16)
    static __device__ __forceinline__ v4u weights(unsigned w)
    {
        const unsigned u = w ^ 0x88888888u;
        if (kBf) return v4u{((u << 3) & 0x00780078u) | 0x41804180u, ((u >> 1) & 0x00780078u) | 0x41804180u,
                            ((u >> 5) & 0x00780078u) | 0x41804180u, ((u >> 9) & 0x00780078u) | 0x41804180u};
        return v4u{((u << 6) & 0x03c003c0u) | 0x4c004c00u, ((u << 2) & 0x03c003c0u) | 0x4c004c00u,
                   ((u >> 2) & 0x03c003c0u) | 0x4c004c00u, ((u >> 6) & 0x03c003c0u) | 0x4c004c00u};
    }
    static __device__ __forceinline__ Sum add(Rows x, v4u w, Sum c)
    {
        if constexpr (kBf) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, w), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0);
    }
    static __device__ __forceinline__ Sum offset(Rows x, Sum c)
    {
        const unsigned minus24 = kBf ? 0xc1c0c1c0u : 0xce00ce00u;
        return add(x, v4u{minus24, minus24, minus24, minus24}, c);
    }
    static constexpr float kUnit = 1.0f;
};
template <> struct W4<bf16> : W4Half<bf16> {};
template <> struct W4<f16> : W4Half<f16> {};

// kRuns: runs of 32 weights to a scale within a block of 128 (1, 2, 4); kM: tiles of 16 rows.
template <typename X, int kRuns, int kM>
__global__ __launch_bounds__(kW4Threads) void gemv_w4_kernel(W4Args a)
{
    typedef W4<X> Q;
    typedef typename Q::Rows Rows;
    __shared__ float s_sum[kW4Waves][kM][16][16];
    const nm_w4_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, column = lane & 15, j = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * kM;
    const int n = min(n0 + column, d.N - 1);
    const uint8_t* wrow = d.W + (long)n * (d.K / 2) + j * 16;
    const int groups = d.K / d.group;
    const X* xrow[kM];
    bool row_there[kM];
#pragma unroll
    for (int t = 0; t < kM; ++t) {
        const int m = m0 + t * 16 + column;
        row_there[t] = m < d.M;
        xrow[t] = static_cast<const X*>(d.x) + (long)min(m, d.M - 1) * d.x_stride + j * 8;
    }
    v4f sum[kM];
#pragma unroll
    for (int t = 0; t < kM; ++t) sum[t] = v4f{0, 0, 0, 0};

    for (int kb = wave; kb < a.blocks; kb += kW4Waves) {
        const int k0 = kb * 128;
        v4u w{};
        if (k0 + j * 32 < d.K) w = *reinterpret_cast<const v4u*>(wrow + kb * 64);
        float scale[4 / kRuns];
#pragma unroll
        for (int i = 0; i < 4 / kRuns; ++i) {
            const int g = kRuns == 4 ? (int)quotient(kb, a.per) : kb * (4 / kRuns) + i;
            scale[i] = load_scale(d.scales, d.scale_dtype, (long)n * groups + min(g, groups - 1)) * Q::kUnit;
        }
        w = exchange(w);
#pragma unroll
        for (int t = 0; t < kM; ++t) {
            typename Q::Sum acc = Q::zero();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Rows x{};
                if (row_there[t] && k0 + i * 32 < d.K) x = *reinterpret_cast<const Rows*>(xrow[t] + k0 + i * 32);
                x = Q::order(x);
                acc = Q::offset(x, acc);
                acc = Q::add(x, Q::weights(w[i]), acc);
                if (i % kRuns == kRuns - 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][e] = __builtin_fmaf((float)acc[e], scale[i / kRuns], sum[t][e]);
                    acc = Q::zero();
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[wave][t][j * 4 + e][column] = sum[t][e];
    __syncthreads();
    for (int i = tid; i < kM * 256; i += kW4Threads) {
        const int c = i & 15, r = (i >> 4) & 15, t = i >> 8, m = m0 + t * 16 + r, col = n0 + c;
        if (m >= d.M || col >= d.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kW4Waves; ++w) v += s_sum[w][t][r][c];
        v = __builtin_fmaf(v, d.alpha, d.bias ? d.bias[col] : 0.0f);
        if (d.table_idx >= 0) {
            int seg;
            v = pwl_eval(v, a.table, a.table.kb, seg);
        }
        store1(d.out, d.out_dtype, (long)m * d.out_stride + col, v, d.out_inv_scale);
    }
}

template <typename X, int kRuns>
static void launch_w4(const W4Args& a, hipStream_t s)
{
    const int columns = (a.d.N + 15) / 16;
    if (a.d.M <= 16) queue_kernel(gemv_w4_kernel<X, kRuns, 1>, dim3(columns), dim3(kW4Threads), 0, s, a);
    else if (a.d.M <= 32) queue_kernel(gemv_w4_kernel<X, kRuns, 2>, dim3(columns), dim3(kW4Threads), 0, s, a);
    else queue_kernel(gemv_w4_kernel<X, kRuns, 4>, dim3(columns, (a.d.M + 63) / 64), dim3(kW4Threads), 0, s, a);
}
template <typename X>
static void launch_w4(const W4Args& a, hipStream_t s)
{
    if (a.d.group == 32) launch_w4<X, 1>(a, s);
    else if (a.d.group == 64) launch_w4<X, 2>(a, s);
    else launch_w4<X, 4>(a, s);
}

}  // namespace nm

using namespace nm;

extern "C" int32_t nm_gemv_w4(const nm_w4_desc* d, void* stream)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: desc is NULL");
    if (d->M < 0 || d->N < 1 || d->K < 1 || d->group < 1) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad shape");
    if (d->x_dtype != NM_DT_I8 && d->x_dtype != NM_DT_BF16 && d->x_dtype != NM_DT_F16) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad x_dtype");
    if (!float_dtype(d->scale_dtype)) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad scale_dtype");
    if (!float_dtype(d->out_dtype) && d->out_dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad out_dtype");
    if (d->group != 32 && d->group != 64 && d->group % 128) return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: group %d is not 32, 64 or a multiple of 128", d->group);
    if (d->K % d->group) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: K is no multiple of group");
    if (d->K > 65536 || d->M > 1 << 20 || d->N >= 1 << 26) return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: K > 65536, M > 2^20 or N >= 2^26");
    if (d->x_stride < d->K || d->out_stride < d->N) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: a stride is shorter than a row");
    if (!(d->alpha == d->alpha) || __builtin_isinf(d->alpha)) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: alpha must be finite");
    W4Args a{};
    a.d = *d;
    if (d->table_idx >= 0) {
        const int32_t rc = get_dev_table(d->tables, d->table_idx, &a.table, "nm_gemv_w4");
        if (rc) return rc;
    }
    if (d->M == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->x || !d->W || !d->scales || !d->out) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: NULL argument");
    if (!aligned_rows(d->x, d->x_stride, d->x_dtype, 16 / dtype_bytes(d->x_dtype)) || !aligned(d->W, 16))
        return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: x, its rows and W must be 16-byte aligned");
    a.blocks = (d->K + 127) / 128;
    a.per = fast_div(d->group >= 128 ? d->group / 128 : 1);
    if (d->x_dtype == NM_DT_I8) launch_w4<int8_t>(a, (hipStream_t)stream);
    else if (d->x_dtype == NM_DT_BF16) launch_w4<bf16>(a, (hipStream_t)stream);
    else launch_w4<f16>(a, (hipStream_t)stream);
    return check_hip(hipGetLastError(), "nm_gemv_w4 launch");
}
