// What the kernels of attention over a paged cache share: tiles of the cache into LDS, and how a cost is divided among workgroups.
#pragma once

#include <utility>

#include "nm_decode.h"
#include "nm_paged_choice.h"

namespace nm {

// What nm_paged_attention checks of a call: first its shapes and types (*divided: rows are long enough to be divided among workgroups), then its
// pointers and strides.
int32_t check_paged_shape(const nm_paged_desc* d, bool* divided, const char* what);
int32_t check_paged(const nm_paged_desc* d, const char* what);

typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef f16 v2h __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

// How a total cost is divided: worker w has [begin(w), begin(w + 1)), the first `more` workers one more than `each`.
struct Shares {
    long each, more;
    __device__ __forceinline__ Shares(long all, long workers) : each(all / workers), more(all % workers) {}
    __device__ __forceinline__ Shares(long e, long m, int) : each(e), more(m) {}
    __device__ __forceinline__ long begin(long w) const { return each * w + min(w, more); }
    __device__ __forceinline__ long owner(long x) const
    {
        const long longer = (each + 1) * more;
        return x < longer ? x / (each + 1) : more + (x - longer) / each;
    }
};

template <typename T> struct Mma;
template <> struct Mma<bf16> {
    static __device__ __forceinline__ v4f mma(v8s a, v8s b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0); }
};
template <> struct Mma<f16> {
    static __device__ __forceinline__ v4f mma(v8s a, v8s b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0); }
};

// 16 bytes of a cache row as elements of the matrix instructions' type, to LDS.
template <typename C, typename T>
__device__ __forceinline__ void put(short* to, v4u w)
{
    if constexpr (sizeof(C) == 2) {
        *reinterpret_cast<v4u*>(to) = w;
    } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            v4u o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned x = w[half * 2 + i / 2];
                if constexpr (std::is_same<T, f16>::value) {
                    // 1024 + (code + 128) is exact under fp16's exponent of 1024, and so is the difference
                    const unsigned u = __builtin_amdgcn_perm(0x64646464u, x ^ 0x80808080u, i % 2 ? 0x04030402u : 0x04010400u);
                    o[i] = __builtin_bit_cast(unsigned, (v2h)(__builtin_bit_cast(v2h, u) - v2h{(f16)1152.0f, (f16)1152.0f}));
                } else {
                    const unsigned y = x >> (i % 2 * 16);
                    const unsigned a = __float_as_uint((float)(int8_t)y), b = __float_as_uint((float)(int8_t)(y >> 8));
                    o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);   // the upper halves: small integers have no bits below
                }
            }
            *reinterpret_cast<v4u*>(to + half * 8) = o;
        }
    }
}

// Lane number I of a lane's row: of 16 lanes where there are eight loads or more, else of four.
template <int kLoads, int I>
__device__ __forceinline__ unsigned row_lane(unsigned v)
{
    return __builtin_amdgcn_update_dpp(0, v, kLoads >= 8 ? 0x150 + I : I * 0x55, 0xf, 0xf, false);
}
template <int kLoads, int... I>
__device__ __forceinline__ void fetch_rows(const char* base, unsigned place, v4u (&to)[kLoads], std::integer_sequence<int, I...>)
{
    ((to[I] = *reinterpret_cast<const v4u*>(base + (unsigned long)row_lane<kLoads, I>(place) * 16)), ...);
}

}  // namespace nm
