// What the kernels of a decode step share: the types of their tensors, groups of four elements, the cache's layout.
#pragma once

#include <initializer_list>

#include "nm_device.h"

namespace nm {

typedef __bf16 bf16;
typedef _Float16 f16;

inline int dtype_bytes(int32_t t) { return t == NM_DT_I8 ? 1 : t == NM_DT_BF16 || t == NM_DT_F16 ? 2 : 4; }
inline bool float_dtype(int32_t t) { return t == NM_DT_F32 || t == NM_DT_BF16 || t == NM_DT_F16; }
inline bool aligned_rows(const void* p, int64_t stride, int32_t dtype, int elements)
{
    return aligned(p, (size_t)elements * dtype_bytes(dtype)) && stride % elements == 0;
}
// log2 of a power of two up to 65536, -1 for any other number.
inline int page_shift(int32_t page_size)
{
    for (int s = 0; s <= 16; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}

// Whether something that is written begins where one of the others does (NULL: not there).
inline bool begins_as(const void* out, std::initializer_list<const void*> others)
{
    for (const void* p : others)
        if (out && p == out) return true;
    return false;
}

// N neighbouring elements, rounded once.  dtype is uniform, so this is a scalar branch; inv_scale for I8.
template <typename T, int N>
__device__ __forceinline__ void store_run_as(void* base, long at, const float (&v)[N])
{
    typedef T Vec __attribute__((ext_vector_type(N)));
    Vec o;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (T)v[i];
    *reinterpret_cast<Vec*>(static_cast<T*>(base) + at) = o;
}
template <int N>
__device__ __forceinline__ void store_run(void* base, int dtype, long at, const float (&v)[N], float inv_scale)
{
    if (dtype == NM_DT_BF16) store_run_as<bf16>(base, at, v);
    else if (dtype == NM_DT_F16) store_run_as<f16>(base, at, v);
    else if (dtype == NM_DT_F32) store_run_as<float>(base, at, v);
    else {
        typedef unsigned Vec __attribute__((ext_vector_type(N / 4)));
        Vec o;
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            o[i] = pack4(requant(v[4 * i], inv_scale), requant(v[4 * i + 1], inv_scale), requant(v[4 * i + 2], inv_scale), requant(v[4 * i + 3], inv_scale));
        *reinterpret_cast<Vec*>(static_cast<int8_t*>(base) + at) = o;
    }
}
__device__ __forceinline__ void store1(void* base, int dtype, long at, float v, float inv_scale)
{
    if (dtype == NM_DT_BF16) static_cast<bf16*>(base)[at] = (bf16)v;
    else if (dtype == NM_DT_F16) static_cast<f16*>(base)[at] = (f16)v;
    else if (dtype == NM_DT_F32) static_cast<float*>(base)[at] = v;
    else static_cast<int8_t*>(base)[at] = (int8_t)requant(v, inv_scale);
}

}  // namespace nm
