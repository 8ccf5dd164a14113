// What the kernels of a decode step share: the types of their tensors, groups of four elements, the cache's layout.
#pragma once

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

// Four neighbouring elements.
__device__ __forceinline__ v4f load4(const float* p) { return *reinterpret_cast<const v4f*>(p); }
template <typename T>
__device__ __forceinline__ v4f load4(const T* p)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    return __builtin_convertvector(*reinterpret_cast<const v4t*>(p), v4f);
}
template <typename T>
__device__ __forceinline__ void store4_as(void* base, long at, v4f v)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<v4t*>(static_cast<T*>(base) + at) = __builtin_convertvector(v, v4t);
}
// dtype is uniform, so this is a scalar branch; inv_scale for I8.
__device__ __forceinline__ void store4(void* base, int dtype, long at, v4f v, float inv_scale)
{
    if (dtype == NM_DT_BF16) store4_as<bf16>(base, at, v);
    else if (dtype == NM_DT_F16) store4_as<f16>(base, at, v);
    else if (dtype == NM_DT_F32) store4_as<float>(base, at, v);
    else *reinterpret_cast<unsigned*>(static_cast<int8_t*>(base) + at) =
             pack4(requant(v[0], inv_scale), requant(v[1], inv_scale), requant(v[2], inv_scale), requant(v[3], inv_scale));
}
__device__ __forceinline__ void store1(void* base, int dtype, long at, float v, float inv_scale)
{
    if (dtype == NM_DT_BF16) static_cast<bf16*>(base)[at] = (bf16)v;
    else if (dtype == NM_DT_F16) static_cast<f16*>(base)[at] = (f16)v;
    else if (dtype == NM_DT_F32) static_cast<float*>(base)[at] = v;
    else static_cast<int8_t*>(base)[at] = (int8_t)requant(v, inv_scale);
}

}  // namespace nm
