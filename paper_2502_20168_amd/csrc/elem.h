// Activations of 32 or 16 bits: loads and stores of neighbouring elements, in registers as they lie in memory, and their conversions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ssm_learn.h"

namespace ssm {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// N neighbouring elements; the pointer is aligned to one of them only (rows of any length, halves of an array)
template <class T, int N> struct Pack {
    typedef T type __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T, int N> __device__ __forceinline__ typename Pack<T, N>::type load_pack(const T *p)
{
    return *reinterpret_cast<const typename Pack<T, N>::loose *>(p);
}
template <class T, int N> __device__ __forceinline__ void store_pack(T *p, typename Pack<T, N>::type v)
{
    *reinterpret_cast<typename Pack<T, N>::loose *>(p) = v;
}
// (to nearest even)
template <class T> __device__ __forceinline__ T rounded(float v) { return static_cast<T>(v); }
template <class T> __device__ __forceinline__ typename Pack<T, 4>::type rounded4(f32x4 v)
{
    return __builtin_convertvector(v, typename Pack<T, 4>::type);
}
template <class T> __device__ __forceinline__ f32x4 widened4(typename Pack<T, 4>::type v) { return __builtin_convertvector(v, f32x4); }

// A grid holds fewer than 2^31 workgroups and fewer than 2^32 threads.
inline bool fits_a_grid(int64_t blocks, int threads) { return blocks <= 0x7fffffffLL && blocks * threads <= 0xffffffffLL; }

// the host's side of a dtype argument
inline bool dtype_known(int dtype) { return dtype == SSM_F32 || dtype == SSM_BF16 || dtype == SSM_F16; }
inline size_t dtype_bytes(int dtype) { return dtype == SSM_F32 ? 4 : 2; }
template <class F> inline auto with_dtype(int dtype, F f)
{
    return dtype == SSM_F32 ? f(float{}) : dtype == SSM_BF16 ? f(bf16_t{}) : f(f16_t{});
}

}  // namespace ssm
