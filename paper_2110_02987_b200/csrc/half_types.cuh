// The element types of the output head (fp32, fp16, bfloat16): conversions, and vectors of a row that end at its last column.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace gad {

namespace {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// One rounding to nearest, ties to even.
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// row[c .. c + VEC) as fp32, zeros from `cols` on.  VEC > 1: 16 bytes, aligned.
template <class T, int VEC>
__device__ __forceinline__ void load_vec(const T* __restrict__ row, int c, int cols, float (&v)[VEC]) {
    if (VEC > 1 && c + VEC <= cols) {
        static_assert(VEC == 1 || VEC * sizeof(T) == 16, "vectors are 16 bytes");
        union { uint4 u; T e[VEC]; } w;
        w.u = *reinterpret_cast<const uint4*>(row + c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = to_float(w.e[j]);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = c + j < cols ? to_float(row[c + j]) : 0.f;
    }
}
template <class T, int VEC>
__device__ __forceinline__ void store_vec(T* __restrict__ row, int c, int cols, const float (&v)[VEC]) {
    if (VEC > 1 && c + VEC <= cols) {
        union { uint4 u; T e[VEC]; } w;
#pragma unroll
        for (int j = 0; j < VEC; ++j) w.e[j] = from_float<T>(v[j]);
        *reinterpret_cast<uint4*>(row + c) = w.u;
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (c + j < cols) row[c + j] = from_float<T>(v[j]);
    }
}

}  // namespace

}  // namespace gad
