// Shared by the operators of the output head: their element types (fp32, fp16, bfloat16), vectors of a row that end at its last column, and launches in a chain.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <utility>

#include "gad_internal.h"

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

// Two values in one conversion.
template <class T> struct Pair;
template <> struct Pair<__half> {
    static __device__ __forceinline__ uint32_t pack(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
};
template <> struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t pack(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u)); }
};
// A vector of 16 bytes as fp32, and back.
template <class T, int VEC>
__device__ __forceinline__ void unpack_vec(const uint4& u, float (&v)[VEC]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(w[j]);
        else { const float2 f = Pair<T>::unpack(w[j]); v[2 * j] = f.x; v[2 * j + 1] = f.y; }
    }
}
template <class T, int VEC>
__device__ __forceinline__ uint4 pack_vec(const float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else return make_uint4(Pair<T>::pack(v[0], v[1]), Pair<T>::pack(v[2], v[3]), Pair<T>::pack(v[4], v[5]), Pair<T>::pack(v[6], v[7]));
}

// VEC values of a row as they lie in memory (VEC > 1: 16 bytes, aligned), and as fp32.
template <class T, int VEC>
union RowVec {
    static_assert(VEC == 1 || VEC * sizeof(T) == 16, "vectors are 16 bytes");
    uint4 u;
    T e[VEC];
    __device__ RowVec() {}
};
template <class T>
union RowVec<T, 1> {
    T e[1];
    __device__ RowVec() {}
};
// row[c .. c + VEC), zeros from `cols` on.
template <class T, int VEC>
__device__ __forceinline__ void load_raw(const T* __restrict__ row, int c, int cols, RowVec<T, VEC>& v) {
    if constexpr (VEC > 1) {
        if (c + VEC <= cols) { v.u = *reinterpret_cast<const uint4*>(row + c); return; }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) v.e[j] = c + j < cols ? row[c + j] : from_float<T>(0.f);
}
template <class T, int VEC>
__device__ __forceinline__ void store_vec(T* __restrict__ row, int c, int cols, const float (&v)[VEC]) {
    if constexpr (VEC > 1) {
        if (c + VEC <= cols) { *reinterpret_cast<uint4*>(row + c) = pack_vec<T, VEC>(v); return; }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (c + j < cols) row[c + j] = from_float<T>(v[j]);
}

// Kernels of one call follow each other by programmatic dependent launch: each comes up while the one in front ends and waits (pdl_wait) before it touches
// memory.  The first waits for all that is in front of it on the stream.
template <class... P, class... Args>
cudaError_t chain(void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, cudaStream_t s, bool first, Args&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = first ? 0 : 1;
    ++g_kernel_launches;
    return cudaLaunchKernelEx(&cfg, kernel, P(std::forward<Args>(args))...);
}

}  // namespace

}  // namespace gad
