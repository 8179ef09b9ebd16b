// Rows of a matrix that a tensor-map descriptor cannot reach (fp32, or rows that do not start on 16 bytes) as operands of the tensor cores.
#pragma once

#include "class_gemm.cuh"

namespace gad {

namespace {

// A row as operands: copied (16-bit types), or in three bfloat16 parts.  dst rows are 16-byte aligned.
template <class T>
__device__ __forceinline__ void pack_row(const T* __restrict__ src, int cols, bool keep, void* __restrict__ dst, int64_t at, int64_t part_stride, int t, int threads) {
    if constexpr (sizeof(T) == 4) {
        __nv_bfloat16* d = reinterpret_cast<__nv_bfloat16*>(dst) + at;
        const int n4 = ((uintptr_t)src & 15) == 0 ? cols >> 2 : 0;
#pragma unroll 4
        for (int c = t; c < n4; c += threads) {
            const float4 x = keep ? reinterpret_cast<const float4*>(src)[c] : make_float4(0.f, 0.f, 0.f, 0.f);
            __nv_bfloat16 p[4][3];
            split3(x.x, p[0]); split3(x.y, p[1]); split3(x.z, p[2]); split3(x.w, p[3]);
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                union { uint2 u; __nv_bfloat16 h[4]; } w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w.h[i] = p[i][k];
                *reinterpret_cast<uint2*>(d + k * part_stride + 4 * c) = w.u;
            }
        }
#pragma unroll 4
        for (int c = 4 * n4 + t; c < cols; c += threads) {
            __nv_bfloat16 p[3];
            split3(keep ? src[c] : 0.f, p);
            for (int k = 0; k < 3; ++k) d[k * part_stride + c] = p[k];
        }
    } else {
        T* d = reinterpret_cast<T*>(dst) + at;
        // in the widest words that the row starts on (the copy does on all)
        const int wide = ((uintptr_t)src & 15) == 0 ? 8 : ((uintptr_t)src & 7) == 0 ? 4 : ((uintptr_t)src & 3) == 0 ? 2 : 1, n = cols / wide;
        if (wide == 8) {
#pragma unroll 4
            for (int c = t; c < n; c += threads) reinterpret_cast<uint4*>(d)[c] = keep ? reinterpret_cast<const uint4*>(src)[c] : make_uint4(0u, 0u, 0u, 0u);
        } else if (wide == 4) {
#pragma unroll 4
            for (int c = t; c < n; c += threads) reinterpret_cast<uint2*>(d)[c] = keep ? reinterpret_cast<const uint2*>(src)[c] : make_uint2(0u, 0u);
        } else if (wide == 2) {
#pragma unroll 4
            for (int c = t; c < n; c += threads) reinterpret_cast<uint32_t*>(d)[c] = keep ? reinterpret_cast<const uint32_t*>(src)[c] : 0u;
        }
        // (eight loads, then their stores: one value behind the other, 500 rows of 1433 single ones took 20 us)
        for (int c = (wide > 1 ? wide * n : 0) + t; c < cols; c += 8 * threads) {
            T v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = keep && c + j * threads < cols ? src[c + j * threads] : from_float<T>(0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j * threads < cols) d[c + j * threads] = v[j];
        }
    }
}

}  // namespace

}  // namespace gad
