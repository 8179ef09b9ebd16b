// The products of the gated feed-forward block for up to 16 rows (serving) of weights that the tensor cores could only read as copies: fp32 (three bfloat16 parts: ten bytes a value written and read beside the four that
// they have), and 16-bit weights whose rows do not start on 16 bytes.  Here they are read as they lie, four rows of them a warp (of Wd; two of Wg and the same two of Wu) with every 32nd vector a lane, and
// multiplied in fp32 by up to four rows of x or h in shared memory; more rows take a block row each (weights again, from the L2 as far as it holds them).  Sums over lanes are halved at each of the first exchanges, so that
// lane l ends up with sum l / (32 / (4 NR)).  Bound by HBM with one row (1 x 4096 x 16 384 fp32: 130 us, 6.2 TB/s; as operands 677), with more by the multiply-adds and the weights' way through the L2 (4 rows 191,
// 16 688; as operands 700).
#pragma once

#include "gated_gemm.cuh"

namespace gad {

namespace {

constexpr int FEW_ROWS = 16, FEW_GROUP = 4, FEW_THREADS = 256, FEW_SMEM = 200 << 10;

struct FewRowsArgs {
    const void* x; long long ldx;
    const void *w0, *w1; long long ldw0, ldw1;            // kGate: Wg and Wu; kPlain: Wd
    int rows, cols, n;                                     // of x; columns; rows of a weight matrix
    void* out; long long ldo;
    int activation, clear;
    int32_t* err;
};
// Rows a block takes at a time: as many as fit shared memory.
int few_group(int64_t rows, int cols) {
    const int64_t fit = FEW_SMEM / 4 / round_up(cols, 8);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(rows, FEW_GROUP), fit);
    return most >= 4 ? 4 : most >= 2 ? 2 : (int)most;      // (0: a row does not fit)
}

template <int USE, int NR, bool WIDE, class T>
__global__ void __launch_bounds__(FEW_THREADS, 1) few_rows_kernel(const __grid_constant__ FewRowsArgs a) {
    extern __shared__ float xs[];                          // [NR][cols, rounded up to a vector]
    constexpr int VEC = 16 / sizeof(T), C = 4 * NR, LC = NR == 1 ? 2 : NR == 2 ? 3 : 4, PER = USE == kGate ? 2 : 4;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, ld = (a.cols + 7) / 8 * 8, row0 = blockIdx.y * NR, rows = min(NR, a.rows - row0);
    pdl_next();
    pdl_wait();
    if (a.clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.err = 0;
    for (int r = 0; r < NR; ++r)
        for (int c = threadIdx.x; c < ld; c += FEW_THREADS) xs[r * ld + c] = r < rows && c < a.cols ? to_float(reinterpret_cast<const T*>(a.x)[(row0 + r) * a.ldx + c]) : 0.f;
    __syncthreads();
    for (int f0 = (blockIdx.x * (FEW_THREADS / 32) + w) * PER; f0 < a.n; f0 += gridDim.x * (FEW_THREADS / 32) * PER) {
        const T* wr[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int f = min(f0 + (USE == kGate ? k & 1 : k), a.n - 1);
            wr[k] = USE == kGate && k >= 2 ? reinterpret_cast<const T*>(a.w1) + (long long)f * a.ldw1 : reinterpret_cast<const T*>(a.w0) + (long long)f * a.ldw0;
        }
        float acc[C];
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = 0.f;
        const int whole = WIDE ? a.cols / VEC : 0;
#pragma unroll 4
        for (int v = lane; v < whole; v += 32) {
            uint4 u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = __ldcs(reinterpret_cast<const uint4*>(wr[k]) + v);
#pragma unroll
            for (int h = 0; h < VEC; h += 4) {
                float wv[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float all[VEC];
                    unpack_vec<T, VEC>(u[k], all);
#pragma unroll
                    for (int j = 0; j < 4; ++j) wv[k][j] = all[h + j];
                }
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const float4 x = *reinterpret_cast<const float4*>(xs + r * ld + VEC * v + h);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[k * NR + r] = fmaf(wv[k][0], x.x, fmaf(wv[k][1], x.y, fmaf(wv[k][2], x.z, fmaf(wv[k][3], x.w, acc[k * NR + r]))));
                }
            }
        }
        // single values, eight loads of each row at a time
        for (int c = VEC * whole + lane; c < a.cols; c += 8 * 32) {
            T u[4][8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k][j] = c + 32 * j < a.cols ? wr[k][c + 32 * j] : from_float<T>(0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const float x = c + 32 * j < a.cols ? xs[r * ld + c + 32 * j] : 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[k * NR + r] = fmaf(to_float(u[k][j]), x, acc[k * NR + r]);
                }
        }
#pragma unroll
        for (int i = 0, n = C; i < 5; ++i) {
            const int o = 16 >> i;
            if (n > 1) {
                n >>= 1;
#pragma unroll
                for (int j = 0; j < C / 2; ++j)
                    if (j < n) {
                        const float keep = (lane & o) ? acc[j + n] : acc[j], give = (lane & o) ? acc[j] : acc[j + n];
                        acc[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                    }
            } else acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], o);
        }
        const int idx = lane >> (5 - LC), k = idx / NR, r = idx % NR;
        const bool mine = (lane & ((1 << (5 - LC)) - 1)) == 0 && r < rows;
        if constexpr (USE == kGate) {
            // u of this lane's unit and row lies two weight rows further on
            const float u = __shfl_sync(0xffffffffu, acc[0], (idx + 2 * NR) << (5 - LC) & 31);
            float g, d;
            activation(a.activation, acc[0], g, d);
            if (mine && k < 2 && f0 + k < a.n) reinterpret_cast<T*>(a.out)[(row0 + r) * a.ldo + f0 + k] = from_float<T>(g * u);
        } else if (mine && f0 + k < a.n) reinterpret_cast<T*>(a.out)[(row0 + r) * a.ldo + f0 + k] = from_float<T>(acc[0]);
    }
}

}  // namespace

}  // namespace gad
