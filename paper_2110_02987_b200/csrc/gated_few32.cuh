// The products of the gated feed-forward block for up to 16 rows of fp32 (serving).  Laid out as operands of the tensor cores, the weights would be read, written as three bfloat16 parts and read again,
// ten bytes a value beside the four that they have: here they are read as they lie, four rows of them a warp (of Wd; two of Wg and the same two of Wu) with every 32nd vector a lane, and multiplied in fp32 by up to
// four rows of x or h in shared memory; more rows take a block row each (weights again, from the L2 as far as it holds them).  Sums over lanes are halved at each of the first exchanges, so that lane l ends up
// with sum l / (32 / (4 NR)).  Bound by HBM with one row (1 x 4096 x 16 384: 130 us, 6.2 TB/s; as operands 677), with more by the multiply-adds and the weights' way through the L2 (4 rows 191, 16 688; as operands 700).
#pragma once

#include "gated_gemm.cuh"

namespace gad {

namespace {

constexpr int FEW32_ROWS = 16, FEW32_GROUP = 4, FEW32_THREADS = 256, FEW32_SMEM = 200 << 10;

struct Few32Args {
    const float* x; long long ldx;
    const float *w0, *w1; long long ldw0, ldw1;           // kGate: Wg and Wu; kPlain: Wd
    int rows, cols, n;                                     // of x; columns; rows of a weight matrix
    float* out; long long ldo;
    int activation, clear;
    int32_t* err;
};
// Rows a block takes at a time: as many as fit shared memory.
int few32_group(int64_t rows, int cols) {
    const int64_t fit = FEW32_SMEM / 4 / round_up(cols, 4);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(rows, FEW32_GROUP), fit);
    return most >= 4 ? 4 : most >= 2 ? 2 : (int)most;      // (0: a row does not fit)
}

template <int USE, int NR, bool WIDE>
__global__ void __launch_bounds__(FEW32_THREADS, 1) few32_kernel(const __grid_constant__ Few32Args a) {
    extern __shared__ float xs[];                          // [NR][cols, rounded up to a vector]
    constexpr int C = 4 * NR, LC = NR == 1 ? 2 : NR == 2 ? 3 : 4, PER = USE == kGate ? 2 : 4;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, ld = (a.cols + 3) / 4 * 4, row0 = blockIdx.y * NR, rows = min(NR, a.rows - row0);
    pdl_next();
    pdl_wait();
    if (a.clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.err = 0;
    for (int r = 0; r < NR; ++r)
        for (int c = threadIdx.x; c < ld; c += FEW32_THREADS) xs[r * ld + c] = r < rows && c < a.cols ? a.x[(row0 + r) * a.ldx + c] : 0.f;
    __syncthreads();
    for (int f0 = (blockIdx.x * (FEW32_THREADS / 32) + w) * PER; f0 < a.n; f0 += gridDim.x * (FEW32_THREADS / 32) * PER) {
        const float* wr[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int f = min(f0 + (USE == kGate ? k & 1 : k), a.n - 1);
            wr[k] = USE == kGate && k >= 2 ? a.w1 + (long long)f * a.ldw1 : a.w0 + (long long)f * a.ldw0;
        }
        float acc[C];
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = 0.f;
        const int whole = WIDE ? a.cols / 4 : 0;
#pragma unroll 4
        for (int v = lane; v < whole; v += 32) {
            float4 u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = __ldcs(reinterpret_cast<const float4*>(wr[k]) + v);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(xs + r * ld + 4 * v);
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[k * NR + r] = fmaf(u[k].x, x.x, fmaf(u[k].y, x.y, fmaf(u[k].z, x.z, fmaf(u[k].w, x.w, acc[k * NR + r]))));
            }
        }
#pragma unroll 4
        for (int c = 4 * whole + lane; c < a.cols; c += 32)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float u = __ldcs(wr[k] + c);
#pragma unroll
                for (int r = 0; r < NR; ++r) acc[k * NR + r] = fmaf(u, xs[r * ld + c], acc[k * NR + r]);
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
            if (mine && k < 2 && f0 + k < a.n) a.out[(row0 + r) * a.ldo + f0 + k] = g * u;
        } else if (mine && f0 + k < a.n) a.out[(row0 + r) * a.ldo + f0 + k] = acc[0];
    }
}

}  // namespace

}  // namespace gad
