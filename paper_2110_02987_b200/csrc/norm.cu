// Layer norm over the columns of a matrix, forward and backward:
//   mu_i = mean_c x_ic,  r_i = 1 / sqrt(mean_c (x_ic - mu_i)^2 + eps),  h = (x - mu) r,  y = h gamma + beta;
//   with g = dy gamma:  dx = r (g - mean_c g - h mean_c (g h)),  dgamma = sum_i dy h,  dbeta = sum_i dy.
// Both are bound by HBM: forward reads x and writes y, backward reads dy and x and writes dx, once.  A row is held in the registers of one
// warp (up to 1024 two-byte or 512 four-byte values) or of one block, so that nothing is read twice; sums are fp32 and the variance is taken from the
// registers in a second pass, from the differences to the mean, which loses nothing to a large mean.
// Measured: 16 384 x 4096 bf16 forward 48 us on the device (5.6 TB/s; a plain copy of these bytes 44 us), 32 768 x 2048 bf16 backward 71 us (5.7 TB/s) and 8 us for the sums of
// the parameters, 20 011 x 1433 fp32 forward, whose rows start on 4 bytes, 42 us (5.4 TB/s).  What is left to the copy is the instructions, 55 to 65 % of the issue slots.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <map>
#include <mutex>

#include "gad_internal.h"
#include "half_types.cuh"

namespace gad {

namespace {

// Blocks of the backward pass at most, each with a partial sum of dgamma and dbeta: four on every SM, as many as 128 threads of 122 registers leave room for.
constexpr int kNormBlocks = 592;
// Long rows from which on a row is eight warps' (2048 x 16 392 bf16 forward: with 32 warps 81 us).
constexpr int kLongRows = 592;

// gamma / beta in fp32 or in the matrix's own type; null is 1 or 0.  `wide`: both start on 16 bytes.
template <class T, int VEC>
__device__ __forceinline__ void load_param(const void* p, bool fp32, bool wide, int c, int cols, float none, float (&v)[VEC]) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = none;
        return;
    }
    if constexpr (VEC > 1) {
        if (wide && c + VEC <= cols) {
            if (fp32 || sizeof(T) == 4) {
#pragma unroll
                for (int j = 0; j < VEC; j += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + c + j);
                    v[j] = q.x; v[j + 1] = q.y; v[j + 2] = q.z; v[j + 3] = q.w;
                }
            } else {
                unpack_vec<T, VEC>(*reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p) + c), v);
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        if (c + j >= cols) v[j] = 0.f;
        else v[j] = fp32 ? reinterpret_cast<const float*>(p)[c + j] : to_float(reinterpret_cast<const T*>(p)[c + j]);
    }
}

template <int WPR> struct RowGroup {   // WPR warps share a row; a block has several rows only with one warp each
    static constexpr int kRows = WPR == 1 ? 4 : 1;
    static constexpr int kThreads = 32 * WPR * kRows;
};

// A row's sum over its WPR warps.  `slot` alternates between two places, so that one barrier a call is enough.
template <int WPR, int NS>
__device__ __forceinline__ void row_sum(float (&v)[NS], float* sm, int slot) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (WPR > 1) {
        float* at = sm + slot * NS * WPR;
        const int w = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < NS; ++i) at[i * WPR + w] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            if constexpr (WPR % 4 == 0) {
                float4 s = *reinterpret_cast<const float4*>(at + i * WPR);
#pragma unroll
                for (int k = 4; k < WPR; k += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(at + i * WPR + k);
                    s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
                }
                v[i] = (s.x + s.y) + (s.z + s.w);
            } else {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < WPR; ++k) s += at[i * WPR + k];
                v[i] = s;
            }
        }
    }
}

// Vector k of a row; without TAIL the row ends with a vector, which is then in it as a whole or not at all.
template <class T, int VEC, bool TAIL>
__device__ __forceinline__ void put_vec(T* __restrict__ row, int c, int cols, const float (&v)[VEC]) {
    if constexpr (VEC > 1 && !TAIL) { if (c < cols) __stcs(reinterpret_cast<uint4*>(row + c), pack_vec<T, VEC>(v)); }
    else store_vec<T, VEC>(row, c, cols, v);
}

// The next rows of a thread's vectors on their way into shared memory (cp.async: no registers, and no barrier, since a thread reads only what it has asked for
// itself): STAGES rows of NMAT matrices.  One row ahead in registers left 24 to 32 KB on their way on an SM, and HBM wants 43 (32768 x 2048
// backward 81 us).  Rows that do not come as vectors wait in registers, one row ahead.
template <class T, int VEC, int NV, int WPR, int NMAT>
struct RowRing {
    static constexpr int THREADS = RowGroup<WPR>::kThreads, TPR = 32 * WPR;
    static constexpr bool ASYNC = VEC > 1;
    static constexpr int STAGE = NMAT * NV * THREADS * 16, STAGES = STAGE > (32 << 10) ? 2 : 3;
    static constexpr int AHEAD = ASYNC ? STAGES : 1;
    static constexpr size_t kSmem = ASYNC ? (size_t)STAGES * STAGE : 0;
    uint8_t* at;                                  // this thread's place in the first stage
    RowVec<T, VEC> reg[ASYNC ? 1 : NMAT][ASYNC ? 1 : NV];
    __device__ __forceinline__ explicit RowRing(uint8_t* smem) : at(smem + threadIdx.x * 16) {}
    __device__ __forceinline__ uint8_t* place(int stage, int m, int k) const { return at + stage * STAGE + (m * NV + k) * THREADS * 16; }
    __device__ __forceinline__ void ask(int stage, int m, const T* row, int t, int cols) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
            if constexpr (ASYNC) {
                const int n = max(0, min(VEC, cols - c));                              // behind the last column: zeros
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(place(stage, m, k))), "l"(n ? row + c : row),
                             "r"(n * (int)sizeof(T)) : "memory");
            } else load_raw<T, VEC>(row, c, cols, reg[m][k]);
        }
    }
    static __device__ __forceinline__ void close() {
        if constexpr (ASYNC) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    static __device__ __forceinline__ void wait() {                                     // for the oldest row
        if constexpr (ASYNC) asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
    }
    __device__ __forceinline__ void take(int stage, int m, int k, float (&v)[VEC]) const {
        if constexpr (ASYNC) unpack_vec<T, VEC>(*reinterpret_cast<const uint4*>(place(stage, m, k)), v);
        else v[0] = to_float(reg[m][k].e[0]);
    }
};

// NV vectors of VEC values a thread hold a row: vector k of thread t starts at column (k * threads + t) * VEC.  A block takes every gridDim-th row (group of rows),
// keeps gamma and beta in registers and has the next rows on their way while it works on one.
template <class T, int VEC, int NV, int WPR, bool TAIL>
__global__ void __launch_bounds__(RowGroup<WPR>::kThreads) norm_kernel(const T* __restrict__ x, long long ldx, long long rows, int cols, const void* __restrict__ gamma,
                                                                       const void* __restrict__ beta, bool p32, bool pwide, float eps, T* __restrict__ y, long long ldy,
                                                                       float* __restrict__ mean, float* __restrict__ rstd) {
    constexpr int TPR = 32 * WPR, ROWS = RowGroup<WPR>::kRows;
    __shared__ __align__(16) float sm[2 * WPR];
    const int t = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * ROWS;
    long long r = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    extern __shared__ __align__(16) uint8_t ring_smem[];
    typedef RowRing<T, VEC, NV, WPR, 1> Ring;
    Ring ring(ring_smem);
    long long ra = r;                            // the next row to ask for
    T* yr = y + r * ldy;
#pragma unroll
    for (int i = 0; i < Ring::AHEAD; ++i, ra += step) {
        if (ra < rows) ring.ask(i, 0, x + ra * ldx, t, cols);
        Ring::close();
    }
    float g[NV][VEC], b[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param<T, VEC>(gamma, p32, pwide, (k * TPR + t) * VEC, cols, 1.f, g[k]);
        load_param<T, VEC>(beta, p32, pwide, (k * TPR + t) * VEC, cols, 0.f, b[k]);
    }
    const float inv = 1.f / (float)cols;
    int stage = 0;
    for (; r < rows; r += step) {                // (a whole warp, or a whole block)
        float v[NV][VEC];
        float s[1] = {0.f};
        Ring::wait();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            ring.take(stage, 0, k, v[k]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += v[k][j];   // (zeros behind the last column)
        }
        if constexpr (!Ring::ASYNC) { if (ra < rows) ring.ask(0, 0, x + ra * ldx, t, cols); }
        row_sum<WPR, 1>(s, sm, 0);
        if constexpr (Ring::ASYNC) {             // (behind the sum: this stage has been read)
            if (ra < rows) ring.ask(stage, 0, x + ra * ldx, t, cols);
            Ring::close();
            if (++stage == Ring::AHEAD) stage = 0;
        }
        ra += step;
        const float mu = s[0] * inv;
        float q[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
            const bool in = TAIL || c < cols;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[k][j] = in ? v[k][j] - mu : 0.f;
                if (!TAIL || c + j < cols) q[0] = fmaf(v[k][j], v[k][j], q[0]);
            }
        }
        row_sum<WPR, 1>(q, sm, 1);
        const float rs = 1.f / sqrtf(q[0] * inv + eps);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[k][j] = fmaf(v[k][j] * rs, g[k][j], b[k][j]);
            put_vec<T, VEC, TAIL>(yr, c, cols, v[k]);
        }
        yr += step * ldy;
        if (t == 0) { mean[r] = mu; rstd[r] = rs; }
    }
}

// Rows longer than a block's registers hold: read three times, twice of them from L2.  Eight warps a row where there are rows for all SMs, else 32.
template <class T, int VEC, int WPR>
__global__ void __launch_bounds__(32 * WPR) norm_long_kernel(const T* __restrict__ x, long long ldx, int cols, const void* __restrict__ gamma, const void* __restrict__ beta,
                                                         bool p32, bool pwide, float eps, T* __restrict__ y, long long ldy, float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ __align__(16) float sm[2 * WPR];
    const long long r = blockIdx.x;
    const T* xr = x + r * ldx;
    RowVec<T, VEC> v;
    float s[1] = {0.f};
#pragma unroll 4
    for (int c = threadIdx.x * VEC; c < cols; c += 32 * WPR * VEC) {
        load_raw<T, VEC>(xr, c, cols, v);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] += to_float(v.e[j]);
    }
    row_sum<WPR, 1>(s, sm, 0);
    const float mu = s[0] / (float)cols;
    float q[1] = {0.f};
#pragma unroll 4
    for (int c = threadIdx.x * VEC; c < cols; c += 32 * WPR * VEC) {
        load_raw<T, VEC>(xr, c, cols, v);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (c + j < cols) { const float d = to_float(v.e[j]) - mu; q[0] = fmaf(d, d, q[0]); }
    }
    row_sum<WPR, 1>(q, sm, 1);
    const float rs = 1.f / sqrtf(q[0] / (float)cols + eps);
#pragma unroll 4
    for (int c = threadIdx.x * VEC; c < cols; c += 32 * WPR * VEC) {
        float g[VEC], b[VEC], o[VEC];
        load_raw<T, VEC>(xr, c, cols, v);
        load_param<T, VEC>(gamma, p32, pwide, c, cols, 1.f, g);
        load_param<T, VEC>(beta, p32, pwide, c, cols, 0.f, b);
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = fmaf((to_float(v.e[j]) - mu) * rs, g[j], b[j]);
        store_vec<T, VEC>(y + r * ldy, c, cols, o);
    }
    if (threadIdx.x == 0) { mean[r] = mu; rstd[r] = rs; }
}

// Every block takes rows blockIdx, blockIdx + gridDim ... (several at once where a row is a warp's), the next ones on their way, and keeps the sums of dy h and dy of
// its columns in registers; they go to partial[block][2][cols], which norm_columns_kernel adds up in block order.
template <class T, int VEC, int NV, int WPR, bool TAIL>
__global__ void __launch_bounds__(RowGroup<WPR>::kThreads) norm_backward_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ x, long long ldx, long long rows,
                                                                                int cols, const void* __restrict__ gamma, bool p32, bool pwide, const float* __restrict__ mean,
                                                                                const float* __restrict__ rstd, T* __restrict__ dx, long long lddx, float* __restrict__ partial) {
    constexpr int TPR = 32 * WPR, ROWS = RowGroup<WPR>::kRows;
    __shared__ __align__(16) float sm[2 * 2 * WPR];
    extern __shared__ __align__(16) uint8_t ring_smem[];
    pdl_next();
    const int t = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * ROWS;
    long long r = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    typedef RowRing<T, VEC, NV, WPR, 2> Ring;
    float* cs = reinterpret_cast<float*>(ring_smem + Ring::kSmem);   // with several rows a block: [2][cols]
    Ring ring(ring_smem);
    T* dxr = dx + r * lddx;
    long long ra = r;                            // the next row to ask for
    float nmu = r < rows ? mean[r] : 0.f, nrs = r < rows ? rstd[r] : 0.f;
    const auto fetch = [&](int stage) {
        if (ra < rows) {
            ring.ask(stage, 0, dy + ra * lddy, t, cols);
            ring.ask(stage, 1, x + ra * ldx, t, cols);
        }
        Ring::close();
        ra += step;
    };
#pragma unroll
    for (int i = 0; i < Ring::AHEAD; ++i) fetch(i);
    float ag[NV][VEC], ab[NV][VEC], g[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param<T, VEC>(gamma, p32, pwide, (k * TPR + t) * VEC, cols, 1.f, g[k]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) ag[k][j] = ab[k][j] = 0.f;
    }
    const float inv = 1.f / (float)cols;
    int slot = 0, stage = 0;
    for (; r < rows; r += step, slot ^= 1) {
        const float mu = nmu, rs = nrs;
        float d[NV][VEC], h[NV][VEC], s[2] = {0.f, 0.f};
        Ring::wait();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            ring.take(stage, 0, k, d[k]);
            ring.take(stage, 1, k, h[k]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[k][j] = (h[k][j] - mu) * rs;   // (behind the last column d = 0: adds nothing)
        }
        if (r + step < rows) { nmu = mean[r + step]; nrs = rstd[r + step]; }
        if constexpr (!Ring::ASYNC) fetch(0);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                ag[k][j] = fmaf(d[k][j], h[k][j], ag[k][j]);
                ab[k][j] += d[k][j];
                d[k][j] *= g[k][j];
                s[0] += d[k][j];
                s[1] = fmaf(d[k][j], h[k][j], s[1]);
            }
        row_sum<WPR, 2>(s, sm, slot);
        if constexpr (Ring::ASYNC) {             // (behind the sum: this stage has been read)
            fetch(stage);
            if (++stage == Ring::AHEAD) stage = 0;
        }
        const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int j = 0; j < VEC; ++j) d[k][j] = fmaf(-h[k][j], m1, d[k][j] - m0) * rs;
            put_vec<T, VEC, TAIL>(dxr, c, cols, d[k]);
        }
        dxr += step * lddx;
    }
    if (!partial) return;
    float* out = partial + (long long)blockIdx.x * 2 * cols;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j < cols) { out[c + j] = ag[k][j]; out[cols + c + j] = ab[k][j]; }
        }
    } else {
        for (int w = 0; w < ROWS; ++w) {          // warp by warp, in order
            if (threadIdx.x / TPR == w) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int c = (k * TPR + t) * VEC;
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (c + j < cols) {
                            cs[c + j] = w ? cs[c + j] + ag[k][j] : ag[k][j];
                            cs[cols + c + j] = w ? cs[cols + c + j] + ab[k][j] : ab[k][j];
                        }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * cols; c += RowGroup<WPR>::kThreads) out[c] = cs[c];
    }
}

// Long rows: dx by a block a row, read twice.
template <class T, int VEC, int WPR>
__global__ void __launch_bounds__(32 * WPR) norm_backward_long_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ x, long long ldx, int cols,
                                                                  const void* __restrict__ gamma, bool p32, bool pwide, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, T* __restrict__ dx, long long lddx) {
    __shared__ __align__(16) float sm[2 * 2 * WPR];
    const long long r = blockIdx.x;
    const float mu = mean[r], rs = rstd[r], inv = 1.f / (float)cols;
    RowVec<T, VEC> vd, vx;
    float s[2] = {0.f, 0.f}, g[VEC];
#pragma unroll 2
    for (int c = threadIdx.x * VEC; c < cols; c += 32 * WPR * VEC) {
        load_raw<T, VEC>(dy + r * lddy, c, cols, vd);
        load_raw<T, VEC>(x + r * ldx, c, cols, vx);
        load_param<T, VEC>(gamma, p32, pwide, c, cols, 1.f, g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float d = to_float(vd.e[j]) * g[j];
            s[0] += d;
            s[1] = fmaf(d, (to_float(vx.e[j]) - mu) * rs, s[1]);
        }
    }
    row_sum<WPR, 2>(s, sm, 0);
    const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll 2
    for (int c = threadIdx.x * VEC; c < cols; c += 32 * WPR * VEC) {
        float o[VEC];
        load_raw<T, VEC>(dy + r * lddy, c, cols, vd);
        load_raw<T, VEC>(x + r * ldx, c, cols, vx);
        load_param<T, VEC>(gamma, p32, pwide, c, cols, 1.f, g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = (to_float(vd.e[j]) * g[j] - m0 - (to_float(vx.e[j]) - mu) * rs * m1) * rs;
        store_vec<T, VEC>(dx + r * lddx, c, cols, o);
    }
}
// ... and their column sums: a block has 32 vectors of columns and every gridDim.y-th eight rows.
template <class T, int VEC>
__global__ void __launch_bounds__(256) norm_long_columns_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ x, long long ldx, long long rows, int cols,
                                                                const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ partial) {
    __shared__ float sm[8][32 * VEC];
    pdl_next();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * VEC;
    float ag[VEC], ab[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) ag[j] = ab[j] = 0.f;
    if (c < cols)
#pragma unroll 4
        for (long long r = (long long)blockIdx.y * 8 + w; r < rows; r += 8ll * gridDim.y) {
            RowVec<T, VEC> vd, vx;
            load_raw<T, VEC>(dy + r * lddy, c, cols, vd);
            load_raw<T, VEC>(x + r * ldx, c, cols, vx);
            const float mu = mean[r], rs = rstd[r];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = to_float(vd.e[j]);
                ag[j] = fmaf(d, (to_float(vx.e[j]) - mu) * rs, ag[j]);
                ab[j] += d;
            }
        }
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < VEC; ++j) sm[w][lane * VEC + j] = k ? ab[j] : ag[j];
        __syncthreads();
        for (int i = threadIdx.x; i < 32 * VEC; i += 256) {
            const int at = blockIdx.x * 32 * VEC + i;
            if (at >= cols) continue;
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) s += sm[q][i];
            partial[((long long)blockIdx.y * 2 + k) * cols + at] = s;
        }
    }
}

// dgamma, dbeta [2 x cols] = the blocks' partial sums, in block order: 32 columns a block, each of its 32 warps a run of blocks.
template <class T>
__global__ void __launch_bounds__(1024) norm_columns_kernel(const float* __restrict__ partial, int nblocks, int cols, bool p32, void* __restrict__ dgamma, void* __restrict__ dbeta) {
    __shared__ float sm[32][33];
    pdl_wait();
    after_wait(partial);
    const int lane = threadIdx.x & 31, i = blockIdx.x * 32 + lane, w = threadIdx.x >> 5;
    const int per = (nblocks + 31) / 32, lo = min(nblocks, w * per), hi = min(nblocks, lo + per);
    float s = 0.f;
    if (i < 2 * cols)
#pragma unroll 8
        for (int b = lo; b < hi; ++b) s += partial[(long long)b * 2 * cols + i];
    sm[w][lane] = s;
    __syncthreads();
    // warp w sums column w of the 32, a run a lane
    s = sm[lane][w];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int j = blockIdx.x * 32 + w;
    if (lane || j >= 2 * cols) return;
    void* out = j < cols ? dgamma : dbeta;
    const int c = j < cols ? j : j - cols;
    if (!out) return;
    if (p32) reinterpret_cast<float*>(out)[c] = s;
    else reinterpret_cast<T*>(out)[c] = from_float<T>(s);
}

bool wide_rows(const void* p, int64_t ld, size_t size) { return ((uintptr_t)p & 15) == 0 && (ld * size) % 16 == 0; }

struct NormCall {
    const void *x, *gamma, *beta;
    int64_t ldx, rows;
    int cols;
    bool p32, pwide;
    float eps;
    void* y;
    int64_t ldy;
    float *mean, *rstd;
};

// Blocks of a kernel that the GPU holds at once.
int blocks_at_once(const void* kernel, int threads, size_t smem) {
    static std::mutex lock;
    static std::map<std::pair<const void*, size_t>, int> known;
    std::lock_guard<std::mutex> guard(lock);
    int& n = known[{kernel, smem}];
    if (n == 0) {
        int per_sm = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess || per_sm < 1) { cudaGetLastError(); per_sm = 1; }
        n = 148 * per_sm;
    }
    return n;
}

template <class T, int VEC, int NV, int WPR>
void norm_go(const NormCall& a, cudaStream_t s) {
    const auto kernel = VEC > 1 && a.cols % VEC == 0 ? norm_kernel<T, VEC, NV, WPR, false> : norm_kernel<T, VEC, NV, WPR, true>;
    const int64_t blocks = (a.rows + RowGroup<WPR>::kRows - 1) / RowGroup<WPR>::kRows;
    constexpr size_t smem = RowRing<T, VEC, NV, WPR, 1>::kSmem;
    if (smem > (40 << 10)) configure_kernel_once((const void*)kernel, 200 << 10, false);   // (48 KB without asking, its fixed arrays included)
    // short calls: a block a row (group), without asking the runtime
    const int64_t grid = blocks <= 148 ? blocks : std::min<int64_t>(blocks, blocks_at_once((const void*)kernel, RowGroup<WPR>::kThreads, smem));
    kernel<<<(unsigned)grid, RowGroup<WPR>::kThreads, smem, s>>>((const T*)a.x, a.ldx, a.rows, a.cols, a.gamma, a.beta, a.p32, a.pwide, a.eps, (T*)a.y, a.ldy, a.mean, a.rstd);
}
// Vectors a thread x warps a row, by the length of a row: a warp as long as 32 values a lane hold it, then blocks of up to 16.  16 384 x 4096 bf16: 2 x 8 52.7 us,
// 4 x 4 54.5, 1 x 16 65 (one row ahead in registers); 20 011 x 1433 fp32 by single values: 6 x 8 48.6, 12 x 4 48.6, 3 x 16 67.
template <class T>
void norm_pick(const NormCall& a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    if (wide_rows(a.x, a.ldx, sizeof(T)) && wide_rows(a.y, a.ldy, sizeof(T))) {
        const int n = (a.cols + V - 1) / V;
        if (n <= 32) return norm_go<T, V, 1, 1>(a, s);
        if (n <= 64) return norm_go<T, V, 2, 1>(a, s);
        if (n <= 128) return norm_go<T, V, 4, 1>(a, s);
        if (n <= 256) return norm_go<T, V, 4, 2>(a, s);
        if (n <= 512) return norm_go<T, V, 2, 8>(a, s);
        if (n <= 1024) return norm_go<T, V, 4, 8>(a, s);
        if (n <= 2048) return norm_go<T, V, 4, 16>(a, s);
    } else {
        if (a.cols <= 128) return norm_go<T, 1, 4, 1>(a, s);
        if (a.cols <= 1024) return norm_go<T, 1, 8, 4>(a, s);
        if (a.cols <= 1536) return norm_go<T, 1, 6, 8>(a, s);
        if (a.cols <= 2048) return norm_go<T, 1, 8, 8>(a, s);
        if (a.cols <= 8192) return norm_go<T, 1, 16, 16>(a, s);
    }
    const bool wide = wide_rows(a.x, a.ldx, sizeof(T)) && wide_rows(a.y, a.ldy, sizeof(T)), many = a.rows >= kLongRows;
    const auto kernel = wide ? (many ? norm_long_kernel<T, V, 8> : norm_long_kernel<T, V, 32>) : many ? norm_long_kernel<T, 1, 8> : norm_long_kernel<T, 1, 32>;
    kernel<<<(unsigned)a.rows, many ? 256 : 1024, 0, s>>>((const T*)a.x, a.ldx, a.cols, a.gamma, a.beta, a.p32, a.pwide, a.eps, (T*)a.y, a.ldy, a.mean, a.rstd);
}

struct NormBackCall {
    const void *dy, *x, *gamma;
    int64_t lddy, ldx, rows;
    int cols;
    bool p32, pwide;
    const float *mean, *rstd;
    void* dx;
    int64_t lddx;
    void *dgamma, *dbeta;
    float* partial;
};

template <class T, int VEC, int NV, int WPR>
int norm_back_go(const NormBackCall& a, cudaStream_t s) {
    constexpr int ROWS = RowGroup<WPR>::kRows;
    const auto kernel = VEC > 1 && a.cols % VEC == 0 ? norm_backward_kernel<T, VEC, NV, WPR, false> : norm_backward_kernel<T, VEC, NV, WPR, true>;
    const size_t smem = RowRing<T, VEC, NV, WPR, 2>::kSmem + (ROWS > 1 ? 8 * (size_t)a.cols : 0);
    if (smem > (40 << 10)) configure_kernel_once((const void*)kernel, 200 << 10, false);
    const int blocks = (int)std::min<int64_t>({(a.rows + ROWS - 1) / ROWS, (int64_t)kNormBlocks, (int64_t) blocks_at_once((const void*)kernel, RowGroup<WPR>::kThreads, smem)});
    kernel<<<(unsigned)blocks, RowGroup<WPR>::kThreads, smem, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.rows, a.cols, a.gamma, a.p32, a.pwide, a.mean, a.rstd, (T*)a.dx, a.lddx, a.partial);
    return blocks;
}
// The same for the backward pass, which holds six values where the forward pass holds four: two vectors a thread.  32 768 x 2048 bf16: 2 x 4 88 us, 1 x 8 95, 4 x 2 93
// (one row ahead in registers).
template <class T>
int norm_back_rows(const NormBackCall& a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    if (wide_rows(a.x, a.ldx, sizeof(T)) && wide_rows(a.dy, a.lddy, sizeof(T)) && wide_rows(a.dx, a.lddx, sizeof(T))) {
        const int n = (a.cols + V - 1) / V;
        if (n <= 32) return norm_back_go<T, V, 1, 1>(a, s);
        if (n <= 64) return norm_back_go<T, V, 2, 1>(a, s);
        if (n <= 128) return norm_back_go<T, V, 2, 2>(a, s);
        if (n <= 256) return norm_back_go<T, V, 2, 4>(a, s);
        if (n <= 512) return norm_back_go<T, V, 2, 8>(a, s);
        if (n <= 1024) return norm_back_go<T, V, 2, 16>(a, s);
    } else {
        if (a.cols <= 128) return norm_back_go<T, 1, 4, 1>(a, s);
        if (a.cols <= 1024) return norm_back_go<T, 1, 8, 4>(a, s);
        if (a.cols <= 2048) return norm_back_go<T, 1, 8, 8>(a, s);
        if (a.cols <= 8192) return norm_back_go<T, 1, 16, 16>(a, s);
    }
    const bool wide = wide_rows(a.x, a.ldx, sizeof(T)) && wide_rows(a.dy, a.lddy, sizeof(T)) && wide_rows(a.dx, a.lddx, sizeof(T)), many = a.rows >= kLongRows;
    const auto kernel = wide ? (many ? norm_backward_long_kernel<T, V, 8> : norm_backward_long_kernel<T, V, 32>)
                             : many ? norm_backward_long_kernel<T, 1, 8> : norm_backward_long_kernel<T, 1, 32>;
    kernel<<<(unsigned)a.rows, many ? 256 : 1024, 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.cols, a.gamma, a.p32, a.pwide, a.mean, a.rstd, (T*)a.dx, a.lddx);
    const int blocks = (int)std::min<int64_t>((a.rows + 7) / 8, 64);
    if (a.partial)
        chain(wide ? norm_long_columns_kernel<T, V> : norm_long_columns_kernel<T, 1>, dim3((unsigned)((a.cols + 32 * (wide ? V : 1) - 1) / (32 * (wide ? V : 1))), (unsigned)blocks), 256, 0, s, false,
              (const T*)a.dy, (long long)a.lddy, (const T*)a.x, (long long)a.ldx, (long long)a.rows, a.cols, a.mean, a.rstd, a.partial);
    return blocks;
}
template <class T>
void norm_back_pick(const NormBackCall& a, cudaStream_t s) {
    const int blocks = a.rows > 0 ? norm_back_rows<T>(a, s) : 0;
    if (a.rows > 0) ++g_kernel_launches;
    if (!a.dgamma && !a.dbeta) return;
    // (behind the kernel that leaves the sums; with no rows it stands alone)
    chain(norm_columns_kernel<T>, dim3((unsigned)((2ll * a.cols + 31) / 32)), 1024, 0, s, a.rows == 0, (const float*)a.partial, blocks, a.cols, a.p32, a.dgamma, a.dbeta);
}

bool norm_sizes_ok(int64_t rows, int32_t cols, int32_t dtype, int32_t param_dtype) {
    return rows >= 0 && rows < ((int64_t)1 << 31) && cols >= 1 && cols <= (1 << 29) && dtype >= GAD_F32 && dtype <= GAD_BF16 && (param_dtype == dtype || param_dtype == GAD_F32);
}

}  // namespace
}  // namespace gad

extern "C" int gad_layer_norm(const void* x, int64_t ldx, int64_t rows, int32_t cols, int32_t dtype, const void* gamma, const void* beta, int32_t param_dtype, float eps,
                              void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
    using namespace gad;
    if (!norm_sizes_ok(rows, cols, dtype, param_dtype) || !(eps >= 0.f)) return GAD_ERR_ARG;
    if (rows == 0) return GAD_OK;
    if (!x || !y || !mean || !rstd || (ldx && ldx < cols) || ldy < cols) return GAD_ERR_ARG;
    const NormCall a{x, gamma, beta, ldx, rows, cols, param_dtype == GAD_F32, (((uintptr_t)gamma | (uintptr_t)beta) & 15) == 0, eps, y, ldy, mean, rstd};
    const cudaStream_t s = (cudaStream_t)stream;
    try {
        if (dtype == GAD_F32) norm_pick<float>(a, s);
        else if (dtype == GAD_F16) norm_pick<__half>(a, s);
        else norm_pick<__nv_bfloat16>(a, s);
    } catch (...) {   // (the table of occupancies could not grow)
        return GAD_ERR_OOM;
    }
    ++g_kernel_launches;
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}

extern "C" int gad_layer_norm_backward_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes) {
    if (!bytes || rows < 0 || cols < 1) return GAD_ERR_ARG;
    *bytes = (size_t)std::min<int64_t>(rows, gad::kNormBlocks) * 2 * (size_t)cols * sizeof(float);
    return GAD_OK;
}

extern "C" int gad_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t rows, int32_t cols, int32_t dtype, const void* gamma,
                                       int32_t param_dtype, const float* mean, const float* rstd, void* dx, int64_t lddx, void* dgamma, void* dbeta, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    using namespace gad;
    if (!norm_sizes_ok(rows, cols, dtype, param_dtype)) return GAD_ERR_ARG;
    if (rows > 0 && (!dy || !x || !mean || !rstd || !dx || (lddy && lddy < cols) || (ldx && ldx < cols) || lddx < cols)) return GAD_ERR_ARG;
    size_t need = 0;
    gad_layer_norm_backward_workspace_bytes(rows, cols, &need);
    if ((dgamma || dbeta) && need > 0 && (!workspace || workspace_bytes < need)) return GAD_ERR_OOM;
    const NormBackCall a{dy, x, gamma, lddy, ldx, rows, cols, param_dtype == GAD_F32, ((uintptr_t)gamma & 15) == 0, mean, rstd, dx, lddx, dgamma, dbeta, dgamma || dbeta ? (float*)workspace : nullptr};
    const cudaStream_t s = (cudaStream_t)stream;
    try {
        if (dtype == GAD_F32) norm_back_pick<float>(a, s);
        else if (dtype == GAD_F16) norm_back_pick<__half>(a, s);
        else norm_back_pick<__nv_bfloat16>(a, s);
    } catch (...) {   // (the table of occupancies could not grow)
        return GAD_ERR_OOM;
    }
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}
