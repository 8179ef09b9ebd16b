// Loss of an output layer with many classes, holding no more than a block of its logits, and the gradients: softmax cross entropy against labels, and distillation
// from a teacher's top logits.  With z_i = W h_i + b over all classes, p = softmax(z), p^T = softmax(z / T), q_i = softmax of row i's teacher logits / T:
//   l_i = a (lse(z) - z_y) + (1 - a) T^2 sum_j q_j (log q_j - log p^T_{c_j})
// Both kinds of target are one sparse list of (class, weight): tau = a [y] + (1 - a) T q at the teacher's classes.  Then
//   l_i = a lse(z) + (1 - a) T^2 (lse(z / T) + sum q log q) - sum_v tau_v z_v,     dl_i / dz = a p + (1 - a) T p^T - tau.
//
// One call: the rows' targets are sorted by class and the rows copied to the operand type (class_rows_kernel).  z = H W^T tile by tile leaves per row and tile
// half the largest value, the sums and sum tau z (kStats); class_finish_kernel joins them.  For gradients the rows are gone through in blocks: of a
// block the tiles leave z too, as 16-bit codes (fp32: as it is), class_grad_kernel turns it into G where it lies, and dH = G W and dW += G^T H follow
// (kOut).  So what is held of the rows x classes matrix is bounded (kBlockBytes), whatever its size.  Taking z again from H and W instead, once its row sums are
// known, needs no codes but a third more flops (8192 x 2048 bf16 against 100 003 classes: 10.7 ms, from codes 9.9 ms at that time, 8.7 now).  Going from z to G in strips of
// 512 to 1024 rows, while the codes are in the L2, cost more tiles than it saved bytes (4096 x 1024 against 32 768: 896 us instead of 851).
//
// Operands: fp16 and bfloat16 as they are.  fp32 in three bfloat16 parts (24 bits), of whose nine products the six that reach 2^-24 are summed.
// G is rounded to the operand type (fp32: not rounded), times a power of two that brings its largest possible value to 2^14 .. 2^15: in fp16 a probability of 1e-9 keeps
// eight bits.  One rounding of each term of a sum whose result is rounded to the same type: in the norm of a tensor the result's error grows by up to the square root of 2 (measured 1.0 to
// 1.5); a row of dH that is mostly its target's shares that one rounding, and is off by up to 2.4 times its own.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "class_gemm.cuh"
#include "gated_launch.cuh"
#include "operand_pack.cuh"
#include "skinny.cuh"

namespace gad {

namespace {

constexpr int kRowThreads = 128;
constexpr int kMostTargets = 1024;                       // teacher logits a row
// Bytes of probabilities and gradients of logits held at once, about a hundredth of the GPU's memory.  Several blocks of rows also hold the sums of dW in fp32 and read and
// write them (8192 x 2048 against 100 003 classes: one block of 1.6 GB 8.6 ms, two of 0.8 GB and 0.8 GB of sums 9.1 ms).
constexpr int64_t kBlockBytes = 2ll << 30;
constexpr int64_t kStartsBytes = kBlockBytes / 8;        // of target starts at once
constexpr float kLog2e = 1.44269504f;

template <class P> __device__ __forceinline__ float load_as_float(const void* p, int64_t i) { return to_float(reinterpret_cast<const P*>(p)[i]); }
__device__ __forceinline__ float load_typed(const void* p, int type, int64_t i) {
    return type == GAD_F32 ? load_as_float<float>(p, i) : type == GAD_F16 ? load_as_float<__half>(p, i) : load_as_float<__nv_bfloat16>(p, i);
}
__device__ __forceinline__ int64_t load_index(const void* p, int bytes, int64_t i) {
    return bytes == 8 ? reinterpret_cast<const int64_t*>(p)[i] : (int64_t)reinterpret_cast<const int32_t*>(p)[i];
}

struct RowArgs {
    const void* H; int64_t ldh; int cols, classes;
    const void* labels; int label_bytes;
    const void* tclasses; int tclass_bytes; const void* teacher; int teacher_type; int k;
    const float* weights;
    float hard, temperature;
    void* Hp; int64_t ldp, part_stride;
    int2* targets; int ntargets;
    uint16_t* starts; int nstarts, start_w;               // [rows x nstarts] first target at or behind every start_w-th class; or null
    float4* rowk;
    int64_t rows;
    struct RowShare* shares; unsigned* ticket;
    int32_t* status;
};

// What a block of the row kernels contributes to the scale of the gradients: rows that count, the largest coefficient of G.
struct RowShare { int n; float most; };

// Labels alone: a warp a row.  Bound by the copy of H (4096 x 1024 bf16: 6 us).
template <class T>
__global__ void __launch_bounds__(256) class_label_rows_kernel(const RowArgs a) {
    __shared__ RowShare part[8];
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    pdl_next();
    pdl_wait();
    if (r < a.rows) {
        const int64_t y = load_index(a.labels, a.label_bytes, r);
        const bool counts = y >= 0, bad = y >= a.classes;
        const float w = counts ? (a.weights ? a.weights[r] : 1.f) : 0.f;
        if (lane == 0) {
            a.targets[r] = make_int2(counts && !bad ? (int)y : INT_MAX, __float_as_int(counts && !bad ? 1.f : 0.f));
            a.rowk[r] = make_float4(counts ? 1.f : 0.f, 0.f, bad ? NAN : 0.f, w);
            part[threadIdx.x >> 5] = {counts, fabsf(w)};
        }
        pack_row<T>(reinterpret_cast<const T*>(a.H) + r * a.ldh, a.cols, counts, a.Hp, r * a.ldp, a.part_stride, lane, 32);
    } else if (lane == 0) part[threadIdx.x >> 5] = {0, 0.f};
    __syncthreads();
    if (threadIdx.x) return;
    RowShare mine = part[0];
    for (int i = 1; i < 8; ++i) { mine.n += part[i].n; mine.most = fmaxf(mine.most, part[i].most); }
    a.shares[blockIdx.x] = mine;
    if (blockIdx.x == 0) { *a.ticket = 0u; *a.status = 0; }
}

// A block a row; the copy of H, the sort of its targets (by counting, k^2 / 128 steps a thread) and where they start in every half tile (4096 x 2048 bf16, 65 targets:
// 29 us of 2.3 ms).  rowk = (coefficient of lse(z), of lse(z / T), sum of q log q with its factor, weight of the row); a row without target: (0, 0, 0, 0).
template <class T>
__global__ void __launch_bounds__(kRowThreads) class_rows_kernel(const RowArgs a) {
    extern __shared__ int sm_rows[];
    int* idx = sm_rows;                                   // [ntargets]
    float* tau = reinterpret_cast<float*>(sm_rows + a.ntargets);
    int* sorted = sm_rows + 2 * a.ntargets;
    __shared__ float red[2][kRowThreads / 32];
    __shared__ int bad, soft_any;
    const int64_t r = blockIdx.x;
    const int t = threadIdx.x, lane = t & 31, w = t >> 5;
    pdl_next();
    pdl_wait();
    if (t == 0) { bad = 0; soft_any = 0; }
    __syncthreads();
    float most = -INFINITY;
    for (int j = t; j < a.k; j += kRowThreads) {
        const int64_t c = load_index(a.tclasses, a.tclass_bytes, r * a.k + j);
        const float x = load_typed(a.teacher, a.teacher_type, r * a.k + j) / a.temperature;
        if (c >= a.classes) bad = 1;
        if (c >= 0) soft_any = 1;
        const bool used = c >= 0 && c < a.classes;
        idx[j] = used ? (int)c : INT_MAX;
        tau[j] = used ? x : -INFINITY;
        if (used) most = fmaxf(most, x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane == 0) red[0][w] = most;
    __syncthreads();
    for (int i = 0; i < kRowThreads / 32; ++i) most = fmaxf(most, red[0][i]);
    __syncthreads();
    float s = 0.f;
    for (int j = t; j < a.k; j += kRowThreads)
        if (idx[j] != INT_MAX) s += expf(tau[j] - most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) red[1][w] = s;
    __syncthreads();
    s = 0.f;
    for (int i = 0; i < kRowThreads / 32; ++i) s += red[1][i];
    const int64_t y = a.labels ? load_index(a.labels, a.label_bytes, r) : -1;
    const bool hard = y >= 0, soft = soft_any != 0;
    const float ha = hard ? a.hard : 0.f, hb = soft ? 1.f - a.hard : 0.f, tt = a.temperature;
    const bool counts = ha > 0.f || hb > 0.f;
    const float logs = logf(s);
    float ent = 0.f;
    __syncthreads();
    for (int j = t; j < a.k; j += kRowThreads)
        if (idx[j] != INT_MAX) {
            const float lq = tau[j] - most - logs, q = expf(lq);
            ent += q > 0.f ? q * lq : q;                  // (a q that is not a number stays one)
            tau[j] = hb > 0.f ? hb * tt * q : 0.f;        // (without weight nothing counts, nor a q that is no number)
            if (tau[j] == 0.f) idx[j] = INT_MAX;          // (its class may be masked: 0 times -infinity)
        }
    if (t == 0 && a.ntargets > a.k) {
        const bool used = hard && y < a.classes;
        if (hard && !used) bad = 1;
        idx[a.k] = used && ha > 0.f ? (int)y : INT_MAX;
        tau[a.k] = ha;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ent += __shfl_xor_sync(0xffffffffu, ent, o);
    if (lane == 0) red[0][w] = ent;
    __syncthreads();
    ent = 0.f;
    for (int i = 0; i < kRowThreads / 32; ++i) ent += red[0][i];
    // by class, equal ones in the order given: each target's place is the number of those in front of it
    for (int j = t; j < a.ntargets; j += kRowThreads) {
        const int c = idx[j];
        int at = 0;
        for (int i = 0; i < a.ntargets; ++i) at += idx[i] < c || (idx[i] == c && i < j);
        const float tv = tau[j];
        a.targets[r * a.ntargets + at] = make_int2(c, __float_as_int(c == INT_MAX ? 0.f : tv));
        sorted[at] = c;
    }
    if (a.starts) {
        __syncthreads();
        for (int b = t; b < a.nstarts; b += kRowThreads) {
            int e = 0, hi = a.ntargets;
            while (e < hi) {
                const int mid = (e + hi) >> 1;
                if (sorted[mid] < b * a.start_w) e = mid + 1; else hi = mid;
            }
            a.starts[r * a.nstarts + b] = (uint16_t)e;
        }
    }
    const float weight = counts ? (a.weights ? a.weights[r] : 1.f) : 0.f;
    if (t == 0) a.rowk[r] = make_float4(ha, hb * tt * tt, counts && bad ? NAN : hb > 0.f ? hb * tt * tt * ent : 0.f, weight);
    pack_row<T>(reinterpret_cast<const T*>(a.H) + r * a.ldh, a.cols, counts, a.Hp, r * a.ldp, a.part_stride, t, kRowThreads);
    if (t == 0) {
        a.shares[r] = {counts, counts ? fabsf(weight) * (ha + hb * tt) : 0.f};
        if (r == 0) { *a.ticket = 0u; *a.status = 0; }
    }
}

// Where a row's targets start in every half tile, for a block of rows: where the table for all rows at once (rows x classes / 64 bytes, from the rows kernel) would be larger than
// kStartsBytes.  A block a row, bound by the latency of its look-ups (16 384 rows of 9 targets against 131 072 classes 90 us of 6.1 ms, in the rows kernel 25).
__global__ void __launch_bounds__(128) class_starts_kernel(const int2* __restrict__ targets, int ntargets, uint16_t* __restrict__ starts, int nstarts, int start_w) {
    const int64_t r = blockIdx.x;
    pdl_next();
    pdl_wait();
    after_wait(targets);
    const int2* list = targets + r * ntargets;
    for (int b = threadIdx.x; b < nstarts; b += 128) {
        int e = 0, hi = ntargets;
        while (e < hi) {
            const int mid = (e + hi) >> 1;
            if (list[mid].x < b * start_w) e = mid + 1; else hi = mid;
        }
        starts[r * nstarts + b] = (uint16_t)e;
    }
}

// Class vectors that no descriptor can reach (fp32, or rows that do not start on 16 bytes) as operands: a warp a row, bound by memory (16 384 x 512 fp32 to three parts: 14 us).
template <class T>
__global__ void __launch_bounds__(256) class_pack_kernel(const T* __restrict__ W, int64_t ldw, int rows, int cols, void* Wp, int64_t ldp, int64_t part_stride) {
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_next();
    pdl_wait();
    if (r < rows) pack_row<T>(W + r * ldw, cols, true, Wp, r * ldp, part_stride, threadIdx.x & 31, 32);
}

// Statistics of a few rows (up to 4: serving): reading W is all that costs, and a tile of 256 rows on the tensor cores mostly multiplies zeros (one row, 128 000 x 4096
// bf16: 237 us at the card's power limit).  A warp takes four classes at a time, each lane every 32nd vector of their rows; the rows of H lie in shared memory in fp32.
// The 4 NR sums over lanes are halved at each of the first exchanges, so that lane l ends up with sum l / (32 / (4 NR)), and keeps its own running softmax
// over the classes it sees, in ascending order.  Bound by HBM: one row of 4096 against 128 000 classes bf16 158 us, 6.65 TB/s; with
// four rows 186 us in all, and with eight the multiply-adds bound it: 407 us, where class_some_kernel takes 203.
constexpr int kFewRows = 4, kFewBlocks = 296, kFewSmem = 160 << 10;
struct FewArgs {
    const void* H; long long ldh;
    const void* W; long long ldw;
    int rows, cols, classes;
    const void* bias;
    const int2* targets; int ntargets;
    const float4* rowk;
    float sc, inv_t;
    float* z; long long ldz;                  // or null
    float4* stats;                            // [blocks x rows]
};
template <class T, int NR, int NL, bool WIDE>
__global__ void __launch_bounds__(256, 2) class_few_kernel(const FewArgs a) {
    extern __shared__ float h[];              // [NR][cols, rounded up to a vector]
    __shared__ float4 sm[8][32];
    constexpr int VEC = WIDE ? 16 / sizeof(T) : 1, C = 4 * NR, LC = NR == 1 ? 2 : NR == 2 ? 3 : 4;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, ldv = (a.cols + VEC - 1) / VEC * VEC;
    pdl_next();
    pdl_wait();
    for (int n = 0; n < NR; ++n) {
        const float4 k = n < a.rows ? a.rowk[n] : make_float4(0.f, 0.f, 0.f, 0.f);
        const bool counts = k.x > 0.f || k.y > 0.f;
        for (int c = threadIdx.x; c < ldv; c += 256) h[n * ldv + c] = counts && c < a.cols ? to_float(reinterpret_cast<const T*>(a.H)[n * a.ldh + c]) : 0.f;
    }
    __syncthreads();
    const int idx = lane >> (5 - LC), kc = idx / NR, row = idx % NR;   // this lane's class of the four, and row
    const bool mine = (lane & ((1 << (5 - LC)) - 1)) == 0 && row < a.rows;
    const int2* tg = a.targets + (long long)min(row, a.rows - 1) * a.ntargets;
    float m = -INFINITY, s1 = 0.f, s2 = 0.f, dot = 0.f;
    int e = 0;
    const int whole = WIDE ? a.cols / VEC * VEC : a.cols, last = a.z ? (int)a.ldz : a.classes;
    for (int c0 = (blockIdx.x * 8 + w) * 4; c0 < last; c0 += gridDim.x * 32) {
        float acc[C];
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = 0.f;
        const T* wr[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) wr[k] = reinterpret_cast<const T*>(a.W) + (long long)min(c0 + k, a.classes - 1) * a.ldw;
        if constexpr (WIDE) {
#pragma unroll 2
            for (int x = lane * VEC; x < whole; x += 32 * VEC) {
                uint4 u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k] = __ldcs(reinterpret_cast<const uint4*>(wr[k] + x));
                float v[4][VEC];
#pragma unroll
                for (int k = 0; k < 4; ++k) unpack_vec<T, VEC>(u[k], v[k]);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    float hv[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; j += 4) {
                        const float4 q = *reinterpret_cast<const float4*>(h + n * ldv + x + j);
                        hv[j] = q.x; hv[j + 1] = q.y; hv[j + 2] = q.z; hv[j + 3] = q.w;
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) acc[k * NR + n] = fmaf(v[k][j], hv[j], acc[k * NR + n]);
                }
            }
        }
        for (int x = (WIDE ? whole : 0) + lane; x < a.cols; x += 32)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float v = to_float(wr[k][x]);
#pragma unroll
                for (int n = 0; n < NR; ++n) acc[k * NR + n] = fmaf(v, h[n * ldv + x], acc[k * NR + n]);
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
        const int c = c0 + kc;
        const bool cls = c < a.classes;
        const float b = cls ? (a.bias ? to_float(reinterpret_cast<const T*>(a.bias)[c]) : 0.f) : -INFINITY;
        const float z = cls ? (acc[0] + b) * a.sc : -INFINITY;
        if (a.z && mine && c < last) a.z[row * a.ldz + c] = z;
        if (!cls) continue;
        const float most = fmaxf(m, z), base = most == -INFINITY ? 0.f : most;
        s1 = s1 * exp2_fast(m - base) + exp2_fast(z - base);
        if (NL == 2) s2 = s2 * exp2_fast((m - base) * a.inv_t) + exp2_fast((z - base) * a.inv_t);
        m = most;
        while (e < a.ntargets && tg[e].x < c) ++e;
        for (; e < a.ntargets && tg[e].x == c; ++e) dot = fmaf(__int_as_float(tg[e].y), z, dot);
    }
    sm[w][lane] = make_float4(m, s1, s2, dot);
    __syncthreads();
    if (threadIdx.x >= a.rows) return;
    float4 at = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    for (int i = 0; i < 8; ++i)
        for (int k = 0; k < 4; ++k) {
            const float4 v = sm[i][(k * NR + threadIdx.x) << (5 - LC)];
            const float most = fmaxf(at.x, v.x), base = most == -INFINITY ? 0.f : most;
            at.y = at.y * exp2f(at.x - base) + v.y * exp2f(v.x - base);
            if (NL == 2) at.z = at.z * exp2f((at.x - base) * a.inv_t) + v.z * exp2f((v.x - base) * a.inv_t);
            at.x = most;
            at.w += v.w;
        }
    a.stats[(long long)blockIdx.x * a.rows + threadIdx.x] = at;
}

// Statistics of 5 to 16 rows of 16-bit operands that fit shared memory (a batch of serving), still bound by reading W: sixteen classes a warp as the rows of
// mma.m16n8k16, eight rows of H as its columns.  (tcgen05 has 128 rows at least: with H as A it multiplies zeros at the card's power limit, 16 rows of 4096 against 128 000
// classes 320 us, here 206, 5.1 TB/s; 32 rows of 2048, at 250 registers a lane, took 144 us here and 125 as tiles.)  The order of the terms is free as long as both operands have the same one, so that a lane's fragments are the 16 bytes it loads: of
// each 32 values lane (g, t) takes 8 t .. 8 t + 7 of class g, of class g + 8 and of row g of H; two products.  A lane ends up with classes g and g + 8 of rows
// 2 t and 2 t + 1 and keeps their running softmax.
constexpr int kSomeRows = 16, kSomeSmem = 200 << 10;
template <class T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Bytes between the rows of H: eight rows of 64 bytes meet no bank twice.
__host__ __device__ __forceinline__ int some_stride(int cols) { return (cols * 2 + 127) / 128 * 128 + 64; }
// NT: groups of eight rows.
constexpr int kSomeWarps = 16;
template <class T, int NT, int NL>
__global__ void __launch_bounds__(32 * kSomeWarps, 1) class_some_kernel(const FewArgs a) {
    constexpr int WARPS = kSomeWarps, U = 4;             // U steps of 32 values are on their way while the U in front are multiplied
    extern __shared__ __align__(16) uint8_t hs[];
    __shared__ float4 sm[WARPS][8 * NT];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, stride = some_stride(a.cols);
    pdl_next();
    pdl_wait();
    for (int n = w; n < 8 * NT; n += WARPS) {
        const float4 k = n < a.rows ? a.rowk[n] : make_float4(0.f, 0.f, 0.f, 0.f);
        const bool counts = k.x > 0.f || k.y > 0.f;
        for (int c = lane; 2 * c < stride; c += 32)
            reinterpret_cast<T*>(hs + (long long)n * stride)[c] = counts && c < a.cols ? reinterpret_cast<const T*>(a.H)[n * a.ldh + c] : from_float<T>(0.f);
    }
    __syncthreads();
    float m[2 * NT], s1[2 * NT], s2[2 * NT], dot[2 * NT];
    int e[2 * NT], cur[2 * NT];
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) {
        const int n = i / 2 * 8 + 2 * t + (i & 1);
        m[i] = -INFINITY; s1[i] = s2[i] = dot[i] = 0.f;
        e[i] = 0;
        cur[i] = n < a.rows ? a.targets[(long long)n * a.ntargets].x : INT_MAX;
    }
    const int last = a.z ? (int)a.ldz : a.classes, steps = (a.cols + 31) / 32;
    const uint8_t* hb = hs + g * stride + t * 16;
    for (int c0 = (blockIdx.x * WARPS + w) * 16; c0 < last; c0 += gridDim.x * WARPS * 16) {
        float sum[NT][4];
#pragma unroll
        for (int k = 0; k < NT; ++k) sum[k][0] = sum[k][1] = sum[k][2] = sum[k][3] = 0.f;
        const T* w0 = reinterpret_cast<const T*>(a.W) + (long long)min(c0 + g, a.classes - 1) * a.ldw;
        const T* w1 = reinterpret_cast<const T*>(a.W) + (long long)min(c0 + g + 8, a.classes - 1) * a.ldw;
        uint4 u[U], v[U];
        const auto load = [&](int i0) {
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int c = 32 * (i0 + j) + 8 * t;
                if (c + 8 <= a.cols) {
                    u[j] = __ldcs(reinterpret_cast<const uint4*>(w0 + c));
                    v[j] = __ldcs(reinterpret_cast<const uint4*>(w1 + c));
                } else {                                     // the end of the rows
                    RowVec<T, 8> q, r;
                    load_raw<T, 8>(w0, c, a.cols, q);
                    load_raw<T, 8>(w1, c, a.cols, r);
                    u[j] = q.u; v[j] = r.u;
                }
            }
        };
        load(0);
        float acc[NT][4];
        for (int i0 = 0; i0 < steps; i0 += U) {
            if (i0 % 32 == 0) {                              // (the accumulator is cut off at every addition: 64 of them at most)
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) { if (i0) sum[k][j] += acc[k][j]; acc[k][j] = 0.f; }
            }
            uint4 pu[U], pv[U];
#pragma unroll
            for (int j = 0; j < U; ++j) { pu[j] = u[j]; pv[j] = v[j]; }
            if (i0 + U < steps) load(i0 + U);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (i0 + j >= steps) break;
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const uint4 b = *reinterpret_cast<const uint4*>(hb + k * 8 * stride + 64 * (i0 + j));
                    mma_16x8x16<T>(acc[k], pu[j].x, pv[j].x, pu[j].y, pv[j].y, b.x, b.y);
                    mma_16x8x16<T>(acc[k], pu[j].z, pv[j].z, pu[j].w, pv[j].w, b.z, b.w);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < NT; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[k][j] += acc[k][j];
        float bias[2];
        bool cls[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int c = c0 + g + 8 * r;
            cls[r] = c < a.classes;
            bias[r] = cls[r] && a.bias ? to_float(reinterpret_cast<const T*>(a.bias)[c]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            const int n = i / 2 * 8 + 2 * t + (i & 1);
            float z[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int c = c0 + g + 8 * r;
                z[r] = cls[r] ? (sum[i / 2][2 * r + (i & 1)] + bias[r]) * a.sc : -INFINITY;
                if (a.z && n < a.rows && c < last) a.z[(long long)n * a.ldz + c] = z[r];
                while (cur[i] <= c) {                        // (classes ascend; INT_MAX is none)
                    if (cur[i] == c) dot[i] = fmaf(__int_as_float(a.targets[(long long)n * a.ntargets + e[i]].y), z[r], dot[i]);
                    cur[i] = ++e[i] < a.ntargets ? a.targets[(long long)n * a.ntargets + e[i]].x : INT_MAX;
                }
            }
            const float most = fmaxf(m[i], fmaxf(z[0], z[1])), base = most == -INFINITY ? 0.f : most;
            s1[i] = fmaf(s1[i], exp2_fast(m[i] - base), exp2_fast(z[0] - base) + exp2_fast(z[1] - base));
            if (NL == 2) s2[i] = fmaf(s2[i], exp2_fast((m[i] - base) * a.inv_t), exp2_fast((z[0] - base) * a.inv_t) + exp2_fast((z[1] - base) * a.inv_t));
            m[i] = most;
        }
    }
    // lanes of the same rows (equal t), then warps, in order
    const auto join = [&](float4& u, const float4& v) {
        const float most = fmaxf(u.x, v.x), base = most == -INFINITY ? 0.f : most;
        u.y = u.y * exp2f(u.x - base) + v.y * exp2f(v.x - base);
        if (NL == 2) u.z = u.z * exp2f((u.x - base) * a.inv_t) + v.z * exp2f((v.x - base) * a.inv_t);
        u.x = most;
        u.w += v.w;
    };
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) {
        float4 at = make_float4(m[i], s1[i], s2[i], dot[i]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            float4 v = make_float4(__shfl_xor_sync(0xffffffffu, at.x, o), __shfl_xor_sync(0xffffffffu, at.y, o), __shfl_xor_sync(0xffffffffu, at.z, o), __shfl_xor_sync(0xffffffffu, at.w, o));
            if (lane & o) { join(v, at); at = v; } else join(at, v);
        }
        if (g == 0) sm[w][i / 2 * 8 + 2 * t + (i & 1)] = at;
    }
    __syncthreads();
    if (threadIdx.x >= a.rows) return;
    float4 at = sm[0][threadIdx.x];
    for (int i = 1; i < WARPS; ++i) join(at, sm[i][threadIdx.x]);
    a.stats[(long long)blockIdx.x * a.rows + threadIdx.x] = at;
}

// Log-probabilities of 3 to 64 rows' actions (16-bit operands, no gradients: scoring), bound by reading W: classes as the rows of the product (skinny.cuh), a class a thread, sixteen rows of H in its
// registers, for which it keeps a running softmax over the classes it sees; joined over threads at the end, over blocks by class_finish_kernel.  Sums are added up in chunks of 256 terms: the drain has
// time, and a ratio of probabilities shows what a logit has lost.  Whole calls, 4096 columns against 128 000 classes: 3 rows 178 us (class_few_kernel 184; one row 177 and 164), 16 rows 179
// (class_some_kernel 195), 64 rows 176 (tiles of 256 rows 291); 1024 against 32 768: 16 rows 19 us (24).
constexpr int kScoreLeast = 3;
constexpr int kScoreRows = 16 * SK_GROUPS;
struct ScoreArgs {
    int rows, width, classes, tiles, nkb, stages, bf16;
    int32_t* err;
    const void* bias; int bias_type;
    float sc;
    const int2* targets;                      // [rows]
    float4* stats;                            // [blocks x rows]
};
__global__ void __launch_bounds__(SK_THREADS, 1) class_score_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmH, const __grid_constant__ ScoreArgs a) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int CHUNK = 4;
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* sm = smem_raw + pad;
    const uint32_t sm_addr = raw_addr + pad;
    const uint32_t bars = sm_addr + SK_RING;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (SK_MOST_STAGES + s); };
    auto tfull = [&](int i) { return bars + 8u * (2 * SK_MOST_STAGES + i); };
    auto tempty = [&](int i) { return bars + 8u * (2 * SK_MOST_STAGES + 2 + i); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + SK_RING + 8 * (2 * SK_MOST_STAGES + 4));
    volatile uint32_t* abort_flag = tmem_slot + 1;
    float2* sums = reinterpret_cast<float2*>(sm + SK_RING + 512);          // [4][kScoreRows] of a quarter of the lanes each
    int* target = reinterpret_cast<int*>(sums + 4 * kScoreRows);
    float* dots = reinterpret_cast<float*>(target + kScoreRows);
    static_assert(4 * kScoreRows * 8 + 8 * kScoreRows <= SK_XCH, "fits where g and u are exchanged");
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(tfull(i), 1); mbar_init(tempty(i), SK_DRAIN / 32); }
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_next();
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(CT_TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t stage_bytes = SK_A + (uint32_t)a.width * (CT_K * 2);
    float m[16], s[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) { m[j] = -INFINITY; s[j] = 0.f; }
    if (warp == 0) {
        if (lane == 0) {
            const auto load_w = [&](int st, int tile, int kb) {
                mbar_expect_tx(full(st), stage_bytes);
                tma_load_3d(sm_addr + st * stage_bytes, &tmW, kb * CT_K, tile * SK_M, 0, full(st));
            };
            const auto load_h = [&](int st, int kb) { tma_load_3d(sm_addr + st * stage_bytes + SK_A, &tmH, kb * CT_K, 0, 0, full(st)); };
            const int ahead = min(a.stages, a.nkb);       // W is the caller's: it need not wait for the copy of H
            for (int i = 0; i < ahead; ++i) load_w(i, blockIdx.x, i);
            pdl_wait();
            for (int i = 0; i < ahead; ++i) load_h(i, i);
            int st = ahead == a.stages ? 0 : ahead, done = ahead;
            uint32_t phase = ahead == a.stages ? 1u : 0u;
            bool ok = true;
            for (int t = blockIdx.x; t < a.tiles && ok; t += gridDim.x) {
                for (int kb = done; kb < a.nkb; ++kb) {
                    if (!(ok = mbar_wait(empty(st), phase ^ 1u, abort_flag, a.err, 61))) break;
                    load_w(st, t, kb);
                    load_h(st, kb);
                    if (++st == a.stages) { st = 0; phase ^= 1u; }
                }
                done = 0;
            }
        }
    } else if (warp == 1) {
        int st = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        const uint32_t idesc = instr_desc_f16(a.width, SK_M) | (a.bf16 ? (1u << 7) | (1u << 10) : 0u);
        bool ok = true;
        for (int t = blockIdx.x; t < a.tiles && ok; t += gridDim.x)
            for (int i = 0; i < a.nkb; ++i) {
                const bool first = i % CHUNK == 0, last = i % CHUNK == CHUNK - 1 || i == a.nkb - 1;
                if (first) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(tempty(acc), acc_phase ^ 1u, abort_flag, a.err, 62)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                }
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(st), phase, abort_flag, a.err, 63)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base = sm_addr + st * stage_bytes;
                const uint64_t da = smem_desc(base), db = smem_desc(base + SK_A);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < CT_K / 16; ++ks) mma_f16_one(tmem_base + (uint32_t)(acc * 256), da + 2 * ks, db + 2 * ks, idesc, !first || ks != 0 ? 1u : 0u);
                    mma_commit(empty(st));
                    if (last) mma_commit(tfull(acc));
                }
                __syncwarp();
                if (++st == a.stages) { st = 0; phase ^= 1u; }
                if (last && ++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
    } else {
        const int q = warp & 3, c0 = ((warp - 2) >> 2) * 16;
        pdl_wait();
        for (int i = threadIdx.x - 64; i < kScoreRows; i += SK_DRAIN) { target[i] = i < a.rows ? a.targets[i].x : INT_MAX; dots[i] = 0.f; }
        all_drain(true);
        int acc = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        for (int t = blockIdx.x; t < a.tiles && ok; t += gridDim.x) {
            const int c = t * SK_M + q * 32 + lane;
            const bool cls = c < a.classes;
            const float b = cls && a.bias ? load_typed(a.bias, a.bias_type, c) : 0.f;
            float z[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) z[j] = 0.f;
            for (int i = 0; i < a.nkb; i += CHUNK) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(tfull(acc), acc_phase, abort_flag, a.err, 66)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (c0 < a.rows) {
                    float v[16];
                    tmem_ld16(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * 256 + c0), v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) z[j] += v[j];
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(tempty(acc));
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
            if (!ok || c0 >= a.rows || !cls) continue;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float x = (z[j] + b) * a.sc;
                if (target[c0 + j] == c) dots[c0 + j] = x;
                const float most = fmaxf(m[j], x), base = most == -INFINITY ? 0.f : most;
                s[j] = fmaf(s[j], exp2_fast(m[j] - base), exp2_fast(x - base));
                m[j] = most;                              // (a logit that is no number stays in the sum)
            }
        }
        if (c0 < a.rows) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float most = m[j];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                s[j] *= exp2_fast(m[j] - (most == -INFINITY ? 0.f : most));
                m[j] = most;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
                if (lane == 0) sums[q * kScoreRows + c0 + j] = make_float2(m[j], s[j]);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < a.rows) {
        float most = -INFINITY, sum = 0.f;
        for (int q = 0; q < 4; ++q) most = fmaxf(most, sums[q * kScoreRows + threadIdx.x].x);
        const float base = most == -INFINITY ? 0.f : most;
        for (int q = 0; q < 4; ++q) sum += sums[q * kScoreRows + threadIdx.x].y * exp2f(sums[q * kScoreRows + threadIdx.x].x - base);
        a.stats[(long long)blockIdx.x * a.rows + threadIdx.x] = make_float4(most, sum, 0.f, dots[threadIdx.x]);
    }
    // Tear-down: after a time-out loads in flight get a bounded chance to land.
    if (*abort_flag && threadIdx.x == 0)
        for (int st = 0; st < a.stages; ++st)
            for (uint32_t i = 0; i < 4096u; ++i)
                if (mbar_try_wait(full(st), 0) || mbar_try_wait(full(st), 1)) break;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(CT_TMEM));
    }
}

constexpr int kFinishRows = 8;

// The policy loss: with lp the log-probability of a row's label, r = exp(lp - old), its row loss is  -min(r A, clip(r, lo, hi) A) + kl (exp(ref - lp) - (ref - lp) - 1).
struct PolicyArgs {
    const float *old, *advantages, *ref;          // of this block of rows; ref null: no KL term.  old null: no policy loss
    float lo, hi, kl;
    float* logp;
    float* most;                                  // [blocks] largest coefficient of G among a block's rows
};

struct FinishArgs {
    const float4* stats; int parts, rows;
    float4* rowk;
    PolicyArgs policy;
    float sc, inv_t, temperature;
    float4* rowc; float* row_loss;
    double* shares; int share0, nshares;          // of the loss: a block's sum of weighted row losses
    const RowShare* row_shares; int nrow_shares;
    unsigned* ticket;
    float scale; int mean, first, final;
    float *scal, *loss;
};

// The parts of a row's statistics joined (bound by the latency of its loads: 4096 rows of 256 parts 12 us): a block has 8 rows, 32 threads each, every 32nd part a thread; joined pairwise in a fixed order.  The block that comes last
// writes, for the first block of rows, scal[0], a power of two that brings the largest coefficient of G to 2^14 .. 2^15, [1]: scale / counted rows / that,
// [2]: scale / counted rows; and for the last one the loss.  [3] and [4]: factors of a block's sums and of what they add up to.  The coefficients of a policy loss are
// known when its rows are finished, block by block, so each block of rows has a power of two of its own, and leaves it out of the sums.
template <int NL>
__global__ void __launch_bounds__(256) class_finish_kernel(const FinishArgs a) {
    __shared__ float4 sm[8][kFinishRows];
    __shared__ bool last;
    __shared__ double smt[8];
    __shared__ RowShare smr[8];
    const int rl = threadIdx.x % kFinishRows, lane = threadIdx.x & 31, w = threadIdx.x >> 5, r = blockIdx.x * kFinishRows + rl;
    pdl_next();
    pdl_wait();
    const float inv_t = a.inv_t;
    const float4 none = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    const auto join = [&](const float4& u, const float4& v) {
        const float most = fmaxf(u.x, v.x), base = most == -INFINITY ? 0.f : most;
        float4 o;
        o.x = most;
        o.y = u.y * exp2f(u.x - base) + v.y * exp2f(v.x - base);
        o.z = NL == 2 ? u.z * exp2f((u.x - base) * inv_t) + v.z * exp2f((v.x - base) * inv_t) : 0.f;
        o.w = u.w + v.w;
        return o;
    };
    float4 at = none;
    if (r < a.rows)
        for (int p = threadIdx.x / kFinishRows; p < a.parts; p += 128) {
            float4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = p + 32 * i < a.parts ? a.stats[(int64_t)(p + 32 * i) * a.rows + r] : none;
            at = join(at, join(join(v[0], v[1]), join(v[2], v[3])));
        }
#pragma unroll
    for (int o = kFinishRows; o < 32; o <<= 1) {
        const float4 v = make_float4(__shfl_xor_sync(0xffffffffu, at.x, o), __shfl_xor_sync(0xffffffffu, at.y, o), __shfl_xor_sync(0xffffffffu, at.z, o), __shfl_xor_sync(0xffffffffu, at.w, o));
        at = lane & o ? join(v, at) : join(at, v);
    }
    if (lane < kFinishRows) sm[w][lane] = at;
    __syncthreads();
    if (w == 0) {
        double mine = 0.0;
        float coefficient = 0.f;
        if (lane < kFinishRows && r < a.rows) {
            at = sm[0][lane];
            for (int i = 1; i < 8; ++i) at = join(at, sm[i][lane]);
            const float4 k = a.rowk[r];
            // in log2: of the (first) softmax, whose logits were scaled by sc, and of the second
            const float l1 = at.x + log2f(at.y), l2 = NL == 2 ? at.x * inv_t + log2f(at.z) : l1;
            const float ln2 = 0.693147181f;
            const bool counts = k.x > 0.f || k.y > 0.f;
            float l = counts ? k.x * (l1 * ln2) + k.y * (l2 * ln2) + k.z - at.w / a.sc : 0.f;
            if (a.policy.old) {
                const PolicyArgs& y = a.policy;
                float lp = 0.f, slope = 0.f;                        // slope: of the row loss by lp
                if (counts) {
                    // dl / dz = slope (one-hot - p): what G = w (p - tau) is given for w, tau = 1
                    lp = (at.w - l1) * ln2 - k.z;
                    const float adv = y.advantages[r], ratio = expf(lp - y.old[r]), plain = ratio * adv, held = fminf(fmaxf(ratio, y.lo), y.hi) * adv;
                    const bool clipped = plain > held;              // (a product that is no number is taken)
                    l = clipped ? -held : -plain;
                    slope = clipped ? 0.f : -plain;
                    if (y.ref) {
                        const float d = y.ref[r] - lp, e = expm1f(d);
                        l = fmaf(y.kl, e - d, l);
                        slope = fmaf(-y.kl, e, slope);
                    }
                    if (k.z != k.z) slope = 0.f;                    // a label that is no class: the loss says so, the gradients are without the row
                }
                y.logp[r] = lp;
                const float c = counts ? -slope * k.w : 0.f;
                a.rowk[r].w = c;
                coefficient = fabsf(c);
            }
            a.row_loss[r] = l;
            // gradient: a p + (1 - a) T p^T; with one softmax both coefficients are its
            const float ca = k.x, cb = k.y / a.temperature;
            if (a.rowc) a.rowc[r] = NL == 2 ? make_float4(ca, cb, l1, l2) : make_float4(ca + cb, 0.f, l1, 0.f);
            if (counts) mine = (double)k.w * (double)l;
        }
#pragma unroll
        for (int o = 1; o < kFinishRows; o <<= 1) {
            mine += __shfl_xor_sync(0xffffffffu, mine, o);
            coefficient = fmaxf(coefficient, __shfl_xor_sync(0xffffffffu, coefficient, o));
        }
        if (lane == 0) {
            if (a.policy.old) a.policy.most[blockIdx.x] = coefficient;
            a.shares[a.share0 + blockIdx.x] = mine;
            __threadfence();
            last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (a.first || a.policy.old) {
        RowShare rows{0, 0.f};
        for (int i = threadIdx.x; i < a.nrow_shares; i += 256) {
            const RowShare v = a.row_shares[i];
            rows.n += v.n;
            rows.most = fmaxf(rows.most, v.most);
        }
        if (a.policy.old) {
            rows.most = 0.f;
            for (int i = threadIdx.x; i < gridDim.x; i += 256) rows.most = fmaxf(rows.most, __ldcg(a.policy.most + i));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            rows.n += __shfl_xor_sync(0xffffffffu, rows.n, o);
            rows.most = fmaxf(rows.most, __shfl_xor_sync(0xffffffffu, rows.most, o));
        }
        if (lane == 0) smr[w] = rows;
    }
    double all = 0.0;
    if (a.final)
        for (int i = threadIdx.x; i < a.nshares; i += 256) all += __ldcg(a.shares + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    if (lane == 0) smt[w] = all;
    __syncthreads();
    if (threadIdx.x) return;
    if (a.first || a.policy.old) {
        RowShare v = smr[0];
        for (int i = 1; i < 8; ++i) { v.n += smr[i].n; v.most = fmaxf(v.most, smr[i].most); }
        const double f = a.mean ? (v.n ? (double)a.scale / v.n : 0.0) : (double)a.scale;
        const int e = v.most > 0.f && v.most < INFINITY ? 14 - ilogbf(v.most) : 0;
        const float g = ldexpf(1.f, max(-100, min(100, e)));
        a.scal[0] = g;
        a.scal[1] = (float)(f / (double)g);
        a.scal[2] = (float)f;
        a.scal[3] = a.policy.old ? 1.f / g : 1.f;
        a.scal[4] = a.policy.old ? (float)f : a.scal[1];
    }
    if (a.final) {
        all = smt[0];
        for (int i = 1; i < 8; ++i) all += smt[i];
        a.loss[0] = (float)((double)a.scal[2] * all);
    }
    *a.ticket = 0u;                               // for the next block of rows
}

// G from what the tiles left of z, in its place (16-bit codes) or beside it (fp32): G = w (a p + (1 - a) T p^T - tau) times scal[0], in the operand type or (T = float) in
// three bfloat16 parts.  A warp takes 1024 classes of a row at a time, a block 32 rows of them, so column sums (for db, before any rounding) cost one
// exchange.  Bound by memory: 4 bytes a value (4096 x 32 768 bf16 104 us, 5.2 TB/s).
struct GradArgs {
    const void* z; long long ldz;             // codes or fp32 [rows x ldz]
    void* G; long long ldg, part_stride;
    const float4* stats; int half_w;          // .x = largest value of (part, row)
    const float4 *rowc, *rowk;
    const int2* targets; int ntargets;
    const float* scal;
    float inv_t, code_unit;                   // code_unit: of z a code (1 / code_steps)
    float* colsum;                            // [row blocks x ldg] or null
    int rows, classes;
};
template <class T, class Z, int NL, bool SUMS>
__global__ void __launch_bounds__(256) class_grad_kernel(const GradArgs a) {
    constexpr int SEG = 4;                    // 256 classes (8 a lane) each
    __shared__ float sm[SUMS ? 8 : 1][256 + 8];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c0 = blockIdx.x * 256 * SEG;
    pdl_next();
    pdl_wait();
    const float gs = a.scal[0];
    float sums[SUMS ? SEG : 1][8];
#pragma unroll
    for (int s = 0; s < (SUMS ? SEG : 1); ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[s][j] = 0.f;
    constexpr int LOADS = sizeof(Z) / 2;
    for (int i = 0; i < 4; ++i) {
        const int r = blockIdx.y * 32 + 8 * i + w;
        if (r >= a.rows) break;
        uint4 q[SEG][LOADS];                  // all loads of a row first
        float m[SEG];
#pragma unroll
        for (int s = 0; s < SEG; ++s) {
            const int c = c0 + 256 * s + 8 * lane;
            const bool in = c < a.ldg;        // (rows of G are whole tiles of 128 classes)
#pragma unroll
            for (int k = 0; k < LOADS; ++k)
                q[s][k] = in ? reinterpret_cast<const uint4*>(reinterpret_cast<const Z*>(a.z) + (long long)r * a.ldz + c)[k] : make_uint4(0u, 0u, 0u, 0u);
            m[s] = sizeof(Z) == 2 && in ? a.stats[(long long)(c / a.half_w) * a.rows + r].x : 0.f;
        }
        const float4 rc = a.rowc[r];
        const float f = a.rowk[r].w * gs;
        const int2* list = a.targets + (long long)r * a.ntargets;
        int e = 0;
        if (a.ntargets > 128) {               // the first target of these classes
            int hi = a.ntargets;
            while (e < hi) {
                const int mid = (e + hi) >> 1;
                if (list[mid].x < c0) e = mid + 1; else hi = mid;
            }
        }
        int2 t = e + lane < a.ntargets ? list[e + lane] : make_int2(INT_MAX, 0);
        // a sum that is not finite makes the whole row not a number, also where the code says zero; a row without weight is zero whatever it holds
        const float fa = f * rc.x + 0.f * rc.z, fb = f * rc.y;
        float v[SEG][8];
        if (f == 0.f) {
#pragma unroll
            for (int s = 0; s < SEG; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[s][j] = 0.f;
        } else {
#pragma unroll
            for (int s = 0; s < SEG; ++s) {
                const uint32_t* h = reinterpret_cast<const uint32_t*>(q[s]);
                float z[8];                   // log2 of exp(z) relative to the (first) sum
                if constexpr (sizeof(Z) == 2) {
                    const float d = m[s] - rc.z;
                    const float unit = NL == 2 ? a.code_unit : 1.f / kCodeSteps;
                    // a code behind the exponent of 2^23 is that number of steps above 2^23 of them: exact
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        z[j] = fmaf(__uint_as_float(__byte_perm(h[j >> 1], 0x4B000000u, j & 1 ? 0x7632 : 0x7610)), -unit, 8388608.f * unit) + d;
                    const uint32_t top = __vmaxu2(__vmaxu2(h[0], h[1]), __vmaxu2(h[2], h[3]));
                    if ((top >> 16) == kCodeZero || (top & 0xFFFFu) == kCodeZero) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (((h[j >> 1] >> (16 * (j & 1))) & 0xFFFFu) == kCodeZero) z[j] = -INFINITY;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(h[j]) - rc.z;
                }
                const float shift = fmaf(rc.z, a.inv_t, -rc.w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[s][j] = fa * exp2_fast(z[j]);
                    if (NL == 2) v[s][j] = fmaf(fb, exp2_fast(fmaf(z[j], a.inv_t, shift)), v[s][j]);
                }
            }
            // the row's targets among these classes, 32 of the list at a time (it is ascending)
            for (;;) {
                for (uint32_t hit = __ballot_sync(0xffffffffu, t.x >= c0 && t.x < c0 + 256 * SEG); hit; hit &= hit - 1) {
                    const int src = __ffs(hit) - 1, x = __shfl_sync(0xffffffffu, t.x, src) - c0 - 8 * lane;
                    const float d = f * __int_as_float(__shfl_sync(0xffffffffu, t.y, src));
#pragma unroll
                    for (int s = 0; s < SEG; ++s)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[s][j] -= x == 256 * s + j ? d : 0.f;
                }
                if (__shfl_sync(0xffffffffu, t.x, 31) >= c0 + 256 * SEG) break;
                e += 32;
                if (e >= a.ntargets) break;
                t = e + lane < a.ntargets ? list[e + lane] : make_int2(INT_MAX, 0);
            }
        }
#pragma unroll
        for (int s = 0; s < SEG; ++s) {
            const int c = c0 + 256 * s + 8 * lane;
            if (c >= a.ldg) break;
            if constexpr (SUMS) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[s][j] += v[s][j];
            }
            if constexpr (sizeof(T) == 4) {
                union { uint4 u; __nv_bfloat16 h[8]; } o[3];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __nv_bfloat16 p[3];
                    split3(v[s][j], p);
                    o[0].h[j] = p[0]; o[1].h[j] = p[1]; o[2].h[j] = p[2];
                }
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.G) + k * a.part_stride + (long long)r * a.ldg + c) = o[k].u;
            } else {
                union { uint4 u; T h[8]; } o;
#pragma unroll
                for (int j = 0; j < 8; ++j) o.h[j] = from_float<T>(v[s][j]);
                *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.G) + (long long)r * a.ldg + c) = o.u;
            }
        }
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int s = 0; s < SEG; ++s) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sm[w][8 * lane + j] = sums[s][j];
            __syncthreads();
            const int x = c0 + 256 * s + threadIdx.x;
            if (x < a.classes) {
                float d = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) d += sm[i][threadIdx.x];
                a.colsum[(long long)blockIdx.y * a.ldg + x] = d;
            }
            __syncthreads();
        }
    }
}

// The shares of the tiles that were cut along their reduction (from L2: 32 tiles of two shares 8 us), added up in order, and put where an uncut tile would have gone: four columns a thread, four (eight)
// rows of a tile a block.
template <class T>
__global__ void __launch_bounds__(256) class_join_kernel(const TileArgs a) {
    const int per_row = a.width / 4, rows = 256 / per_row, per_tile = CT_M / rows;
    const int i = blockIdx.x / per_tile, r = blockIdx.x % per_tile * rows + threadIdx.x / per_row, x = threadIdx.x % per_row * 4;
    pdl_next();
    pdl_wait();
    const TileAt t = tile_at(a, a.whole + (long long)i * a.shares);
    const int row = t.m * CT_M + r, c = t.n * a.width + x;
    if (row >= a.M || c >= a.N) return;
    const float factor = a.scal[a.add == kAddNone ? 1 : 4], pre = a.add == kAddNone ? 1.f : a.scal[3];
    const float* slot = a.slots + ((long long)i * a.shares * CT_M + r) * a.width + x;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < a.shares; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(slot + (long long)k * CT_M * a.width);
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
    }
    float* sum = a.sums + (long long)row * a.N + c;
    T* out = reinterpret_cast<T*>(a.C) + (long long)row * a.ldc + c;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (c + j >= a.N) break;
        if (a.add != kAddNone) s[j] *= pre;
        if (a.add == kAddMore || a.add == kAddLast) s[j] += sum[j];
        if (a.add == kAddFirst || a.add == kAddMore) sum[j] = s[j];
        else out[j] = from_float<T>(factor * s[j]);
    }
}

// db from the column sums of 32 rows each that class_grad_kernel leaves: 32 classes a block, each of its eight warps a run of them, in order.
template <class T>
__global__ void __launch_bounds__(256) class_bias_kernel(const float* __restrict__ colsum, int64_t ld, int n, int classes, const float* __restrict__ scal, int add, float* __restrict__ sums,
                                                         T* __restrict__ db) {
    __shared__ float sm[8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    const int per = (n + 7) / 8, lo = min(n, w * per), hi = min(n, lo + per);
    float s = 0.f;
    pdl_next();
    pdl_wait();
    after_wait(colsum);
    after_wait(scal);
    if (c < classes)
#pragma unroll 8
        for (int i = lo; i < hi; ++i) s += colsum[i * ld + c];
    sm[w][threadIdx.x & 31] = s;
    __syncthreads();
    if (w || c >= classes) return;
    s = 0.f;
    for (int k = 0; k < 8; ++k) s += sm[k][threadIdx.x & 31];
    if (add != kAddNone) s *= scal[3];
    if (add == kAddMore || add == kAddLast) s += sums[c];
    if (add == kAddFirst || add == kAddMore) sums[c] = s;
    else db[c] = from_float<T>(s * scal[add == kAddNone ? 1 : 4]);
}

template <class T>
__global__ void __launch_bounds__(256) class_zero_kernel(T* __restrict__ p, int64_t ld, int64_t rows, int cols) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_float<T>(0.f);
}
__global__ void class_empty_kernel(float* loss, int32_t* status) { *loss = 0.f; *status = 0; }

// ---------------------------------------------------------------------------------------------
// How a call is cut up; the same for the workspace and the launches.
// ---------------------------------------------------------------------------------------------
int width_for(int n) { return n <= 128 ? 128 : 256; }

int few_rows(int64_t n) { return n <= 1 ? 1 : n <= 2 ? 2 : 4; }
size_t some_smem(const gad_class_loss_args& a) { return (size_t)(a.rows <= 8 ? 8 : 16) * some_stride(a.cols); }
size_t few_smem(const gad_class_loss_args& a) { return 4 * (size_t)few_rows(a.rows) * (size_t)round_up(a.cols, 8); }

// Blocks of 64 terms of a chunk: 2048 terms are cut by 1.8e-6 of their sum; of fp32 operands 512, by 4.5e-7.  Longer logits go in tiles
// 128 wide: with chunks of 1024 the distillation of 4096 x 2048 took 2.71 ms instead of 2.34.
constexpr int kChunk = 32, kChunkParts = 8, kChunkPolicy = 16;

struct ClassPlan {
    int parts, pairs;                // operand parts, products of them
    bool grads, pack_w, few, some, add_up;   // add_up: logits longer than a chunk are added up in chunks
    bool score;                      // a few rows' log-probabilities alone
    bool sums;                       // policy: logits longer than a chunk are added up in chunks, in wide tiles
    bool starts_at_once;             // target starts of all rows from the rows kernel
    int ntargets, nl, save;
    float code_steps;
    int width_v, tiles_v, width_d, tiles_d;
    int64_t ldp, ldg;                // row lengths of the packed operands, and of z and G
    int64_t block;                   // rows a block
    int nblocks;
    // fp32 gradients of a policy loss in one block of rows: dH and dW in one launch of gated_gemm_kernel, which loads all parts of a block of the reduction at once (8192 x 256 against 2048 classes:
    // the whole call 177 us, with a launch each of class_gemm_kernel's 203)
    bool joint;
    Shape shape[2];
    Cut cut[2];
    int64_t o_joint[2];
    int64_t o_hp, o_wp, o_targets, o_starts, o_rowk, o_rowc, o_stats, o_rshares, o_lshares, o_scal, o_z, o_g, o_colsum, o_dbsum, o_slots, o_sums, o_most, total;
};

ClassPlan plan_class(const gad_class_loss_args& a, bool policy = false) {
    ClassPlan p{};
    const int64_t N = a.rows;
    const int D = a.cols, V = a.classes;
    p.parts = a.dtype == GAD_F32 ? 3 : 1;
    p.pairs = a.dtype == GAD_F32 ? 6 : 1;
    p.grads = a.dH || a.dW || a.db;
    const bool wide = ((uintptr_t)a.W & 15) == 0 && (a.ldw * (a.dtype == GAD_F32 ? 4 : 2)) % 16 == 0;
    p.few = N <= kFewRows && few_smem(a) <= kFewSmem;
    p.score = policy && !p.grads && N >= kScoreLeast && N <= kScoreRows && a.dtype != GAD_F32 && wide;
    if (p.score) p.few = false;
    p.some = !p.few && !p.score && N <= kSomeRows && a.dtype != GAD_F32 && wide && some_smem(a) <= kSomeSmem;
    p.few |= p.some || p.score;
    p.pack_w = (!p.few || a.dH) && (a.dtype == GAD_F32 || ((uintptr_t)a.W & 15) != 0 || (a.ldw * 2) % 16 != 0);
    p.ntargets = a.k + (a.labels ? 1 : 0);
    p.nl = a.k > 0 && a.labels && a.hard_weight > 0.f && a.hard_weight < 1.f && a.temperature != 1.f ? 2 : 1;
    // a code's step is T (1 / T) times as large in the sharper of two softmaxes: twice it is still below what G is rounded by in fp16, eight times in bfloat16
    const float most_t = a.dtype == GAD_F16 ? 2.f : 8.f;
    p.save = !p.grads ? kSaveNone : a.dtype == GAD_F32 || p.few || (p.nl == 2 && (a.temperature > most_t || a.temperature * most_t < 1.f)) ? kSaveFloat : kSaveCode;
    p.code_steps = p.nl == 2 ? kCodeSteps / std::max(1.f, a.temperature) : kCodeSteps;
    p.ldp = round_up(D, 8);
    p.sums = policy && p.parts == 1 && (D + CT_K - 1) / CT_K > kChunkPolicy;
    p.add_up = !p.sums && (D + CT_K - 1) / CT_K > (p.parts > 1 ? kChunkParts : kChunk);
    p.width_v = p.add_up ? 128 : width_for(V);
    p.tiles_v = (V + p.width_v - 1) / p.width_v;
    p.width_d = width_for(D);
    p.tiles_d = (D + p.width_d - 1) / p.width_d;
    p.ldg = (int64_t)p.tiles_v * p.width_v;
    const int64_t per_logit = !p.grads ? 1 : p.save == kSaveCode ? 2 : 4 + 2 * p.parts;
    const int64_t most = std::min<int64_t>(1 << 20, std::max<int64_t>(CT_M, kBlockBytes / (per_logit * p.ldg) / CT_M * CT_M));
    p.nblocks = (int)((N + most - 1) / most);
    p.block = std::min(N, round_up((N + p.nblocks - 1) / p.nblocks, CT_M));
    p.nblocks = (int)((N + p.block - 1) / p.block);
    int64_t at = 0;
    const auto room = [&](int64_t bytes) { const int64_t o = at; at += round_up(bytes, 256); return o; };
    p.o_scal = room(256);
    p.o_hp = room(2 * p.parts * N * p.ldp);
    p.o_wp = p.pack_w ? room(2 * p.parts * (int64_t)V * p.ldp) : 0;
    p.o_targets = room(8 * N * p.ntargets);
    p.starts_at_once = 4 * N * p.tiles_v <= kStartsBytes;
    p.o_starts = p.ntargets > 1 && !p.few ? room(4 * (p.starts_at_once ? N : p.block) * p.tiles_v) : 0;
    p.o_rowk = room(16 * N);
    p.o_rshares = room((int64_t)sizeof(RowShare) * N);
    p.o_lshares = room((int64_t)sizeof(double) * ((N + kFinishRows - 1) / kFinishRows));
    p.o_stats = room(16 * p.block * (p.few ? kFewBlocks : 2 * p.tiles_v));
    if (p.grads) {
        p.o_rowc = room(16 * p.block);
        p.o_z = room((p.save == kSaveCode ? 2 : 4) * p.block * p.ldg);
        p.o_g = p.save == kSaveCode ? p.o_z : room(2 * p.parts * p.block * p.ldg);
        if (a.db) { p.o_colsum = room(4 * ((p.block + 31) / 32) * p.ldg); p.o_dbsum = room(4 * (int64_t)V); }
        p.joint = policy && p.parts == 3 && p.nblocks == 1 && (a.dH || a.dW);
        if (p.joint) {
            int n = 0;
            if (a.dH) p.shape[n++] = {N, D, V, 1, 1};
            if (a.dW) p.shape[n++] = {V, D, N, 1, 1};
            cut_group(p.shape, n, p.pairs, p.cut);
            for (int i = 0; i < n; ++i) p.o_joint[i] = room(slot_bytes(p.cut[i]));
        } else if (a.dH || a.dW) p.o_slots = room((int64_t)kPairs * CT_M * p.width_d * 4);
        if (a.dW && p.nblocks > 1) p.o_sums = room(4 * (int64_t)V * D);
    }
    if (policy) p.o_most = room(4 * ((p.block + kFinishRows - 1) / kFinishRows));
    p.total = at;
    return p;
}

template <int USE, bool A_MN, bool B_MN, class T, int NL, bool ADD_UP>
cudaError_t gemm_launch(const CUtensorMap& A, const CUtensorMap& B, const TileArgs& a, cudaStream_t s) {
    const auto kernel = class_gemm_kernel<USE, A_MN, B_MN, T, NL, ADD_UP>;
    cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), CT_SMEM, false);
    if (e != cudaSuccess) return e;
    static std::atomic<int> known{0};
    if (known.load() <= 0) known.store(max_active_pairs(reinterpret_cast<const void*>(kernel), CT_THREADS, CT_SMEM, 2 * kPairs));
    const int64_t units = a.whole + ((int64_t)a.tiles_m * a.tiles_n - a.whole) * a.shares;
    const int ncl = (int)std::min<int64_t>(units, known.load());
    return chain(kernel, dim3((unsigned)(2 * ncl)), CT_THREADS, CT_SMEM, s, false, A, B, a);
}
// The statistics of a block of rows.
template <int NL>
cudaError_t go_stats(const CUtensorMap& A, const CUtensorMap& B, const TileArgs& a, bool add_up, cudaStream_t s) {
    return add_up ? gemm_launch<kStats, false, false, float, NL, true>(A, B, a, s) : gemm_launch<kStats, false, false, float, NL, false>(A, B, a, s);
}
template <class T, int NL, bool WIDE>
cudaError_t few_launch(const FewArgs& f, size_t smem, int blocks, cudaStream_t s) {
    const int n = few_rows(f.rows);
    const auto kernel = n == 1 ? class_few_kernel<T, 1, NL, WIDE> : n == 2 ? class_few_kernel<T, 2, NL, WIDE> : class_few_kernel<T, 4, NL, WIDE>;
    const cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), kFewSmem, false);
    return e != cudaSuccess ? e : chain(kernel, dim3((unsigned)blocks), 256, smem, s, false, f);
}
template <class T, int NL>
cudaError_t some_launch(const FewArgs& f, size_t smem, int blocks, cudaStream_t s) {
    const auto kernel = f.rows <= 8 ? class_some_kernel<T, 1, NL> : class_some_kernel<T, 2, NL>;
    const cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), kSomeSmem, false);
    return e != cudaSuccess ? e : chain(kernel, dim3((unsigned)blocks), 32 * kSomeWarps, smem, s, false, f);
}
// Blocks of 64 terms of a gradient's sum that the tensor core adds up before the sum moves to registers: it cuts off at most 2^-23 of the sum every 16 terms.  In 16-bit types
// all of a chunk costs at most an eighth of what the result is rounded by (2^-11 in fp16, 2^-8 in bfloat16): uncut sums of one sign over 2^19 classes
// were off by 3.6 times the rounding of fp16, now 0.1; 4096 x 1024 fp16 against 32 768 classes 848 us instead of 838.  fp32 gradients are off by 3.2e-7 to 3.6e-7 with chunks of 256 terms,
// by 6.6e-7 with 512 (8192 x 256 against 4096 classes 374 us instead of 371, 2048 x 512 against 16 384 645 instead of 628).
template <class T> constexpr int kChunkOut = 4;
template <> constexpr int kChunkOut<__half> = 128;
template <> constexpr int kChunkOut<__nv_bfloat16> = 1024;
// A gradient.  Tiles that are left over when all pairs have had the same number are cut along their reduction, so that they keep every pair busy too
// (4096 x 1024 over 47 classes: 4 tiles, 18 shares each), down to 8 ring stages a share.  Sums for an fp32 result, and longer ones than a chunk for the others, are added up in chunks.
template <bool A_MN, class T>
cudaError_t go_out(const CUtensorMap& A, const CUtensorMap& B, TileArgs a, cudaStream_t s) {
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n, rest = tiles % kPairs;
    a.whole = (int)tiles; a.shares = 1; a.kb_share = a.nkb; a.chunk = kChunkOut<T>;
    if (rest) {
        const int want = (int)std::min<int64_t>(kPairs / rest, (int64_t)a.nkb * a.pairs / 8);
        if (want > 1) {
            a.kb_share = (a.nkb + want - 1) / want;
            a.shares = (a.nkb + a.kb_share - 1) / a.kb_share;
            a.whole = (int)(tiles - rest);
        }
    }
    const bool add_up = sizeof(T) == 4 || (a.whole > 0 ? a.nkb : a.kb_share) > a.chunk;
    cudaError_t e = add_up ? gemm_launch<kOut, A_MN, true, T, 1, true>(A, B, a, s) : gemm_launch<kOut, A_MN, true, T, 1, sizeof(T) == 4>(A, B, a, s);
    if (e == cudaSuccess && a.shares > 1) e = chain(class_join_kernel<T>, dim3((unsigned)(rest * (CT_M * a.width / 1024))), 256, 0, s, false, a);
    return e;
}

template <class T>
cudaError_t run_class_steps(const gad_class_loss_args& a, const gad_policy_loss_args* policy, uint8_t* ws, cudaStream_t s) {
#define GAD_TRY(x) do { const cudaError_t e_ = (x); if (e_ != cudaSuccess) return e_; } while (0)
    const ClassPlan p = plan_class(a, policy != nullptr);
    const int64_t N = a.rows;
    const int D = a.cols, V = a.classes;
    float* scal = reinterpret_cast<float*>(ws + p.o_scal);
    float4* rowk = reinterpret_cast<float4*>(ws + p.o_rowk);
    float4* rowc = p.grads ? reinterpret_cast<float4*>(ws + p.o_rowc) : nullptr;
    float4* stats = reinterpret_cast<float4*>(ws + p.o_stats);
    int2* targets = reinterpret_cast<int2*>(ws + p.o_targets);
    uint8_t* Hp = ws + p.o_hp;
    const float T0 = a.k > 0 ? a.temperature : 1.f;

    RowArgs ra{};
    ra.H = a.H; ra.ldh = a.ldh; ra.cols = D; ra.classes = V; ra.labels = a.labels; ra.label_bytes = a.label_bytes;
    ra.tclasses = a.target_classes; ra.tclass_bytes = a.target_bytes; ra.teacher = a.teacher; ra.teacher_type = a.teacher_dtype; ra.k = a.k;
    ra.weights = a.row_weights; ra.hard = a.k > 0 ? (a.labels ? a.hard_weight : 0.f) : 1.f; ra.temperature = T0;
    ra.Hp = Hp; ra.ldp = p.ldp; ra.part_stride = N * p.ldp; ra.targets = targets; ra.ntargets = p.ntargets; ra.rowk = rowk;
    uint16_t* starts = p.o_starts ? reinterpret_cast<uint16_t*>(ws + p.o_starts) : nullptr;
    ra.starts = p.starts_at_once ? starts : nullptr; ra.nstarts = 2 * p.tiles_v; ra.start_w = p.width_v / 2;
    ra.rows = N; ra.shares = reinterpret_cast<RowShare*>(ws + p.o_rshares); ra.ticket = reinterpret_cast<unsigned*>(scal + 8); ra.status = a.status;
    const int nrshares = (int)(a.k > 0 ? N : (N + 7) / 8);
    GAD_TRY(a.k > 0 ? chain(class_rows_kernel<T>, dim3((unsigned)N), kRowThreads, 12 * (size_t)p.ntargets, s, true, ra)
                    : chain(class_label_rows_kernel<T>, dim3((unsigned)nrshares), 256, 0, s, true, ra));
    const void* Wo = a.W;
    int64_t ldw = a.ldw;
    if (p.pack_w) {
        GAD_TRY(chain(class_pack_kernel<T>, dim3((unsigned)((V + 7) / 8)), 256, 0, s, false, (const T*)a.W, a.ldw, V, D, (void*)(ws + p.o_wp), p.ldp, (int64_t)V * p.ldp));
        Wo = ws + p.o_wp;
        ldw = p.ldp;
    }
    CUtensorMap mapH, mapW, mapH_mn, mapW_mn, mapG, mapG_mn;
    const auto make = [&](CUtensorMap& m, const void* base, int64_t inner, int64_t rows, int64_t ld, int64_t part_rows, uint32_t box) {
        return tc_make_map(&m, base, (uint64_t)inner, (uint64_t)rows, (uint64_t)p.parts, (uint64_t)ld * 2, (uint64_t)(ld * 2 * part_rows), box, false, true) ? cudaSuccess : cudaErrorInvalidValue;
    };
    // operands that are read along their columns, `box` of them a CTA and stage: whole boxes where rows have whole chunks of 64 columns
    const auto make_mn = [&](CUtensorMap& m, const void* base, int64_t inner, int64_t rows, int64_t ld, int box, int& chunks) {
        chunks = inner % 64 == 0;
        if (!chunks) return make(m, base, inner, rows, ld, rows, CT_K);
        return tc_make_chunk_map(&m, base, (uint64_t)inner / 64, (uint64_t)rows, (uint64_t)p.parts, (uint64_t)ld * 2, (uint64_t)(ld * 2 * rows), (uint32_t)box / 64) ? cudaSuccess : cudaErrorInvalidValue;
    };
    int h_chunks = 0, w_chunks = 0;
    if (!p.few) {
        GAD_TRY(make(mapH, Hp, D, N, p.ldp, N, CT_H));
        GAD_TRY(make(mapW, Wo, D, V, ldw, V, (uint32_t)p.width_v / 2));
    }
    if (a.dW) GAD_TRY(make_mn(mapH_mn, Hp, D, N, p.ldp, p.width_d / 2, h_chunks));
    if (a.dH) GAD_TRY(make_mn(mapW_mn, Wo, D, V, ldw, p.width_d / 2, w_chunks));
    for (int b = 0; b < p.nblocks; ++b) {
        const int64_t r0 = b * p.block;
        const int nr = (int)std::min(p.block, N - r0), blocks = (nr + kFinishRows - 1) / kFinishRows;
        TileArgs t{};
        t.err = a.status; t.bf16 = a.dtype != GAD_F16; t.pairs = p.pairs; t.chunk = p.parts > 1 ? kChunkParts : p.sums ? kChunkPolicy : kChunk; t.scal = scal;
        t.M = nr; t.tiles_m = (nr + CT_M - 1) / CT_M;
        TileArgs z = t;
        z.N = V; z.tiles_n = p.tiles_v; z.width = p.width_v; z.nkb = (D + CT_K - 1) / CT_K; z.whole = z.tiles_m * z.tiles_n; z.shares = 1; z.kb_share = z.nkb;
        z.group = 32; z.a_row0 = (int)r0;
        z.bias = a.bias; z.bias_type = a.dtype;
        z.sc = kLog2e * (p.nl == 1 && a.k > 0 && ra.hard < 1.f ? 1.f / T0 : 1.f);
        z.inv_t = 1.f / T0;
        z.targets = targets + r0 * p.ntargets; z.ntargets = p.ntargets; z.starts = ra.starts ? ra.starts + r0 * ra.nstarts : starts; z.stats = stats;
        z.save = p.save; z.code_steps = p.code_steps; z.code_lowest = -(float)kCodeZero / p.code_steps; z.C = ws + p.o_z; z.ldc = p.ldg;
        int nparts = 2 * p.tiles_v;
        if (p.score) {
            ScoreArgs k{};
            k.rows = nr; k.width = (int)round_up(nr, 16); k.classes = V; k.nkb = z.nkb; k.bf16 = z.bf16; k.err = a.status;
            k.tiles = (V + SK_M - 1) / SK_M;
            k.stages = std::min<int>(SK_MOST_STAGES, SK_RING / (SK_A + k.width * (CT_K * 2)));
            k.bias = a.bias; k.bias_type = a.dtype; k.sc = z.sc; k.targets = targets; k.stats = stats;
            nparts = std::min(2 * kPairs, k.tiles);
            GAD_TRY(make(mapW, Wo, D, V, ldw, V, SK_M));
            GAD_TRY(make(mapH, Hp, D, N, p.ldp, N, (uint32_t)k.width));
            GAD_TRY(configure_kernel_once(reinterpret_cast<const void*>(class_score_kernel), SK_SMEM, false));
            GAD_TRY(chain(class_score_kernel, dim3((unsigned)nparts), SK_THREADS, SK_SMEM, s, false, mapW, mapH, k));
        } else if (p.few) {
            FewArgs w{};
            w.H = a.H; w.ldh = a.ldh; w.W = a.W; w.ldw = a.ldw; w.rows = nr; w.cols = D; w.classes = V; w.bias = a.bias; w.targets = targets; w.ntargets = p.ntargets; w.rowk = rowk;
            w.sc = z.sc; w.inv_t = z.inv_t; w.z = p.grads ? reinterpret_cast<float*>(z.C) : nullptr; w.ldz = p.ldg; w.stats = stats;
            nparts = (int)std::min<int64_t>(kFewBlocks, (p.ldg + 31) / 32);
            if (p.some) {
                const size_t smem = some_smem(a);
                nparts = (int)std::min<int64_t>(2 * kPairs, (p.ldg + 127) / 128);
                if constexpr (sizeof(T) == 2) GAD_TRY(p.nl == 2 ? (some_launch<T, 2>(w, smem, nparts, s)) : (some_launch<T, 1>(w, smem, nparts, s)));
            } else {
                const bool wide = ((uintptr_t)a.W & 15) == 0 && (a.ldw * (int64_t)sizeof(T)) % 16 == 0;
                GAD_TRY(p.nl == 2 ? (wide ? few_launch<T, 2, true>(w, few_smem(a), nparts, s) : few_launch<T, 2, false>(w, few_smem(a), nparts, s))
                              : (wide ? few_launch<T, 1, true>(w, few_smem(a), nparts, s) : few_launch<T, 1, false>(w, few_smem(a), nparts, s)));
            }
        } else {
            if (starts && !p.starts_at_once) GAD_TRY(chain(class_starts_kernel, dim3((unsigned)nr), 128, 0, s, false, z.targets, p.ntargets, starts, ra.nstarts, ra.start_w));
            if (p.sums) GAD_TRY((gemm_launch<kStatsSums, false, false, float, 1, true>(mapH, mapW, z, s)));
            else GAD_TRY(p.nl == 2 ? go_stats<2>(mapH, mapW, z, p.add_up, s) : go_stats<1>(mapH, mapW, z, p.add_up, s));
        }
        FinishArgs f{};
        f.stats = stats; f.parts = nparts; f.rows = nr; f.rowk = rowk + r0; f.sc = z.sc; f.inv_t = z.inv_t; f.temperature = T0; f.rowc = rowc; f.row_loss = a.row_loss + r0;
        f.shares = reinterpret_cast<double*>(ws + p.o_lshares); f.share0 = (int)(r0 / kFinishRows); f.nshares = (int)((N + kFinishRows - 1) / kFinishRows);
        f.row_shares = ra.shares; f.nrow_shares = nrshares; f.ticket = ra.ticket; f.scale = a.scale; f.mean = a.mean; f.first = b == 0; f.final = b == p.nblocks - 1;
        f.scal = scal; f.loss = a.loss;
        if (policy)
            f.policy = {policy->old_logp + r0, policy->advantages + r0, policy->ref_logp && policy->kl_weight != 0.f ? policy->ref_logp + r0 : nullptr, 1.f - policy->clip_low, 1.f + policy->clip_high,
                        policy->kl_weight, policy->logp + r0, reinterpret_cast<float*>(ws + p.o_most)};
        GAD_TRY(chain(p.nl == 2 ? class_finish_kernel<2> : class_finish_kernel<1>, dim3((unsigned)blocks), 256, 0, s, false, f));
        if (!p.grads) continue;
        GradArgs g{};
        g.z = z.C; g.ldz = p.ldg; g.G = ws + p.o_g; g.ldg = p.ldg; g.part_stride = nr * p.ldg; g.stats = stats; g.half_w = p.width_v / 2;
        g.rowc = rowc; g.rowk = rowk + r0; g.targets = z.targets; g.ntargets = p.ntargets; g.scal = scal; g.inv_t = z.inv_t; g.code_unit = 1.f / p.code_steps;
        g.colsum = a.db ? reinterpret_cast<float*>(ws + p.o_colsum) : nullptr; g.rows = nr; g.classes = V;
        auto grad = a.db ? (p.nl == 2 ? class_grad_kernel<T, float, 2, true> : class_grad_kernel<T, float, 1, true>)
                         : (p.nl == 2 ? class_grad_kernel<T, float, 2, false> : class_grad_kernel<T, float, 1, false>);
        if constexpr (sizeof(T) == 2)
            if (p.save == kSaveCode)
                grad = a.db ? (p.nl == 2 ? class_grad_kernel<T, uint16_t, 2, true> : class_grad_kernel<T, uint16_t, 1, true>)
                            : (p.nl == 2 ? class_grad_kernel<T, uint16_t, 2, false> : class_grad_kernel<T, uint16_t, 1, false>);
        const int slices = (nr + 31) / 32;
        GAD_TRY(chain(grad, dim3((unsigned)((p.ldg + 1023) / 1024), (unsigned)slices), 256, 0, s, false, g));
        const int add = p.nblocks == 1 ? kAddNone : b == 0 ? kAddFirst : b < p.nblocks - 1 ? kAddMore : kAddLast;
        if (a.db)
            GAD_TRY(chain(class_bias_kernel<T>, dim3((unsigned)((V + 31) / 32)), 256, 0, s, false, (const float*)g.colsum, p.ldg, slices, V, (const float*)scal, add,
                          reinterpret_cast<float*>(ws + p.o_dbsum), reinterpret_cast<T*>(a.db)));
        if (p.joint) {
            if constexpr (sizeof(T) == 4) {
                GatedGroup<kGroup> r{};
                Sequence q{s, false, false};
                const auto add = [&](bool of_w, void* C, int64_t ldc) {
                    const int i = r.n++;
                    r.p[i] = product(p.shape[i], p.cut[i], a.dtype, of_w, 8, a.status);
                    r.p[i].t.slots = reinterpret_cast<float*>(ws + p.o_joint[i]);
                    r.p[i].C[0] = C; r.p[i].ldc[0] = ldc; r.p[i].factor = scal + 1;
                    const int box = p.cut[i].width / 2;
                    if (!of_w) {
                        const cudaError_t e = make(r.A[i], g.G, V, nr, p.ldg, nr, CT_H);
                        return e != cudaSuccess ? e : make_mn(r.B0[i], Wo, D, V, ldw, box, r.p[i].b_chunks);
                    }
                    const cudaError_t e = make_mn(r.A[i], g.G, p.ldg, nr, p.ldg, CT_H, r.p[i].a_chunks);
                    return e != cudaSuccess ? e : make_mn(r.B0[i], Hp, D, N, p.ldp, box, r.p[i].b_chunks);
                };
                if (a.dH) GAD_TRY(add(false, a.dH, a.lddh));
                if (a.dW) GAD_TRY(add(true, a.dW, a.lddw));
                GAD_TRY((go<kPlain, kAnyMN, T>(r, q)));
            }
            continue;
        }
        t.slots = reinterpret_cast<float*>(ws + p.o_slots);
        t.N = D; t.tiles_n = p.tiles_d; t.width = p.width_d; t.group = 8;
        if (a.dH) {
            TileArgs h = t;
            GAD_TRY(make(mapG, g.G, V, nr, p.ldg, nr, CT_H));
            h.nkb = (V + CT_K - 1) / CT_K; h.b_chunks = w_chunks;
            h.C = reinterpret_cast<T*>(a.dH) + r0 * a.lddh; h.ldc = a.lddh;
            GAD_TRY((go_out<false, T>(mapG, mapW_mn, h, s)));
        }
        if (a.dW) {
            TileArgs w = t;
            // (rows of G are whole tiles: what lies behind the classes is zero, and rows of dW that are not written)
            GAD_TRY(make_mn(mapG_mn, g.G, p.ldg, nr, p.ldg, CT_H, w.a_chunks));
            w.b_chunks = h_chunks;
            w.M = V; w.tiles_m = (V + CT_M - 1) / CT_M; w.nkb = (nr + CT_K - 1) / CT_K; w.b_row0 = (int)r0;
            w.C = a.dW; w.ldc = a.lddw; w.add = add; w.sums = reinterpret_cast<float*>(ws + p.o_sums);
            GAD_TRY((go_out<true, T>(mapG_mn, mapH_mn, w, s)));
        }
    }
    return cudaGetLastError();
#undef GAD_TRY
}
template <class T>
int run_class(const gad_class_loss_args& a, const gad_policy_loss_args* policy, uint8_t* ws, cudaStream_t s) { return run_class_steps<T>(a, policy, ws, s) == cudaSuccess ? GAD_OK : GAD_ERR_CUDA; }

// No rows: no loss, and gradients of zero.
template <class T>
int run_empty(const gad_class_loss_args& a, cudaStream_t s) {
    class_empty_kernel<<<1, 1, 0, s>>>(a.loss, a.status);
    ++g_kernel_launches;
    if (a.dW) { class_zero_kernel<T><<<592, 256, 0, s>>>((T*)a.dW, a.lddw, a.classes, a.cols); ++g_kernel_launches; }
    if (a.db) { class_zero_kernel<T><<<592, 256, 0, s>>>((T*)a.db, a.classes, 1, a.classes); ++g_kernel_launches; }
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}

int check_class(const gad_class_loss_args* a) {
    if (!a) return GAD_ERR_ARG;
    if (a->dtype < GAD_F32 || a->dtype > GAD_BF16 || a->rows < 0 || a->cols < 1 || a->classes < 1) return GAD_ERR_ARG;
    if (a->rows > (1 << 30) || a->cols > (1 << 20) || a->classes > (1 << 24)) return GAD_ERR_RANGE;
    if (a->k < 0) return GAD_ERR_ARG;
    if (a->k > kMostTargets) return GAD_ERR_RANGE;
    if (a->ldw < a->cols || (a->rows > 0 && a->ldh != 0 && a->ldh < a->cols) || (a->dH && a->lddh < a->cols) || (a->dW && a->lddw < a->cols)) return GAD_ERR_ARG;
    if (a->labels && a->label_bytes != 4 && a->label_bytes != 8) return GAD_ERR_ARG;
    if (a->k > 0) {
        if (!(a->temperature >= 1e-3f && a->temperature <= 1e3f) || !(a->hard_weight >= 0.f && a->hard_weight <= 1.f)) return GAD_ERR_ARG;
        if (a->target_bytes != 4 && a->target_bytes != 8) return GAD_ERR_ARG;
        if (a->teacher_dtype < GAD_F32 || a->teacher_dtype > GAD_BF16) return GAD_ERR_ARG;
    }
    if (!std::isfinite(a->scale) || (a->mean != 0 && a->mean != 1) || (a->db && !a->bias)) return GAD_ERR_ARG;
    return GAD_OK;
}

}  // namespace
}  // namespace gad

extern "C" int gad_class_loss_workspace_bytes(const gad_class_loss_args* args, size_t* bytes) {
    const int rc = gad::check_class(args);
    if (rc != GAD_OK) return rc;
    if (!bytes) return GAD_ERR_ARG;
    *bytes = args->rows == 0 ? 0 : (size_t)gad::plan_class(*args).total;
    return GAD_OK;
}

namespace gad {
namespace {

int run_loss(const gad_class_loss_args& a, const gad_policy_loss_args* policy, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a.W || !a.loss || !a.status) return GAD_ERR_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    if (a.rows == 0) return a.dtype == GAD_F32 ? run_empty<float>(a, s) : a.dtype == GAD_F16 ? run_empty<__half>(a, s) : run_empty<__nv_bfloat16>(a, s);
    if (!a.H || !a.row_loss || (a.k == 0 && !a.labels) || (a.k > 0 && (!a.target_classes || !a.teacher))) return GAD_ERR_ARG;
    if (policy && (!policy->old_logp || !policy->advantages || !policy->logp)) return GAD_ERR_ARG;
    if (policy && (((uintptr_t)policy->old_logp | (uintptr_t)policy->advantages | (uintptr_t)policy->ref_logp | (uintptr_t)policy->logp) & 3) != 0) return GAD_ERR_ARG;   // (off their elements)
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < (size_t)plan_class(a, policy != nullptr).total) return GAD_ERR_OOM;
    try {
        uint8_t* ws = (uint8_t*)workspace;
        return a.dtype == GAD_F32 ? run_class<float>(a, policy, ws, s) : a.dtype == GAD_F16 ? run_class<__half>(a, policy, ws, s) : run_class<__nv_bfloat16>(a, policy, ws, s);
    } catch (...) {   // (the table of configured kernels could not grow)
        return GAD_ERR_OOM;
    }
}

int check_policy(const gad_policy_loss_args* a) {
    if (!a) return GAD_ERR_ARG;
    const int rc = check_class(&a->head);
    if (rc != GAD_OK) return rc;
    if (a->head.k != 0 || (a->head.rows > 0 && !a->head.labels)) return GAD_ERR_ARG;
    if (!(a->clip_low >= 0.f && a->clip_low <= 1.f) || !(a->clip_high >= 0.f) || !(a->kl_weight >= 0.f) || !std::isfinite(a->kl_weight)) return GAD_ERR_ARG;
    return GAD_OK;
}

}  // namespace
}  // namespace gad

extern "C" int gad_class_loss(const gad_class_loss_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = gad::check_class(args);
    return rc != GAD_OK ? rc : gad::run_loss(*args, nullptr, workspace, workspace_bytes, stream);
}

extern "C" int gad_policy_loss_workspace_bytes(const gad_policy_loss_args* args, size_t* bytes) {
    const int rc = gad::check_policy(args);
    if (rc != GAD_OK) return rc;
    if (!bytes) return GAD_ERR_ARG;
    *bytes = args->head.rows == 0 ? 0 : (size_t)gad::plan_class(args->head, true).total;
    return GAD_OK;
}

extern "C" int gad_policy_loss(const gad_policy_loss_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = gad::check_policy(args);
    return rc != GAD_OK ? rc : gad::run_loss(args->head, args, workspace, workspace_bytes, stream);
}
