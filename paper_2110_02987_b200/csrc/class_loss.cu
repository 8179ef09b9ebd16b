// Loss of an output layer with many classes, without keeping its logits, and the gradients: softmax cross entropy against labels, and distillation
// from a teacher's top logits.  With z_i = W h_i + b over all classes, p = softmax(z), p^T = softmax(z / T), q_i = softmax of row i's teacher logits / T:
//   l_i = a (lse(z) - z_y) + (1 - a) T^2 sum_j q_j (log q_j - log p^T_{c_j})
// Both kinds of target are one sparse list of (class, weight): tau = a [y] + (1 - a) T q at the teacher's classes.  Then
//   l_i = a lse(z) + (1 - a) T^2 (lse(z / T) + sum q log q) - sum_v tau_v z_v,     dl_i / dz = a p + (1 - a) T p^T - tau.
//
// One call: the rows' targets are sorted by class and the rows copied to the operand type (class_rows_kernel); z = H W^T tile by tile leaves per row and tile
// half the largest value, the sums and sum tau z (kStats), class_finish_kernel joins them.  For the gradients the classes are gone through in pieces: z
// again, turned into G (kGrad), and from it dH += G W and dW = G^T H (kOut, kPartial).  The logits take 2 N V D flops twice instead of N V values kept.
//
// Operands: fp16 and bfloat16 as they are.  fp32 in three bfloat16 parts (24 bits), of whose nine products the six that reach 2^-24 are summed.
// G is rounded to the operand type (fp32: not rounded), times a power of two that brings its largest possible value to 2^14 .. 2^15: in fp16 a probability of 1e-9 keeps
// eight bits.  One rounding of each term of a sum whose result is rounded to the same type: the result's error grows by at most the square root of 2.
#include <algorithm>
#include <atomic>

#include "class_gemm.cuh"

namespace gad {

namespace {

constexpr int kRowThreads = 128;
constexpr int kMostTargets = 1024;                       // teacher logits a row
constexpr int64_t kPieceBytes = 512ll << 20;             // of G held at once
constexpr float kLog2e = 1.44269504f;

template <class P> __device__ __forceinline__ float load_as_float(const void* p, int64_t i) { return to_float(reinterpret_cast<const P*>(p)[i]); }
__device__ __forceinline__ float load_typed(const void* p, int type, int64_t i) {
    return type == GAD_F32 ? load_as_float<float>(p, i) : type == GAD_F16 ? load_as_float<__half>(p, i) : load_as_float<__nv_bfloat16>(p, i);
}
__device__ __forceinline__ int64_t load_index(const void* p, int bytes, int64_t i) {
    return bytes == 8 ? reinterpret_cast<const int64_t*>(p)[i] : (int64_t)reinterpret_cast<const int32_t*>(p)[i];
}

// A row as operands: copied (16-bit types), or in three bfloat16 parts.  dst rows are 16-byte aligned.
template <class T>
__device__ __forceinline__ void pack_row(const T* __restrict__ src, int cols, bool keep, void* dst, int64_t at, int64_t part_stride, int t, int threads) {
    if constexpr (sizeof(T) == 4) {
        __nv_bfloat16* d = reinterpret_cast<__nv_bfloat16*>(dst) + at;
        const int n4 = ((uintptr_t)src & 15) == 0 ? cols >> 2 : 0;
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
        for (int c = 4 * n4 + t; c < cols; c += threads) {
            __nv_bfloat16 p[3];
            split3(keep ? src[c] : 0.f, p);
            for (int k = 0; k < 3; ++k) d[k * part_stride + c] = p[k];
        }
    } else {
        T* d = reinterpret_cast<T*>(dst) + at;
        if (((uintptr_t)src & 15) == 0) {
            const int n8 = cols >> 3;
            for (int c = t; c < n8; c += threads)
                reinterpret_cast<uint4*>(d)[c] = keep ? reinterpret_cast<const uint4*>(src)[c] : make_uint4(0u, 0u, 0u, 0u);
            for (int c = 8 * n8 + t; c < cols; c += threads) d[c] = keep ? src[c] : from_float<T>(0.f);
        } else {
            for (int c = t; c < cols; c += threads) d[c] = keep ? src[c] : from_float<T>(0.f);
        }
    }
}

struct RowArgs {
    const void* H; int64_t ldh; int cols, classes;
    const void* labels; int label_bytes;
    const void* tclasses; int tclass_bytes; const void* teacher; int teacher_type; int k;
    const float* weights;
    float hard, temperature;
    void* Hp; int64_t ldp, part_stride;
    int2* targets; int ntargets;
    float4* rowk;
    int32_t* status;
    int64_t rows;
    unsigned* ticket;
};

// Labels alone: a warp a row.
template <class T>
__global__ void __launch_bounds__(256) class_label_rows_kernel(const RowArgs a) {
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    pdl_next();
    if (blockIdx.x == 0 && threadIdx.x == 0) { *a.status = 0; *a.ticket = 0u; }
    if (r >= a.rows) return;
    const int64_t y = load_index(a.labels, a.label_bytes, r);
    const bool counts = y >= 0, bad = y >= a.classes;
    if (lane == 0) {
        a.targets[r] = make_int2(counts && !bad ? (int)y : INT_MAX, __float_as_int(counts && !bad ? 1.f : 0.f));
        a.rowk[r] = make_float4(counts ? 1.f : 0.f, 0.f, bad ? NAN : 0.f, counts ? (a.weights ? a.weights[r] : 1.f) : 0.f);
    }
    pack_row<T>(reinterpret_cast<const T*>(a.H) + r * a.ldh, a.cols, counts, a.Hp, r * a.ldp, a.part_stride, lane, 32);
}

// A block a row.  rowk = (coefficient of lse(z), of lse(z / T), sum of q log q with its factor, weight of the row); a row without target: (0, 0, 0, 0).
template <class T>
__global__ void __launch_bounds__(kRowThreads) class_rows_kernel(const RowArgs a) {
    extern __shared__ int sm_rows[];
    int* idx = sm_rows;                                   // [ntargets]
    float* tau = reinterpret_cast<float*>(sm_rows + a.ntargets);
    __shared__ float red[2][kRowThreads / 32];
    __shared__ int bad, soft_any;
    const int64_t r = blockIdx.x;
    const int t = threadIdx.x, lane = t & 31, w = t >> 5;
    pdl_next();
    if (t == 0) { bad = 0; soft_any = 0; if (r == 0) { *a.status = 0; *a.ticket = 0u; } }
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
            tau[j] = hb * tt * q;
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
    }
    if (t == 0) a.rowk[r] = make_float4(ha, hb * tt * tt, counts && bad ? NAN : hb * tt * tt * ent, counts ? (a.weights ? a.weights[r] : 1.f) : 0.f);
    pack_row<T>(reinterpret_cast<const T*>(a.H) + r * a.ldh, a.cols, counts, a.Hp, r * a.ldp, a.part_stride, t, kRowThreads);
}

// Class vectors that no descriptor can reach (fp32, or rows that do not start on 16 bytes) as operands: a warp a row.
template <class T>
__global__ void __launch_bounds__(256) class_pack_kernel(const T* __restrict__ W, int64_t ldw, int rows, int cols, void* Wp, int64_t ldp, int64_t part_stride) {
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_next();
    pdl_wait();
    if (r < rows) pack_row<T>(W + r * ldw, cols, true, Wp, r * ldp, part_stride, threadIdx.x & 31, 32);
}

// What a block of class_finish_kernel adds to the loss: sum of weighted row losses, the largest coefficient of G, counted rows.
struct LossShare { double sum; float most; int n; };
constexpr int kFinishRows = 8;

// The parts of a row's statistics joined (a block has 8 rows, 32 threads each, every 32nd part a thread; joined pairwise in a fixed order), and in the block that
// comes last the loss and what the gradients are multiplied with.  scal[0]: a power of two that brings the largest coefficient of G to 2^14 .. 2^15;
// [1]: scale / counted rows / that.
template <int NL>
__global__ void __launch_bounds__(256) class_finish_kernel(const float4* __restrict__ stats, int parts, int rows, const float4* __restrict__ rowk, float sc, float inv_t, float hard_t,
                                                           float4* __restrict__ rowc, float* __restrict__ row_loss, LossShare* shares, unsigned* ticket, float scale, int mean,
                                                           float* __restrict__ scal, float* __restrict__ loss) {
    __shared__ float4 sm[8][kFinishRows];
    __shared__ bool last;
    __shared__ LossShare smt[8];
    const int rl = threadIdx.x % kFinishRows, lane = threadIdx.x & 31, w = threadIdx.x >> 5, r = blockIdx.x * kFinishRows + rl;
    pdl_next();
    pdl_wait();
    after_wait(stats);
    after_wait(rowk);
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
    if (r < rows)
        for (int p = threadIdx.x / kFinishRows; p < parts; p += 128) {
            float4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = p + 32 * i < parts ? stats[(int64_t)(p + 32 * i) * rows + r] : none;
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
        LossShare mine{0.0, 0.f, 0};
        if (lane < kFinishRows && r < rows) {
            at = sm[0][lane];
            for (int i = 1; i < 8; ++i) at = join(at, sm[i][lane]);
            const float4 k = rowk[r];
            // in log2: of the (first) softmax, whose logits were scaled by sc, and of the second
            const float l1 = at.x + log2f(at.y), l2 = NL == 2 ? at.x * inv_t + log2f(at.z) : l1;
            const float ln2 = 0.693147181f;
            const bool counts = k.x > 0.f || k.y > 0.f;
            const float l = counts ? k.x * (l1 * ln2) + k.y * (l2 * ln2) + k.z - at.w / sc : 0.f;
            row_loss[r] = l;
            // gradient: a p + (1 - a) T p^T; with one softmax both coefficients are its
            const float a = k.x, b = k.y / hard_t;
            if (rowc) rowc[r] = NL == 2 ? make_float4(a, b, l1, l2) : make_float4(a + b, 0.f, l1, 0.f);
            if (counts) { mine.sum = (double)k.w * (double)l; mine.most = fabsf(k.w) * (a + b); mine.n = 1; }
        }
#pragma unroll
        for (int o = 1; o < kFinishRows; o <<= 1) {
            mine.sum += __shfl_xor_sync(0xffffffffu, mine.sum, o);
            mine.most = fmaxf(mine.most, __shfl_xor_sync(0xffffffffu, mine.most, o));
            mine.n += __shfl_xor_sync(0xffffffffu, mine.n, o);
        }
        if (lane == 0) {
            shares[blockIdx.x] = mine;
            __threadfence();
            last = atomicAdd(ticket, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    LossShare all{0.0, 0.f, 0};
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) {
        const double s = __ldcg(&shares[i].sum);
        all.sum += s;
        all.most = fmaxf(all.most, __ldcg(&shares[i].most));
        all.n += __ldcg(&shares[i].n);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        all.sum += __shfl_xor_sync(0xffffffffu, all.sum, o);
        all.most = fmaxf(all.most, __shfl_xor_sync(0xffffffffu, all.most, o));
        all.n += __shfl_xor_sync(0xffffffffu, all.n, o);
    }
    if (lane == 0) smt[w] = all;
    __syncthreads();
    if (threadIdx.x) return;
    all = smt[0];
    for (int i = 1; i < 8; ++i) { all.sum += smt[i].sum; all.most = fmaxf(all.most, smt[i].most); all.n += smt[i].n; }
    const double f = mean ? (all.n ? (double)scale / all.n : 0.0) : (double)scale;
    loss[0] = (float)(f * all.sum);
    const int e = all.most > 0.f && all.most < INFINITY ? 14 - ilogbf(all.most) : 0;
    scal[0] = ldexpf(1.f, max(-100, min(100, e)));
    scal[1] = (float)(f / (double)scal[0]);
}

// result [rows x cols] = factor x the sum of the shares, in order; VEC columns a thread.
template <class T, int VEC>
__global__ void __launch_bounds__(256) join_parts_kernel(const float* __restrict__ part, int splits, int64_t part_stride, int64_t rows, int cols, const float* __restrict__ scal,
                                                         T* __restrict__ out, int64_t ld) {
    pdl_next();
    pdl_wait();
    after_wait(part);
    after_wait(scal);
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC;
    if (i >= rows * cols) return;
    const int64_t r = i / cols;
    const int c = (int)(i - r * cols);
    float s[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) s[j] = 0.f;
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
        const float* p = part + k * part_stride + i;
        if constexpr (VEC == 4) {
            const float4 v = *reinterpret_cast<const float4*>(p);
            s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
        } else s[0] += *p;
    }
    const float f = scal[1];
    union { T e[VEC]; uint4 u4; uint2 u2; } w;
#pragma unroll
    for (int j = 0; j < VEC; ++j) w.e[j] = from_float<T>(f * s[j]);
    T* o = out + r * ld + c;
    if constexpr (VEC == 4 && sizeof(T) == 4) *reinterpret_cast<uint4*>(o) = w.u4;
    else if constexpr (VEC == 4) *reinterpret_cast<uint2*>(o) = w.u2;
    else *o = w.e[0];
}

// db of a piece from the column sums of 32 rows each that the drain of G leaves: 32 classes a block, each of its eight warps a run of them, in order.
template <class T>
__global__ void __launch_bounds__(256) class_bias_kernel(const float* __restrict__ colsum, int64_t ld, int n, int classes, const float* __restrict__ scal, T* __restrict__ db) {
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
    db[c] = from_float<T>(s * scal[1]);
}

template <class T>
__global__ void __launch_bounds__(256) class_zero_kernel(T* __restrict__ p, int64_t ld, int64_t rows, int cols) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_float<T>(0.f);
}
__global__ void class_empty_kernel(float* loss, int32_t* status) { *loss = 0.f; *status = 0; }

// ---------------------------------------------------------------------------------------------
// How a call is cut up; the same for the workspace and the launches.
// ---------------------------------------------------------------------------------------------
struct Cut { int splits, kb; };
// Shares of the reduction: where there are fewer tiles than pairs of CTAs, as many as bring them near, of 8 blocks (512 values) and more.
Cut cut_reduction(int64_t tiles, int nkb) {
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(74 / tiles, nkb / 8));
    const int kb = (int)((nkb + want - 1) / want);
    return {(nkb + kb - 1) / kb, kb};
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
template <class T>
cudaError_t join_parts(const float* part, int splits, int64_t part_stride, int64_t rows, int cols, const float* scal, T* out, int64_t ld, cudaStream_t s) {
    const bool wide = cols % 4 == 0 && ld % 4 == 0 && ((uintptr_t)out & (4 * sizeof(T) - 1)) == 0;
    const int64_t n = rows * cols, per = wide ? 1024 : 256;
    return chain(wide ? join_parts_kernel<T, 4> : join_parts_kernel<T, 1>, dim3((unsigned)((n + per - 1) / per)), 256, 0, s, false, part, splits, part_stride, rows, cols, scal, out, ld);
}

int width_for(int n) { return n <= 128 ? 128 : 256; }

struct ClassPlan {
    int parts, pairs, es;            // operand parts, products of them, bytes of a caller's value
    bool grads, pack_w;
    int ntargets, nl;
    int width_v, tiles_v, tiles_m, width_d, tiles_d;
    int64_t ldp, ldg, piece;         // row lengths of the packed operands and of G, classes a piece
    int npieces;
    Cut cut_h, cut_w;
    bool h_parts, w_parts;
    int64_t o_hp, o_wp, o_targets, o_rowk, o_rowc, o_stats, o_shares, o_scal, o_g, o_colsum, o_dh, o_dw, total;
};

ClassPlan plan_class(const gad_class_loss_args& a) {
    ClassPlan p{};
    const int64_t N = a.rows;
    const int D = a.cols, V = a.classes;
    p.parts = a.dtype == GAD_F32 ? 3 : 1;
    p.pairs = a.dtype == GAD_F32 ? 6 : 1;
    p.es = a.dtype == GAD_F32 ? 4 : 2;
    p.grads = a.dH || a.dW || a.db;
    p.pack_w = a.dtype == GAD_F32 || ((uintptr_t)a.W & 15) != 0 || (a.ldw * 2) % 16 != 0;
    p.ntargets = a.k + (a.labels ? 1 : 0);
    p.nl = a.k > 0 && a.labels && a.hard_weight > 0.f && a.hard_weight < 1.f && a.temperature != 1.f ? 2 : 1;
    p.ldp = round_up(D, 8);
    p.tiles_m = (int)((N + CT_M - 1) / CT_M);
    p.width_v = width_for(V);
    p.tiles_v = (V + p.width_v - 1) / p.width_v;
    p.width_d = width_for(D);
    p.tiles_d = (D + p.width_d - 1) / p.width_d;
    int64_t most = std::max<int64_t>(1, kPieceBytes / (2 * p.parts * N * p.width_v)) * p.width_v;
    p.npieces = (int)((V + most - 1) / most);
    p.piece = round_up((V + p.npieces - 1) / p.npieces, p.width_v);
    p.npieces = (int)((V + p.piece - 1) / p.piece);
    p.ldg = p.piece;
    p.cut_h = cut_reduction((int64_t)p.tiles_m * p.tiles_d, (int)((std::min<int64_t>(p.piece, V) + CT_K - 1) / CT_K));
    p.cut_w = cut_reduction((int64_t)((p.piece + CT_M - 1) / CT_M) * p.tiles_d, (int)((N + CT_K - 1) / CT_K));
    p.h_parts = p.cut_h.splits > 1 || p.npieces > 1;
    p.w_parts = p.cut_w.splits > 1;
    int64_t at = 0;
    const auto room = [&](int64_t bytes) { const int64_t o = at; at += round_up(bytes, 256); return o; };
    p.o_scal = room(256);
    p.o_hp = room(2 * p.parts * N * p.ldp);
    p.o_wp = p.pack_w ? room(2 * p.parts * (int64_t)V * p.ldp) : 0;
    p.o_targets = room(8 * N * std::max(1, p.ntargets));
    p.o_rowk = room(16 * N);
    p.o_rowc = room(16 * N);
    p.o_stats = room(16 * N * 2 * p.tiles_v);
    p.o_shares = room((int64_t)sizeof(LossShare) * ((N + kFinishRows - 1) / kFinishRows));
    if (p.grads) {
        p.o_g = room(2 * p.parts * N * p.ldg);
        if (a.db) p.o_colsum = room(4 * 8 * (int64_t)p.tiles_m * p.ldg);
        if (a.dH && p.h_parts) p.o_dh = room(4 * p.cut_h.splits * N * D);
        if (a.dW && p.w_parts) p.o_dw = room(4 * p.cut_w.splits * std::min<int64_t>(p.piece, V) * D);
    }
    p.total = at;
    return p;
}

// Ring stages (64 terms each) of a chunk: 64 additions to an accumulator, about 3e-7 of its value.
constexpr int kChunk = 16;

template <int USE, bool A_MN, bool B_MN, class T, int NL, bool ADD_UP>
cudaError_t gemm_launch(const CUtensorMap& A, const CUtensorMap& B, const TileArgs& a, cudaStream_t s) {
    const auto kernel = class_gemm_kernel<USE, A_MN, B_MN, T, NL, ADD_UP>;
    cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), CT_SMEM, false);
    if (e != cudaSuccess) return e;
    static std::atomic<int> known{0};
    if (known.load() <= 0) known.store(max_active_pairs(reinterpret_cast<const void*>(kernel), CT_THREADS, CT_SMEM, 148));
    const int64_t units = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    const int ncl = (int)std::min<int64_t>(units, known.load());
    return chain(kernel, dim3((unsigned)(2 * ncl)), CT_THREADS, CT_SMEM, s, false, A, B, a);
}
// What is wanted to fp32 accuracy and longer than a chunk is added up in chunks: everything of fp32 operands, and the logits of the loss.
template <int USE, bool A_MN, bool B_MN, class T, int NL>
cudaError_t gemm_go(const CUtensorMap& A, const CUtensorMap& B, TileArgs a, cudaStream_t s) {
    a.chunk = kChunk;
    const bool exact = (a.pairs > 1 || USE == kStats) && a.kb_split * a.pairs > kChunk;
    if constexpr (USE == kStats || USE == kPartial || sizeof(T) == 4)
        if (exact) return gemm_launch<USE, A_MN, B_MN, T, NL, true>(A, B, a, s);
    if constexpr (!(USE == kGrad && sizeof(T) == 4)) return gemm_launch<USE, A_MN, B_MN, T, NL, false>(A, B, a, s);
    else return gemm_launch<USE, A_MN, B_MN, T, NL, true>(A, B, a, s);   // (of one chunk)
}

template <class T>
int run_class(const gad_class_loss_args& a, uint8_t* ws, cudaStream_t s) {
    const ClassPlan p = plan_class(a);
    const int N = (int)a.rows, D = a.cols, V = a.classes;
    float* scal = reinterpret_cast<float*>(ws + p.o_scal);
    float4* rowk = reinterpret_cast<float4*>(ws + p.o_rowk);
    float4* rowc = p.grads ? reinterpret_cast<float4*>(ws + p.o_rowc) : nullptr;
    float4* stats = reinterpret_cast<float4*>(ws + p.o_stats);
    int2* targets = reinterpret_cast<int2*>(ws + p.o_targets);
    uint8_t* Hp = ws + p.o_hp;
    uint8_t* G = ws + p.o_g;
    const float T0 = a.k > 0 ? a.temperature : 1.f;

    RowArgs ra{};
    ra.H = a.H; ra.ldh = a.ldh; ra.cols = D; ra.classes = V; ra.labels = a.labels; ra.label_bytes = a.label_bytes;
    ra.tclasses = a.target_classes; ra.tclass_bytes = a.target_bytes; ra.teacher = a.teacher; ra.teacher_type = a.teacher_dtype; ra.k = a.k;
    ra.weights = a.row_weights; ra.hard = a.k > 0 ? (a.labels ? a.hard_weight : 0.f) : 1.f; ra.temperature = T0;
    ra.Hp = Hp; ra.ldp = p.ldp; ra.part_stride = (int64_t)N * p.ldp; ra.targets = targets; ra.ntargets = p.ntargets; ra.rowk = rowk; ra.status = a.status;
    ra.rows = N; ra.ticket = reinterpret_cast<unsigned*>(scal + 2);
    cudaError_t e = a.k > 0 ? chain(class_rows_kernel<T>, dim3((unsigned)N), kRowThreads, 8 * (size_t)p.ntargets, s, true, ra)
                            : chain(class_label_rows_kernel<T>, dim3((unsigned)((N + 7) / 8)), 256, 0, s, true, ra);
    if (e != cudaSuccess) return GAD_ERR_CUDA;
    const void* Wo = a.W;
    int64_t ldw = a.ldw;
    if (p.pack_w) {
        if (chain(class_pack_kernel<T>, dim3((unsigned)((V + 7) / 8)), 256, 0, s, false, (const T*)a.W, a.ldw, V, D, (void*)(ws + p.o_wp), p.ldp, (int64_t)V * p.ldp) != cudaSuccess)
            return GAD_ERR_CUDA;
        Wo = ws + p.o_wp;
        ldw = p.ldp;
    }

    CUtensorMap mapH, mapW, mapH_mn, mapW_mn, mapG, mapG_mn;
    const auto make = [&](CUtensorMap& m, const void* base, int64_t inner, int64_t rows, int64_t ld, uint32_t box) {
        return tc_make_map(&m, base, (uint64_t)inner, (uint64_t)rows, (uint64_t)p.parts, (uint64_t)ld * 2, (uint64_t)(ld * 2 * rows), box, false, true);
    };
    if (!make(mapH, Hp, D, N, p.ldp, CT_H) || !make(mapW, Wo, D, V, ldw, (uint32_t)p.width_v / 2)) return GAD_ERR_CUDA;

    TileArgs t{};
    t.err = a.status; t.bf16 = a.dtype != GAD_F16; t.pairs = p.pairs;
    t.M = N; t.N = V; t.tiles_m = p.tiles_m; t.tiles_n = p.tiles_v; t.width = p.width_v;
    t.nkb = (D + CT_K - 1) / CT_K; t.splits = 1; t.kb_split = t.nkb; t.group = 32;
    t.bias = a.bias; t.bias_type = a.dtype; t.classes = V;
    t.sc = kLog2e * (p.nl == 1 && a.k > 0 && ra.hard < 1.f ? 1.f / T0 : 1.f);
    t.inv_t = 1.f / T0;
    t.targets = targets; t.ntargets = p.ntargets; t.stats = stats; t.rowk = rowk; t.rowc = rowc; t.scal = scal;
    e = p.nl == 2 ? gemm_go<kStats, false, false, float, 2>(mapH, mapW, t, s) : gemm_go<kStats, false, false, float, 1>(mapH, mapW, t, s);
    if (e != cudaSuccess) return GAD_ERR_CUDA;
    e = chain(p.nl == 2 ? class_finish_kernel<2> : class_finish_kernel<1>, dim3((unsigned)((N + kFinishRows - 1) / kFinishRows)), 256, 0, s, false, (const float4*)stats, 2 * p.tiles_v, N,
              (const float4*)rowk, t.sc, t.inv_t, T0, rowc, a.row_loss, reinterpret_cast<LossShare*>(ws + p.o_shares), ra.ticket, a.scale, (int)a.mean, scal, a.loss);
    if (e != cudaSuccess) return GAD_ERR_CUDA;
    if (!p.grads) return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;

    if (!make(mapH_mn, Hp, D, N, p.ldp, CT_K) || !make(mapW_mn, Wo, D, V, ldw, CT_K)) return GAD_ERR_CUDA;
    float* dh_part = reinterpret_cast<float*>(ws + p.o_dh);
    float* dw_part = reinterpret_cast<float*>(ws + p.o_dw);
    for (int i = 0; i < p.npieces; ++i) {
        const int v0 = (int)(i * p.piece), nv = (int)std::min<int64_t>(p.piece, V - v0);
        TileArgs g = t;
        g.N = nv; g.tiles_n = (nv + p.width_v - 1) / p.width_v; g.col0 = v0; g.b_row0 = v0;
        g.C = G; g.ldc = p.ldg; g.part_stride = (int64_t)N * p.ldg;
        g.colsum = a.db ? reinterpret_cast<float*>(ws + p.o_colsum) : nullptr;
        e = p.nl == 2 ? gemm_go<kGrad, false, false, T, 2>(mapH, mapW, g, s) : gemm_go<kGrad, false, false, T, 1>(mapH, mapW, g, s);
        if (e != cudaSuccess) return GAD_ERR_CUDA;
        const auto makeg = [&](CUtensorMap& m, uint32_t box) {
            return tc_make_map(&m, G, (uint64_t)nv, (uint64_t)N, (uint64_t)p.parts, (uint64_t)p.ldg * 2, (uint64_t)(p.ldg * 2 * (int64_t)N), box, false, true);
        };
        if (!makeg(mapG, CT_H) || !makeg(mapG_mn, CT_K)) return GAD_ERR_CUDA;
        if (a.dH) {
            TileArgs h = t;
            h.M = N; h.N = D; h.tiles_m = p.tiles_m; h.tiles_n = p.tiles_d; h.width = p.width_d; h.group = 8;
            h.nkb = (nv + CT_K - 1) / CT_K;
            h.kb_split = std::min(p.cut_h.kb, h.nkb); h.splits = (h.nkb + h.kb_split - 1) / h.kb_split;
            h.b_row0 = v0;
            if (p.h_parts) {
                h.C = dh_part; h.ldc = D; h.part_stride = (int64_t)N * D; h.accumulate = i > 0;
                e = gemm_go<kPartial, false, true, float, 1>(mapG, mapW_mn, h, s);
            } else {
                h.C = a.dH; h.ldc = a.lddh;
                e = gemm_go<kOut, false, true, T, 1>(mapG, mapW_mn, h, s);
            }
            if (e != cudaSuccess) return GAD_ERR_CUDA;
        }
        if (a.dW) {
            TileArgs w = t;
            w.M = nv; w.N = D; w.tiles_m = (nv + CT_M - 1) / CT_M; w.tiles_n = p.tiles_d; w.width = p.width_d; w.group = 8;
            w.nkb = (N + CT_K - 1) / CT_K; w.kb_split = p.cut_w.kb; w.splits = p.cut_w.splits; w.b_row0 = 0;
            T* out = reinterpret_cast<T*>(a.dW) + (int64_t)v0 * a.lddw;
            if (p.w_parts) {
                w.C = dw_part; w.ldc = D; w.part_stride = (int64_t)nv * D;
                e = gemm_go<kPartial, true, true, float, 1>(mapG_mn, mapH_mn, w, s);
                if (e != cudaSuccess) return GAD_ERR_CUDA;
                if (join_parts<T>(dw_part, w.splits, w.part_stride, nv, D, scal, out, a.lddw, s) != cudaSuccess) return GAD_ERR_CUDA;
            } else {
                w.C = out; w.ldc = a.lddw;
                e = gemm_go<kOut, true, true, T, 1>(mapG_mn, mapH_mn, w, s);
                if (e != cudaSuccess) return GAD_ERR_CUDA;
            }
        }
        if (a.db) {
            e = chain(class_bias_kernel<T>, dim3((unsigned)((nv + 31) / 32)), 256, 0, s, false, (const float*)g.colsum, p.ldg, 8 * p.tiles_m, nv, (const float*)scal, reinterpret_cast<T*>(a.db) + v0);
            if (e != cudaSuccess) return GAD_ERR_CUDA;
        }
    }
    if (a.dH && p.h_parts && join_parts<T>(dh_part, p.cut_h.splits, (int64_t)N * D, N, D, scal, reinterpret_cast<T*>(a.dH), a.lddh, s) != cudaSuccess) return GAD_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}

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
    if (a->rows > (1 << 30) || a->cols > (1 << 20) || a->classes > (1 << 30)) return GAD_ERR_RANGE;
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

extern "C" int gad_class_loss(const gad_class_loss_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace gad;
    const int rc = check_class(args);
    if (rc != GAD_OK) return rc;
    const gad_class_loss_args& a = *args;
    if (!a.W || !a.loss || !a.status) return GAD_ERR_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    if (a.rows == 0) return a.dtype == GAD_F32 ? run_empty<float>(a, s) : a.dtype == GAD_F16 ? run_empty<__half>(a, s) : run_empty<__nv_bfloat16>(a, s);
    if (!a.H || !a.row_loss || (a.k == 0 && !a.labels) || (a.k > 0 && (!a.target_classes || !a.teacher))) return GAD_ERR_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < (size_t)plan_class(a).total) return GAD_ERR_OOM;
    return a.dtype == GAD_F32 ? run_class<float>(a, (uint8_t*)workspace, s) : a.dtype == GAD_F16 ? run_class<__half>(a, (uint8_t*)workspace, s) : run_class<__nv_bfloat16>(a, (uint8_t*)workspace, s);
}
