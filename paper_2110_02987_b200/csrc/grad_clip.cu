// The norm over all gradients of a program, n = sqrt(sum g^2), and the gradients scaled by f = min(1, max_norm / n), in place or into tensors of their own.
//
// Two launches for up to 440 tensors.  The list of tensors is a parameter of the kernels, so nothing is copied to the device beforehand and a captured graph holds it.  Tensors are cut
// into chunks of 8192 or 32 768 values; block b takes chunks b, b + blocks, ... and leaves one sum (grad_squares_kernel).  Every block of the second launch adds those sums up
// itself, in the same order (a ticket for the last block would have to be cleared beforehand: a launch more), and scales its chunks, the last first: those the L2 still holds.
// Bound by HBM: the gradients are read twice, as far as the L2 does not hold them, and written once.
//
// Sums of squares are fp32 over the values of a chunk a thread has (two sums of at most 64 each; of rows that start anywhere 34 each, however many rows a warp has), fp64 above.  A sum outside 2^-80 .. 2^100 is taken again in fp64, so no
// square over- or underflows; whether a sum of zero is one of zeros shows in the values' bits.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

#include "half_types.cuh"

namespace gad {

namespace {

constexpr int kClipThreads = 256;
constexpr int kSmallChunk = 8192, kLargeChunk = 32768;    // values
// Chunks of 8192 values, of which a thread has four vectors (fp32: eight), by 1184 blocks, or where every block still has several of 32 768, eight vectors at a time, by 592: a tensor is looked up less often.
// (Eight vectors at a time of short chunks: half of them behind their ends, 20 million bf16 values 53 us, with four 30; four of long ones, 750 million 751 us, with eight 716.)
constexpr int kSmallBlocks = 1184, kLargeBlocks = 592;

struct ClipEntry {
    const void* g; void* out;
    long long rows, cols, ld, out_ld;
    int type, out_type;
    int first;                                           // chunk, among those of a launch
    int rows_per, pieces;                                // rows a chunk has, or pieces a row has
    int wide;                                            // every row of both starts on 16 bytes
};
template <int MOST> struct ClipTable { ClipEntry e[MOST]; int n, chunks, values; };   // values: of a chunk

// A chunk: `rows` rows of `cols` values.
struct ClipChunk { long long row, col; int rows, cols; };
template <int MOST>
__device__ __forceinline__ const ClipEntry& find_chunk(const ClipTable<MOST>& t, int c, ClipChunk& k) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].first <= c) lo = mid; else hi = mid - 1;
    }
    const ClipEntry& e = t.e[lo];
    const long long i = c - e.first;
    if (e.pieces > 1) {
        k.row = i / e.pieces;
        k.col = (i - k.row * e.pieces) * t.values;
        k.rows = 1;
        k.cols = (int)min((long long)t.values, e.cols - k.col);
    } else {
        k.row = i * e.rows_per;
        k.col = 0;
        k.rows = (int)min((long long)e.rows_per, e.rows - k.row);
        k.cols = (int)e.cols;
    }
    return e;
}

// A thread's vectors of a chunk (16 bytes, or one value: VEC = 1), AHEAD of them at a time: all are loaded before the first is used, since a store may be to where the next load is from.
template <int VEC, int AHEAD, class F>
__device__ __forceinline__ void each_vectors(const ClipChunk& k, F f) {
    const int n = (k.cols + VEC - 1) / VEC, total = n * k.rows;
    for (int i0 = threadIdx.x; i0 < total; i0 += AHEAD * kClipThreads) {
        int r[AHEAD], c[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = i0 + j * kClipThreads;
            r[j] = k.rows == 1 ? 0 : i / n;
            c[j] = i < total ? (i - r[j] * n) * VEC : k.cols;             // (behind the end of a row: nothing)
        }
        f(r, c);
    }
}

template <class T, int VEC, int AHEAD>
__device__ __forceinline__ double chunk_squares(const ClipEntry& e, const ClipChunk& k) {
    const T* base = reinterpret_cast<const T*>(e.g) + k.row * e.ld + k.col;
    float s[2] = {0.f, 0.f};
    uint32_t bits = 0;
    each_vectors<VEC, AHEAD>(k, [&](const int (&r)[AHEAD], const int (&c)[AHEAD]) {
        RowVec<T, VEC> raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) load_raw<T, VEC>(base + r[j] * e.ld, c[j], k.cols, raw[j]);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float v[VEC];
            if constexpr (VEC > 1) {
                unpack_vec<T, VEC>(raw[j].u, v);
                bits |= raw[j].u.x | raw[j].u.y | raw[j].u.z | raw[j].u.w;
            } else {
                v[0] = to_float(raw[j].e[0]);
                bits |= __float_as_uint(v[0]);
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[j & 1] = fmaf(v[i], v[i], s[j & 1]);
        }
    });
    const float both = s[0] + s[1];
    if (both >= 0x1p-80f && both <= 0x1p100f) return both;
    if ((bits & (sizeof(T) == 4 || VEC == 1 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0) return 0.0;
    double d = 0.0;
    each_vectors<VEC, AHEAD>(k, [&](const int (&r)[AHEAD], const int (&c)[AHEAD]) {
        for (int j = 0; j < AHEAD; ++j)
            for (int i = 0; i < VEC && c[j] + i < k.cols; ++i) { const double v = to_float(base[r[j] * e.ld + c[j] + i]); d = fma(v, v, d); }
    });
    return d;
}
// Rows that start anywhere: a warp has up to kRun values of a row at a time, single ones up to the first and from the last 16-byte boundary on, vectors between.  (A value a lane, with a
// division for its place, took 92 us for the norm of clip-sized 60 million values of three types, half of them in such rows, and 177 us for scaling them into fp32; now 57 and 120.)
constexpr int kRun = 2048, kLeastRun = 128;
constexpr int kRunMost = 2 + kRun / 64;                  // values of a whole run in one of a lane's two sums: single ones in front and behind, and half of its vectors
template <class F>
__device__ __forceinline__ void each_run(const ClipChunk& k, F f) {
    const int per = (k.cols + kRun - 1) / kRun, n = per * k.rows;
    for (int i = threadIdx.x >> 5; i < n; i += kClipThreads / 32) {
        const int r = per == 1 ? i : i / per, c = (i - r * per) * kRun;
        f(r, c, min(kRun, k.cols - c));
    }
}
template <class T> __device__ __forceinline__ int values_to_16(const T* p) { return (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T); }

template <class T>
__device__ __forceinline__ double run_squares(const ClipEntry& e, const ClipChunk& k) {
    constexpr int VEC = 16 / sizeof(T), U = 4;
    const T* base = reinterpret_cast<const T*>(e.g) + k.row * e.ld + k.col;
    const int lane = threadIdx.x & 31;
    double total = 0.0;
    float s[2] = {0.f, 0.f};
    uint32_t some = 0;                                   // any bit of a value but its sign
    int held = 0;                                        // values that a lane may have in either sum
    const auto one = [&](const T* p) { const float v = to_float(*p); some |= __float_as_uint(v) & 0x7FFFFFFFu; s[0] = fmaf(v, v, s[0]); };
    each_run(k, [&](int r, int c, int len) {
        const T* p = base + r * e.ld + c;
        const int head = min(len, values_to_16(p)), nv = (len - head) / VEC, tail = head + nv * VEC;
        const uint4* q = reinterpret_cast<const uint4*>(p + head);
        // short rows: their sums go on in fp64 before either has more than kRunMost values
        const int more = 2 + ((nv + 31) / 32 + 1) / 2 * VEC;
        if (held + more > kRunMost) {
            total += s[0] + s[1];
            s[0] = s[1] = 0.f;
            held = 0;
        }
        held += more;
        if (lane < head) one(p + lane);
        if (tail + lane < len) one(p + tail + lane);
        for (int i = lane; i < nv; i += 32 * U) {
            uint4 u[U];
#pragma unroll
            for (int j = 0; j < U; ++j) u[j] = i + 32 * j < nv ? q[i + 32 * j] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float v[VEC];
                unpack_vec<T, VEC>(u[j], v);
                some |= (u[j].x | u[j].y | u[j].z | u[j].w) & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
#pragma unroll
                for (int x = 0; x < VEC; ++x) s[j & 1] = fmaf(v[x], v[x], s[j & 1]);
            }
        }
    });
    total += s[0] + s[1];
    if (total >= 0x1p-80 && total <= 0x1p100) return total;
    if (some == 0) return 0.0;
    double d = 0.0;
    each_run(k, [&](int r, int c, int len) {
        const T* p = base + r * e.ld + c;
        const int head = min(len, values_to_16(p)), nv = (len - head) / VEC, tail = head + nv * VEC;
        const auto more = [&](int i) { const double v = to_float(p[i]); d = fma(v, v, d); };
        if (lane < head) more(lane);
        if (tail + lane < len) more(tail + lane);
        for (int i = lane; i < nv; i += 32)
            for (int x = 0; x < VEC; ++x) more(head + i * VEC + x);
    });
    return d;
}
template <class T, int AHEAD>
__device__ __forceinline__ double any_squares(const ClipEntry& e, const ClipChunk& k) {
    return e.wide ? chunk_squares<T, 16 / (int)sizeof(T), AHEAD>(e, k) : k.cols >= kLeastRun ? run_squares<T>(e, k) : chunk_squares<T, 1, AHEAD>(e, k);
}

__device__ __forceinline__ double block_sum(double s, double* sm) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kClipThreads / 32; ++i) s += sm[i];
    return s;
}

template <int MOST, int AHEAD>
__global__ void __launch_bounds__(kClipThreads) grad_squares_kernel(const __grid_constant__ ClipTable<MOST> t, double* __restrict__ sums) {
    __shared__ double sm[kClipThreads / 32];
    pdl_next();
    pdl_wait();
    double s = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        ClipChunk k;
        const ClipEntry& e = find_chunk(t, c, k);
        s += e.type == GAD_F32 ? any_squares<float, AHEAD>(e, k) : e.type == GAD_F16 ? any_squares<__half, AHEAD>(e, k) : any_squares<__nv_bfloat16, AHEAD>(e, k);
    }
    s = block_sum(s, sm);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <class T, class O, int VEC, int AHEAD>
__device__ __forceinline__ void scale_chunk(const ClipEntry& e, const ClipChunk& k, float f) {
    const T* src = reinterpret_cast<const T*>(e.g) + k.row * e.ld + k.col;
    O* dst = reinterpret_cast<O*>(e.out) + k.row * e.out_ld + k.col;
    each_vectors<VEC, AHEAD>(k, [&](const int (&r)[AHEAD], const int (&c)[AHEAD]) {
        RowVec<T, VEC> raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) load_raw<T, VEC>(src + r[j] * e.ld, c[j], k.cols, raw[j]);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            O* to = dst + r[j] * e.out_ld;
            if constexpr (std::is_same<T, O>::value) {
                if (f == 1.f) {                          // a copy, to the bit: a product makes one NaN of all
                    if constexpr (VEC > 1) {
                        if (c[j] + VEC <= k.cols) { *reinterpret_cast<uint4*>(to + c[j]) = raw[j].u; continue; }
                    }
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (c[j] + i < k.cols) to[c[j] + i] = raw[j].e[i];
                    continue;
                }
            }
            float v[VEC];
            if constexpr (VEC > 1) unpack_vec<T, VEC>(raw[j].u, v); else v[0] = to_float(raw[j].e[0]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] *= f;
            if constexpr (VEC == 1) {
                if (c[j] < k.cols) to[c[j]] = from_float<O>(v[0]);
            } else if constexpr (sizeof(O) == sizeof(T)) store_vec<O, VEC>(to, c[j], k.cols, v);
            else {
                // 16-bit gradients into fp32: two vectors
                const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
                store_vec<O, 4>(to, c[j], k.cols, a);
                store_vec<O, 4>(to, c[j] + 4, k.cols, b);
            }
        }
    });
}
// Scaled values leave through shared memory (256 of a warp at a time), a value a lane, where the result does not start on 16 bytes when the gradient does.
template <class T, class O>
__device__ __forceinline__ void scale_runs(const ClipEntry& e, const ClipChunk& k, float f, O* __restrict__ buf) {
    constexpr int VEC = 16 / sizeof(T), U = 4;
    const T* src = reinterpret_cast<const T*>(e.g) + k.row * e.ld + k.col;
    O* dst = reinterpret_cast<O*>(e.out) + k.row * e.out_ld + k.col;
    const int lane = threadIdx.x & 31;
    const bool copy = std::is_same<T, O>::value && f == 1.f;
    each_run(k, [&](int r, int c, int len) {
        const T* p = src + r * e.ld + c;
        O* to = dst + r * e.out_ld + c;
        const int head = min(len, values_to_16(p)), nv = (len - head) / VEC, tail = head + nv * VEC;
        const uint4* q = reinterpret_cast<const uint4*>(p + head);
        const bool vectors = ((uintptr_t)(to + head) & 15) == 0;
        const auto one = [&](int i) {
            if constexpr (std::is_same<T, O>::value) { if (copy) { to[i] = p[i]; return; } }
            to[i] = from_float<O>(to_float(p[i]) * f);
        };
        if (lane < head) one(lane);
        if (tail + lane < len) one(tail + lane);
        for (int i0 = 0; i0 < nv; i0 += 32 * U) {
            uint4 u[U];
#pragma unroll
            for (int j = 0; j < U; ++j) u[j] = i0 + 32 * j + lane < nv ? q[i0 + 32 * j + lane] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int first = i0 + 32 * j, n = (nv - first) * VEC;      // values of this and the following vectors
                if (n <= 0) break;
                union { uint4 q[sizeof(O) / sizeof(T)]; O v[VEC]; } w;
                if (copy) w.q[0] = u[j];
                else {
                    float v[VEC];
                    unpack_vec<T, VEC>(u[j], v);
#pragma unroll
                    for (int x = 0; x < VEC; ++x) w.v[x] = from_float<O>(v[x] * f);
                }
                if (vectors) {
                    if (first + lane < nv)
#pragma unroll
                        for (int x = 0; x < (int)(sizeof(O) / sizeof(T)); ++x) reinterpret_cast<uint4*>(to + head + (first + lane) * VEC)[x] = w.q[x];
                } else {
                    __syncwarp();
#pragma unroll
                    for (int x = 0; x < (int)(sizeof(O) / sizeof(T)); ++x) reinterpret_cast<uint4*>(buf + lane * VEC)[x] = w.q[x];
                    __syncwarp();
#pragma unroll
                    for (int x = 0; x < VEC; ++x)
                        if (32 * x + lane < n) to[head + first * VEC + 32 * x + lane] = buf[32 * x + lane];
                }
            }
        }
    });
}
template <class T, class O, int AHEAD>
__device__ __forceinline__ void scale_any(const ClipEntry& e, const ClipChunk& k, float f, float* buf) {
    if (e.wide) scale_chunk<T, O, 16 / (int)sizeof(T), AHEAD>(e, k, f);
    else if (k.cols >= kLeastRun) scale_runs<T, O>(e, k, f, reinterpret_cast<O*>(buf));
    else scale_chunk<T, O, 1, AHEAD>(e, k, f);
}

// write: this launch writes the norm.
template <int MOST, int AHEAD>
__global__ void __launch_bounds__(kClipThreads) grad_scale_kernel(const __grid_constant__ ClipTable<MOST> t, const double* __restrict__ sums, int nsums, float max_norm, float* __restrict__ norm, int write) {
    __shared__ double sm[kClipThreads / 32];
    __shared__ __align__(16) float staging[kClipThreads / 32][256];
    pdl_next();
    pdl_wait();
    after_wait(sums);
    double s = 0.0;
    for (int i = threadIdx.x; i < nsums; i += kClipThreads) s += sums[i];
    s = block_sum(s, sm);
    const double n = sqrt(s);
    const float nf = (float)n;
    if (write && blockIdx.x == 0 && threadIdx.x == 0) *norm = nf;
    float* buf = staging[threadIdx.x >> 5];
    // a norm that is not finite (in fp32) leaves the gradients as they are
    const float f = nf > max_norm && isfinite(nf) ? (float)((double)max_norm / n) : 1.f;
    for (int c = t.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        ClipChunk k;
        const ClipEntry& e = find_chunk(t, c, k);
        if (!e.out || (f == 1.f && e.out == e.g)) continue;
        if (e.type == GAD_F32) scale_any<float, float, AHEAD>(e, k, f, buf);
        else if (e.type == GAD_F16) { if (e.out_type == GAD_F32) scale_any<__half, float, AHEAD>(e, k, f, buf); else scale_any<__half, __half, AHEAD>(e, k, f, buf); }
        else { if (e.out_type == GAD_F32) scale_any<__nv_bfloat16, float, AHEAD>(e, k, f, buf); else scale_any<__nv_bfloat16, __nv_bfloat16, AHEAD>(e, k, f, buf); }
    }
}

constexpr int kClipMost = 440;                           // tensors a launch; parameters may take 32 764 bytes

int64_t value_bytes(int type) { return type == GAD_F32 ? 4 : 2; }
bool empty_tensor(const gad_grad_tensor& t) { return t.rows == 0 || t.cols == 0; }
// Whole rows one behind the other are one row.
void as_rows(const gad_grad_tensor& t, int64_t& rows, int64_t& cols) {
    rows = t.rows; cols = t.cols;
    if (rows > 1 && t.ld == cols && (!t.out || t.out_ld == cols)) { cols *= rows; rows = 1; }
}

int check_tensor(const gad_grad_tensor& t) {
    if (t.dtype < GAD_F32 || t.dtype > GAD_BF16 || t.rows < 0 || t.cols < 0) return GAD_ERR_ARG;
    if (t.rows > (int64_t)1 << 40 || t.cols > (int64_t)1 << 40 || (t.cols && t.rows > ((int64_t)1 << 40) / t.cols) || t.ld > (int64_t)1 << 40 || t.out_ld > (int64_t)1 << 40) return GAD_ERR_RANGE;
    if (empty_tensor(t)) return GAD_OK;
    const uintptr_t mask = (uintptr_t)value_bytes(t.dtype) - 1;
    if (!t.g || ((uintptr_t)t.g & mask) != 0 || (t.rows > 1 && t.ld < t.cols)) return GAD_ERR_ARG;
    if (!t.out) return GAD_OK;
    if (t.out_dtype != t.dtype && t.out_dtype != GAD_F32) return GAD_ERR_ARG;
    if (((uintptr_t)t.out & ((uintptr_t)value_bytes(t.out_dtype) - 1)) != 0 || (t.rows > 1 && t.out_ld < t.cols)) return GAD_ERR_ARG;
    if (t.out == t.g && (t.out_dtype != t.dtype || (t.rows > 1 && t.out_ld != t.ld))) return GAD_ERR_ARG;
    return GAD_OK;
}

// What is written must not be read or written elsewhere in the list.  Column ranges of the same matrix do not meet although their first to last bytes do: of all of its rows, of every second
// (third ..) one, of one (ld 0).
struct Region { uintptr_t lo, hi; int64_t ld, width; bool written; };
bool meet(const Region& a, const Region& b) {                        // (a.lo <= b.lo < a.hi)
    const int64_t least = std::min(a.ld, b.ld), period = least ? least : std::max(a.ld, b.ld);
    if (period && a.ld % period == 0 && b.ld % period == 0) {
        const int64_t d = (int64_t)((b.lo - a.lo) % (uintptr_t)period);
        if (d >= a.width && d + b.width <= period) return false;
    }
    return true;
}
int check_regions(const gad_grad_tensor* t, int64_t count) {
    std::vector<Region> all;
    all.reserve(2 * (size_t)count);
    for (int64_t i = 0; i < count; ++i) {
        if (empty_tensor(t[i])) continue;
        const auto add = [&](const void* p, int64_t ld, int type, bool written) {
            const int64_t e = value_bytes(type);
            const bool rows = t[i].rows > 1 && ld != t[i].cols;
            all.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)(((t[i].rows - 1) * (t[i].rows > 1 ? ld : 0) + t[i].cols) * e), rows ? ld * e : 0, t[i].cols * e, written});
        };
        const bool inside = t[i].out == t[i].g;
        add(t[i].g, t[i].ld, t[i].dtype, inside);
        if (t[i].out && !inside) add(t[i].out, t[i].out_ld, t[i].out_dtype, true);
    }
    std::sort(all.begin(), all.end(), [](const Region& a, const Region& b) { return a.lo < b.lo; });
    for (size_t i = 0; i < all.size(); ++i)
        for (size_t j = i + 1; j < all.size() && all[j].lo < all[i].hi; ++j)
            if ((all[i].written || all[j].written) && meet(all[i], all[j])) return GAD_ERR_ARG;
    return GAD_OK;
}

template <int MOST>
int fill_table(const gad_grad_tensor* t, int64_t& i, int64_t count, bool scaled, int values, ClipTable<MOST>& table) {
    table.n = 0;
    table.values = values;
    int64_t chunks = 0;
    for (; i < count && table.n < MOST; ++i) {
        if (empty_tensor(t[i]) || (scaled && !t[i].out)) continue;
        ClipEntry& e = table.e[table.n];
        int64_t rows, cols;
        as_rows(t[i], rows, cols);
        const int64_t a = value_bytes(t[i].dtype), b = value_bytes(t[i].out_dtype);
        e.g = t[i].g; e.out = t[i].out; e.rows = rows; e.cols = cols; e.ld = t[i].ld; e.out_ld = t[i].out_ld;
        e.type = t[i].dtype; e.out_type = t[i].out_dtype;
        e.wide = ((uintptr_t)e.g % 16 == 0) && (rows == 1 || t[i].ld * a % 16 == 0);
        if (t[i].out) e.wide = e.wide && ((uintptr_t)e.out % 16 == 0) && (rows == 1 || t[i].out_ld * b % 16 == 0);
        e.pieces = (int)((cols + values - 1) / values);
        e.rows_per = e.pieces > 1 ? 1 : (int)std::min<int64_t>(rows, std::max<int64_t>(1, values / cols));
        e.first = (int)chunks;
        const int64_t more = e.pieces > 1 ? rows * e.pieces : (rows + e.rows_per - 1) / e.rows_per;
        if (chunks + more > INT32_MAX / 2) { if (table.n == 0) return GAD_ERR_RANGE; break; }
        chunks += more;
        ++table.n;
    }
    table.chunks = (int)chunks;
    return GAD_OK;
}


template <int MOST, int AHEAD>
int run_clip(const gad_grad_tensor* t, int64_t count, float max_norm, float* norm, double* sums, cudaStream_t s) {
    ClipTable<MOST> table;
    const int values = AHEAD == 8 ? kLargeChunk : kSmallChunk;
    const auto blocks_for = [](int chunks) { return std::max(1, std::min(chunks, AHEAD == 8 ? kLargeBlocks : kSmallBlocks)); };
    int nsums = 0;
    bool first = true;
    for (int64_t i = 0; i < count || first;) {
        const int rc = fill_table(t, i, count, false, values, table);
        if (rc != GAD_OK) return rc;
        const int blocks = blocks_for(table.chunks);
        if (chain((grad_squares_kernel<MOST, AHEAD>), dim3((unsigned)blocks), kClipThreads, 0, s, first, table, sums + nsums) != cudaSuccess) return GAD_ERR_CUDA;
        nsums += blocks;
        first = false;
    }
    bool write = true;
    for (int64_t i = 0; i < count || write;) {
        const int rc = fill_table(t, i, count, true, values, table);
        if (rc != GAD_OK) return rc;
        if (!table.chunks && !write) break;
        if (chain((grad_scale_kernel<MOST, AHEAD>), dim3((unsigned)blocks_for(table.chunks)), kClipThreads, 0, s, false, table, (const double*)sums, nsums, max_norm, norm, (int)write) != cudaSuccess) return GAD_ERR_CUDA;
        write = false;
    }
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}

// Launches of the first kernel are at most one a kClipMost tensors, and one for every run of 2^30 chunks.
size_t clip_bytes(int64_t count) { return sizeof(double) * kSmallBlocks * (size_t)(2 + count / 16); }
template <int AHEAD>
int run_clip(const gad_grad_tensor* t, int64_t count, float max_norm, float* norm, double* sums, cudaStream_t s) {
    return count <= 16 ? run_clip<16, AHEAD>(t, count, max_norm, norm, sums, s) : count <= 64 ? run_clip<64, AHEAD>(t, count, max_norm, norm, sums, s) : run_clip<kClipMost, AHEAD>(t, count, max_norm, norm, sums, s);
}

int check_list(const gad_grad_tensor* t, int64_t count) {
    if (count < 0 || (count > 0 && !t)) return GAD_ERR_ARG;
    if (count > 1 << 20) return GAD_ERR_RANGE;
    for (int64_t i = 0; i < count; ++i) {
        const int rc = check_tensor(t[i]);
        if (rc != GAD_OK) return rc;
    }
    return GAD_OK;
}

}  // namespace
}  // namespace gad

extern "C" int gad_clip_grads_workspace_bytes(int64_t count, size_t* bytes) {
    if (count < 0 || !bytes) return GAD_ERR_ARG;
    if (count > 1 << 20) return GAD_ERR_RANGE;
    *bytes = gad::clip_bytes(count);
    return GAD_OK;
}

extern "C" int gad_clip_grads(const gad_grad_tensor* tensors, int64_t count, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace gad;
    try {
        int rc = check_list(tensors, count);
        if (rc != GAD_OK) return rc;
        if (!norm || !(max_norm >= 0.f)) return GAD_ERR_ARG;
        rc = check_regions(tensors, count);
        if (rc != GAD_OK) return rc;
        if (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < clip_bytes(count)) return GAD_ERR_OOM;
        const cudaStream_t s = (cudaStream_t)stream;
        double* sums = (double*)workspace;
        int64_t all = 0;
        for (int64_t i = 0; i < count; ++i) all += tensors[i].rows * tensors[i].cols;
        return all >= (int64_t)8 * kLargeBlocks * kLargeChunk ? run_clip<8>(tensors, count, max_norm, norm, sums, s) : run_clip<4>(tensors, count, max_norm, norm, sums, s);
    } catch (...) {   // (the list of regions could not grow)
        return GAD_ERR_OOM;
    }
}
