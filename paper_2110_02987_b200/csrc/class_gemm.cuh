// The matrix product of the output head: C [M x N] = A B^T over 16-bit operands with fp32 accumulators, by pairs of CTAs on tcgen05, and what
// the loss does with a finished tile.  Used by class_loss.cu for
//   kStats     z = H W^T + b: per row and half a tile the largest value, the sum(s) of the softmax and the product with the row's targets; where gradients are
//              wanted, z itself for class_grad_kernel: in 16 bits below that largest value, or in fp32
//   kOut       dH = G W and dW = G^T H, scaled and rounded to the result's type
//
// Tiles of 256 x 256 by two CTAs (cta_group::2): each loads its 128 rows of A and 128 of the 256 rows of B, 64 values of the reduction at a time, into a ring of six
// stages of 32 KB, so that a value that is multiplied 256 times comes from L2 62 bytes a cycle and SM; two accumulators, one filled while eight warps drain
// the other.  Both operands may be K-major (a row of the matrix is a row of the reduction) or MN-major (the reduction runs over rows), so that H, W and G are read as they
// lie.  Tiles are gone through in groups of rows whose operands fit the L2 beside what streams past.
// What bounds it, 4096 x 1024 against 32 768 classes (275 GFLOP each): the tensor pipe, 77 to 79 % busy (statistics 173 us, dH 165 us with 64 tiles on 74 pairs, dW 170 us)
// at 1.7 GHz, and in long runs the card's power: at 990 W it settles at 1.4 to 1.5 GHz, where a library's three plain products of these sizes take 682 us.
#pragma once

#include <cuda.h>

#include "gad_internal.h"
#include "half_types.cuh"
#include "tc_common.cuh"

namespace gad {

namespace {

constexpr int CT_M = 256, CT_H = 128, CT_K = 64;            // rows of a pair's tile, of a CTA's share, reduction per ring stage
constexpr int CT_OPERAND = CT_H * CT_K * 2;                 // 16 KiB
constexpr int CT_STAGE = 2 * CT_OPERAND;                    // A | B
constexpr int CT_STAGES = 6;
constexpr int CT_RING = CT_STAGES * CT_STAGE;
constexpr int CT_EPI_WARPS = 8, CT_EPI_WARP0 = 2;           // two per quarter of the tensor-memory lanes, half of the columns each
constexpr int CT_THREADS = 32 * (CT_EPI_WARP0 + CT_EPI_WARPS);
constexpr int CT_BIAS = CT_EPI_WARPS * 128 * 4;             // a draining warp's biases
constexpr int CT_STAGING = CT_EPI_WARPS * 2048;             // and 64 bytes of each of its rows on their way out
constexpr int CT_SMEM = CT_RING + 1024 + 256 + CT_BIAS + CT_STAGING;
constexpr int CT_TMEM = 512;                                // two accumulators of 256 columns, or four of 128

enum TileUse { kStats, kOut };

// z of a row is kept as whole numbers of 1 / 2048 octaves below the largest of the 128 (64) classes that a draining warp has of it: 16 bits reach 32 octaves, and a
// probability is off by 1.7e-4 of itself, a fourteenth of what bfloat16 and two thirds of what fp16 rounds off it.  The last code is a probability of zero.
// Of two softmaxes the flatter one's octaves count (T > 1: those of z / T), or else classes behind the last code would lose their part of it; the sharper one is off by T (1 / T) times as much.
constexpr float kCodeSteps = 2048.f;
constexpr int kCodeZero = 65535;
enum SaveAs { kSaveNone, kSaveCode, kSaveFloat };
enum AddTo { kAddNone, kAddFirst, kAddMore, kAddLast };   // result; sums [M x N] in fp32: begun, added to, added and turned into the result

struct TileArgs {
    int M, N;                  // result
    int tiles_m, tiles_n, width;   // tiles of 256 x width (128 or 256)
    int nkb;                   // 64-blocks of the reduction
    int whole;                 // tiles whose reduction is one unit of work; those behind them come in `shares` of kb_share blocks each
    int shares, kb_share;
    int group;                 // row tiles that are gone through together, for the L2
    int pairs;                 // products of operand parts: 1, or 6 for operands in three parts
    int chunk;                 // ADD_UP: blocks that are summed in tensor memory (of operands in parts all products, the smallest first) before the sum moves to registers
    int a_row0;                // first row of A (K-major)
    int b_row0;                // first row of B (MN-major)
    int bf16;                  // operand type: 1 bfloat16, 0 fp16
    int32_t* err;
    // kStats
    const void* bias;          // [classes] in the caller's type, or null
    int bias_type;
    float sc, inv_t;           // of the logits: log2(e) (/ T with one softmax); 1 / T of the second softmax
    const int2* targets;       // [M x ntargets] (class, weight), classes ascending
    int ntargets;
    const uint16_t* starts;    // [M x 2 tiles_n] a row's first target at or behind the first column of each half tile; null with one target
    float4* stats;             // [2 tiles_n x M]
    int save;                  // SaveAs
    float code_steps, code_lowest;   // codes a unit of z (two softmaxes may need fewer than kCodeSteps), and what the last code stands for
    // what is written
    void* C;                   // kStats: z as saved [M x ldc]; kOut: the result
    long long ldc;
    int add;                   // AddTo
    float* sums;               // [M x N]
    float* slots;              // [tiles - whole][shares][256 x width] sums of shares
    const float* scal;         // [1] factor of the results
};

// Products of operand parts, the smallest first, so that what an addition to the accumulator cuts off is small for as long as possible.
__device__ __forceinline__ void part_pair(int p, int pairs, int& a, int& b) {
    if (pairs == 1) { a = b = 0; return; }
    a = (0x012010 >> (4 * (5 - p))) & 15;     // 0 1 2 0 1 0
    b = (0x210100 >> (4 * (5 - p))) & 15;     // 2 1 0 1 0 0
}

// Shared-memory descriptors: K-major as smem_desc; MN-major (16-bit): blocks of 64 values of the M or N axis (128 bytes, 64 reduction rows: 8 KiB apart),
// groups of eight reduction rows 1024 bytes apart.
template <bool MN>
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr) {
    if (!MN) return smem_desc(saddr);
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// A tile into this CTA's shared memory whose bytes count at a barrier of the pair's leader.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t leader_bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(leader_bar)
                 : "memory");
}
__device__ __forceinline__ uint32_t leader_address(uint32_t addr) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

// This warp's 32 tensor-memory lanes x 32 columns, complete on return.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// The same in two steps, so that a block of columns is on its way while the one in front is worked on.
__device__ __forceinline__ void tmem_ld32_start(uint32_t addr, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
          "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(addr)
        : "memory");
}
// (the values pass through, so that nothing reads them before)
__device__ __forceinline__ void tmem_ld32_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
          "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
          "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
        :
        : "memory");
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// v[c] for a c that is not known to the compiler, by halving.
__device__ __forceinline__ float pick(const float (&v)[32], int c) {
    float a[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) a[j] = (c & 16) ? v[j + 16] : v[j];
#pragma unroll
    for (int w = 8; w > 0; w >>= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < w) a[j] = (c & w) ? a[j + w] : a[j];
    return a[0];
}

// The bfloat16 parts of a value: x = hi + mid + lo, each the nearest to what is left (a finite value stays finite).
__device__ __forceinline__ void split3(float x, __nv_bfloat16 (&p)[3]) {
    __nv_bfloat16 h = __float2bfloat16_rn(x);
    if (__hisinf(h) && !isinf(x)) h = __ushort_as_bfloat16((unsigned short)(0x7F7F | (__float_as_uint(x) >> 31 << 15)));
    const float r = x - __bfloat162float(h);
    p[0] = h;
    p[1] = __float2bfloat16_rn(r);
    p[2] = __float2bfloat16_rn(r - __bfloat162float(p[1]));
}

// Rows leave through shared memory, 64 bytes of each of a warp's 32 rows at a time: written from registers they would go out as 32 separate 16-byte (or,
// where rows do not start on 16 bytes, one-element) stores, each half a sector or less (dW of 10 007 x 500 fp16, whose rows start on 8 bytes: 83 us, as whole sectors
// 20).  Units of 16 bytes are swizzled by the row, so neither side has bank conflicts.
__device__ __forceinline__ uint8_t* staged(uint8_t* buf, int row, int unit) { return buf + row * 64 + ((unit ^ ((row >> 1) & 3)) << 4); }

// GB: bytes of a store, a divisor of every row's address.
template <int GB, class T, bool ADD>
__device__ __forceinline__ void copy_out(uint8_t* buf, int lane, T* __restrict__ out, long long ld, int rows, int cols) {
    constexpr int PER = 64 / GB, ROWS = 32 / PER, E = GB / sizeof(T);
    const int g = lane % PER, e0 = g * E;
    if (e0 >= cols) return;
#pragma unroll
    for (int r = lane / PER; r < 32; r += ROWS) {
        if (r >= rows) break;
        union { T e[E]; uint4 u4; uint2 u2; uint32_t u1; uint16_t h; } w;
        const uint8_t* src = staged(buf, r, (g * GB) >> 4) + ((g * GB) & 15);
        if constexpr (GB == 16) w.u4 = *reinterpret_cast<const uint4*>(src);
        else if constexpr (GB == 8) w.u2 = *reinterpret_cast<const uint2*>(src);
        else if constexpr (GB == 4) w.u1 = *reinterpret_cast<const uint32_t*>(src);
        else w.h = *reinterpret_cast<const uint16_t*>(src);
        T* at = out + r * ld + e0;
        if (E == 1 || e0 + E <= cols) {
            if constexpr (ADD) {
#pragma unroll
                for (int i = 0; i < E; ++i) w.e[i] += at[i];
            }
            if constexpr (GB == 16) *reinterpret_cast<uint4*>(at) = w.u4;
            else if constexpr (GB == 8) *reinterpret_cast<uint2*>(at) = w.u2;
            else if constexpr (GB == 4) *reinterpret_cast<uint32_t*>(at) = w.u1;
            else *reinterpret_cast<uint16_t*>(at) = w.h;
        } else {
            for (int i = 0; i < E && e0 + i < cols; ++i) {
                if constexpr (ADD) w.e[i] += at[i];
                at[i] = w.e[i];
            }
        }
    }
}
// The largest store every row of a matrix allows.
__device__ __forceinline__ int store_bytes(const void* p, long long ld_bytes) {
    const unsigned long long m = (unsigned long long)p | (unsigned long long)ld_bytes;
    return m % 16 == 0 ? 16 : m % 8 == 0 ? 8 : m % 4 == 0 ? 4 : 2;
}
// A lane's 32 values (a row each) to out[row of the warp][0 .. 32), at most `cols` columns of `rows` rows.
template <class T, bool ADD = false>
__device__ __forceinline__ void drain_rows(uint8_t* buf, int lane, const float (&v)[32], T* __restrict__ out, long long ld, int rows, int cols, int bytes) {
    constexpr int PER = 64 / sizeof(T);           // columns a time
#pragma unroll
    for (int c = 0; c < 32; c += PER) {
        if (c >= cols) break;
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            union { uint4 u; T e[16 / sizeof(T)]; } w;
#pragma unroll
            for (int i = 0; i < 16 / (int)sizeof(T); ++i) w.e[i] = from_float<T>(v[c + k * (16 / sizeof(T)) + i]);
            *reinterpret_cast<uint4*>(staged(buf, lane, k)) = w.u;
        }
        __syncwarp();
        if (bytes == 16) copy_out<16, T, ADD>(buf, lane, out + c, ld, rows, cols - c);
        else if (bytes == 8) copy_out<8, T, ADD>(buf, lane, out + c, ld, rows, cols - c);
        else if (bytes == 4 || sizeof(T) == 4) copy_out<4, T, ADD>(buf, lane, out + c, ld, rows, cols - c);
        else copy_out<sizeof(T) == 4 ? 4 : 2, T, ADD>(buf, lane, out + c, ld, rows, cols - c);
    }
}

// The same for codes, already whole numbers in the low 16 bits of the values.
__device__ __forceinline__ void drain_codes(uint8_t* buf, int lane, const float (&v)[32], uint16_t* __restrict__ out, long long ld, int rows) {
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __byte_perm(__float_as_uint(v[8 * k + 2 * i]), __float_as_uint(v[8 * k + 2 * i + 1]), 0x5410);
        *reinterpret_cast<uint4*>(staged(buf, lane, k)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncwarp();
    copy_out<16, uint16_t, false>(buf, lane, out, ld, rows, 32);
}

// A unit of work: a tile, and the blocks of its reduction.
struct TileAt { int m, n, kb0, nkb, slot; };
__device__ __forceinline__ long long units_of(const TileArgs& a) { return a.whole + ((long long)a.tiles_m * a.tiles_n - a.whole) * a.shares; }
__device__ __forceinline__ TileAt tile_at(const TileArgs& a, long long u) {
    TileAt t;
    long long i = u;
    t.kb0 = 0; t.nkb = a.nkb; t.slot = -1;
    if (u >= a.whole && a.shares > 1) {
        t.slot = (int)(u - a.whole);
        i = a.whole + t.slot / a.shares;
        t.kb0 = t.slot % a.shares * a.kb_share;
        t.nkb = min(a.kb_share, a.nkb - t.kb0);
    }
    const long long per = (long long)a.group * a.tiles_n;
    const int g = (int)(i / per), first = g * a.group, rows = min(a.group, a.tiles_m - first);
    const int r = (int)(i - g * per);
    t.m = first + r % rows;
    t.n = r / rows;
    return t;
}

// USE as above; A_MN, B_MN: operand is MN-major; T: type of the result; NL: softmaxes (temperatures) at once.
// ADD_UP: the tensor core cuts its accumulator off at every addition (it does not round), always towards zero, so that a sum of 16 n terms comes out short by about 1.4e-8 n of
// itself (measured over logits of 256 to 2048 terms of either sign; of one sign 4e-8 in bfloat16 and 9e-8 in fp16; the worst is 2^-23), and one whose parts need no more
// than 24 bits, as whole numbers or rows with few values, not at all.  (A factor that gave the mean back made those wrong by as much.)  Where a result is wanted to fp32 accuracy, or the sum is so long that a 16-bit result would show it, the
// reduction is cut into chunks whose sums the draining threads add up in registers.  Of operands in parts a chunk has all products, the smallest first (what they lose is
// small), so that the parts come from HBM once: with the products one behind the other over the whole reduction G was read six times (8192 x 4096 x 256: 92 us).
// Logits are then taken in tiles 128 columns wide: 64 sums a thread, four accumulators, three of which fill while the sums of a tile are worked on.  Gradients, with many
// chunks a tile, keep tiles of 256: at 128 the operands come from L2 half as fast again as it can (8192 x 256 x 4096 fp32: 157 us instead of 92).
template <int USE, bool A_MN, bool B_MN, class T, int NL, bool ADD_UP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(CT_THREADS, 1)
class_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ TileArgs a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;   // the same in both CTAs
    uint8_t* sm = smem_raw + pad;
    const uint32_t sm_addr = raw_addr + pad;
    const uint32_t rank = cluster_rank();
    const uint32_t bars = sm_addr + CT_RING;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (CT_STAGES + s); };
    auto tfull = [&](int i) { return bars + 8u * (2 * CT_STAGES + i); };
    constexpr int NACC = ADD_UP && USE == kStats ? 4 : 2, ACC_COLS = CT_TMEM / NACC;
    auto tempty = [&](int i) { return bars + 8u * (2 * CT_STAGES + NACC + i); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + CT_RING + 8 * (2 * CT_STAGES + 2 * NACC));
    volatile uint32_t* abort_flag = tmem_slot + 1;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < CT_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int i = 0; i < NACC; ++i) { mbar_init(tfull(i), 1); mbar_init(tempty(i), 2 * CT_EPI_WARPS); }
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_next();
    if (warp == 0) tmem_alloc2(smem_u32(tmem_slot), CT_TMEM);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();           // the peer's barriers exist before anything arrives at them
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    const int ncl = gridDim.x >> 1, half_w = a.width / 2;
    const long long units = units_of(a);

    if (warp == 0 && lane == 0) {
        // ---------------- TMA producer: this CTA's rows of A and half of the rows of B, 64 of the reduction at a time; the leader's barrier counts both CTAs' bytes
        // (passed on by a thread of the other CTA, a full stage was known too late for the six of the ring to bridge: all products 4 to 5 % longer) ----------------
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long u = blockIdx.x >> 1; u < units && ok; u += ncl) {
            const TileAt t = tile_at(a, u);
            const int ra = t.m * CT_M + (int)rank * CT_H, rb = t.n * a.width + (int)rank * half_w;
            const int group = ADD_UP ? a.chunk : t.nkb;
            for (int g = 0; g < t.nkb && ok; g += group)
                for (int p = 0; p < a.pairs && ok; ++p) {
                    int za, zb;
                    part_pair(p, a.pairs, za, zb);
                    for (int kb = t.kb0 + g; kb < t.kb0 + min(g + group, t.nkb); ++kb) {
                        if (!(ok = mbar_wait(empty(stage), phase ^ 1u, abort_flag, a.err, 31))) break;
                        if (rank == 0) mbar_expect_tx(full(stage), 2u * (uint32_t)(CT_H + half_w) * (CT_K * 2));
                        const uint32_t base = sm_addr + stage * CT_STAGE, bar = leader_address(full(stage));
                        if (A_MN) {
                            tma_load_3d_pair(base, &tmA, ra, kb * CT_K, za, bar);
                            tma_load_3d_pair(base + 8192, &tmA, ra + 64, kb * CT_K, za, bar);
                        } else {
                            tma_load_3d_pair(base, &tmA, kb * CT_K, a.a_row0 + ra, za, bar);
                        }
                        if (B_MN) {
                            for (int j = 0; j < half_w; j += 64) tma_load_3d_pair(base + CT_OPERAND + j * 128, &tmB, rb + j, a.b_row0 + kb * CT_K, zb, bar);
                        } else {
                            tma_load_3d_pair(base + CT_OPERAND, &tmB, kb * CT_K, rb, zb, bar);
                        }
                        if (++stage == CT_STAGES) { stage = 0; phase ^= 1u; }
                    }
                }
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------- MMA issuer (leader of the pair): the whole warp runs the loop, one elected lane issues ----------------
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        const uint32_t idesc = instr_desc_f16(a.width, CT_M) | (a.bf16 ? (1u << 7) | (1u << 10) : 0u) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
        constexpr uint32_t stepA = A_MN ? 128 : 2, stepB = B_MN ? 128 : 2;    // 16 values of the reduction: 16 rows of 128 bytes, or 32 bytes of a row
        bool ok = true;
        for (long long u = blockIdx.x >> 1; u < units && ok; u += ncl) {
            const int steps = tile_at(a, u).nkb * a.pairs;
            int left = 0;                                          // stages until this accumulator is full
            for (int i = 0; i < steps; ++i) {
                const bool first = left == 0;
                if (first) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(tempty(acc), acc_phase ^ 1u, abort_flag, a.err, 32)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    left = ADD_UP ? min(a.chunk * a.pairs, steps - i) : steps;
                }
                const uint32_t d = tmem_base + (uint32_t)(acc * ACC_COLS);
                if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(full(stage), phase, abort_flag, a.err, 33)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base = sm_addr + stage * CT_STAGE;
                const uint64_t da = operand_desc<A_MN>(base), db = operand_desc<B_MN>(base + CT_OPERAND);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < CT_K / 16; ++ks) mma_f16_pair(d, da + stepA * ks, db + stepB * ks, idesc, !first || ks != 0 ? 1u : 0u);
                    mma_commit2(empty(stage));                    // in both CTAs
                    if (left == 1) mma_commit2(tfull(acc));
                }
                __syncwarp();
                if (++stage == CT_STAGES) { stage = 0; phase ^= 1u; }
                if (--left == 0 && ++acc == NACC) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else if (warp >= CT_EPI_WARP0) {   // (warp 1 of the other CTA has nothing to do)
        // ---------------- drain: this warp's 32 rows (a row a lane) x half of the tile's columns ----------------
        const int ew = warp - CT_EPI_WARP0, q = warp & 3, half = ew >> 2;
        float* bias = reinterpret_cast<float*>(sm + CT_RING + 256) + ew * 128;
        uint8_t* buf = sm + CT_RING + 256 + CT_BIAS + ew * 2048;
        int acc = 0;
        uint32_t acc_phase = 0;
        const float factor = USE == kOut ? a.scal[1] : 1.f;
        const int bytes = USE == kOut ? store_bytes(a.C, a.ldc * (long long)sizeof(T)) : 16, sum_bytes = a.N % 4 == 0 ? 16 : a.N % 2 == 0 ? 8 : 4;
        for (long long u = blockIdx.x >> 1; u < units; u += ncl) {
            const TileAt t = tile_at(a, u);
            const int row0 = t.m * CT_M + (int)rank * CT_H + q * 32, rows = a.M - row0;   // this warp's rows
            const int row = row0 + lane;
            const bool rv = row < a.M;
            const int tile_c = t.n * a.width + half * half_w;               // first column of this warp
            float m2 = -INFINITY, s1 = 0.f, s2 = 0.f, dot = 0.f;
            int e = 0;
            int2 cur = make_int2(INT_MAX, 0), nxt = cur;                    // the row's next target among these columns, and the one behind it
            const int2* tg = a.targets + (long long)(rv ? row : 0) * a.ntargets;
            if (USE == kStats) {
                __syncwarp();                                               // the previous tile's biases have been read
                for (int j = lane; j < half_w; j += 32) {
                    const int c = tile_c + j;
                    float b = c < a.N ? 0.f : -INFINITY;                    // columns that are no class carry no weight
                    if (a.bias && c < a.N)
                        b = a.bias_type == GAD_F32 ? reinterpret_cast<const float*>(a.bias)[c]
                            : a.bias_type == GAD_F16 ? to_float(reinterpret_cast<const __half*>(a.bias)[c]) : to_float(reinterpret_cast<const __nv_bfloat16*>(a.bias)[c]);
                    bias[j] = b * a.sc;
                }
                __syncwarp();
                if (rv) {
                    if (a.starts) e = a.starts[(long long)row * (2 * a.tiles_n) + 2 * t.n + half];
                    if (e < a.ntargets) cur = tg[e];
                    if (e + 1 < a.ntargets) nxt = tg[e + 1];
                    if (cur.x < tile_c) cur.x = INT_MAX;                    // (one target, in front of these columns)
                }
            }
            // No bias and nothing but classes: the logit and its distance from the largest are one multiply-add, which rounds once.  The largest logit is therefore rounded up: rounded
            // to nearest it can lie below the exact product, and the distance of its own class, behind the multiply-add, above zero, where there is no code.
            const bool plain = !a.bias && (t.n + 1) * a.width <= a.N;
            const auto largest = [&](int c0, const float (&v)[32]) {
                float m[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) m[k] = plain ? v[k] : fmaf(v[k], a.sc, bias[c0 + k]);
                if (plain) {
#pragma unroll
                    for (int j = 4; j < 32; ++j) m[j & 3] = fmaxf(m[j & 3], v[j]);
                } else {
#pragma unroll
                    for (int j = 4; j < 32; ++j) m[j & 3] = fmaxf(m[j & 3], fmaf(v[j], a.sc, bias[c0 + j]));
                }
                m2 = fmaxf(m2, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
            };
            // 32 finished values of this thread's row, from column c0 of the warp's columns on
            const auto take = [&](int c0, float (&v)[32]) {
                if (USE == kStats) {
                    const float base = m2 == -INFINITY ? 0.f : m2;          // nothing but masked classes: all terms are zero
                    if (a.save == kSaveFloat) {
                        float z[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = plain ? v[j] * a.sc : fmaf(v[j], a.sc, bias[c0 + j]);
                        drain_rows<float>(buf, lane, z, reinterpret_cast<float*>(a.C) + (long long)row0 * a.ldc + tile_c + c0, a.ldc, rows, 32, 16);
                    }
                    if (plain) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(v[j], a.sc, -base);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(v[j], a.sc, bias[c0 + j]) - base;
                    }
                    float p1[4] = {0.f, 0.f, 0.f, 0.f}, p2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        p1[j & 3] += exp2_fast(v[j]);
                        if (NL == 2) p2[j & 3] += exp2_fast(v[j] * a.inv_t);
                    }
                    s1 += (p1[0] + p1[1]) + (p1[2] + p1[3]);
                    if (NL == 2) s2 += (p2[0] + p2[1]) + (p2[2] + p2[3]);
                    while (cur.x < tile_c + c0 + 32) {                      // (the target that is loaded here is not looked at before the next but one)
                        dot = fmaf(__int_as_float(cur.y), pick(v, cur.x - tile_c - c0) + base, dot);
                        cur = nxt;
                        ++e;
                        nxt = e + 1 < a.ntargets ? tg[e + 1] : make_int2(INT_MAX, 0);
                    }
                    if (a.save == kSaveCode) {
                        // rounded by the addition of 2^23, whose sum has the whole number in its low bits
                        const float steps = NL == 2 ? a.code_steps : kCodeSteps, lowest = NL == 2 ? a.code_lowest : -(float)kCodeZero / kCodeSteps;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(fmaxf(v[j], lowest), -steps, 8388608.f);
                        drain_codes(buf, lane, v, reinterpret_cast<uint16_t*>(a.C) + (long long)row0 * a.ldc + tile_c + c0, a.ldc, rows);
                    }
                } else if (tile_c + c0 < a.N) {
                    const int cols = a.N - tile_c - c0;
                    const long long at = (long long)row0 * a.N + tile_c + c0;
                    if (t.slot >= 0) {
                        float* out = a.slots + (long long)t.slot * CT_M * a.width + (long long)(row0 - t.m * CT_M) * a.width + half * half_w + c0;
                        drain_rows<float>(buf, lane, v, out, a.width, 32, 32, 16);
                    } else if (a.add == kAddFirst) {
                        drain_rows<float>(buf, lane, v, a.sums + at, a.N, rows, cols, sum_bytes);
                    } else if (a.add == kAddMore) {
                        drain_rows<float, true>(buf, lane, v, a.sums + at, a.N, rows, cols, sum_bytes);
                    } else {
                        if (a.add == kAddLast) {
                            // sums come in through the staging buffer, as they left
#pragma unroll
                            for (int c = 0; c < 32; c += 16) {
                                __syncwarp();
                                for (int i = lane; i < 32 * 16; i += 32) {
                                    const int r = i >> 4, x = i & 15;
                                    *reinterpret_cast<float*>(staged(buf, r, x >> 2) + (x & 3) * 4) = r < rows && c + x < cols ? a.sums[at + (long long)r * a.N + c + x] : 0.f;
                                }
                                __syncwarp();
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[c + j] += *reinterpret_cast<const float*>(staged(buf, lane, j >> 2) + (j & 3) * 4);
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= factor;
                        drain_rows<T>(buf, lane, v, reinterpret_cast<T*>(a.C) + (long long)row0 * a.ldc + tile_c + c0, a.ldc, rows, cols, bytes);
                    }
                }
            };
            const uint32_t tm_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * half_w);
            const auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_leader_tmem(tempty(acc));
                if (++acc == NACC) { acc = 0; acc_phase ^= 1u; }
            };
            bool ok = true;
            const auto wait_full = [&]() {
                ok = __all_sync(0xffffffffu, mbar_wait(tfull(acc), acc_phase, abort_flag, a.err, 36));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            if constexpr (ADD_UP) {
                const int chunks = (t.nkb + a.chunk - 1) / a.chunk;
                constexpr int BLOCKS = USE == kStats ? 2 : 4;               // of 32 columns a warp has
                float sum[BLOCKS][32];
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[c][j] = 0.f;
                for (int i = 0; i < chunks; ++i) {
                    if (!wait_full()) break;
#pragma unroll
                    for (int c = 0; c < BLOCKS; ++c) {
                        if (32 * c >= half_w) break;
                        float v[32];
                        tmem_ld32(tm_row + (uint32_t)(acc * ACC_COLS + 32 * c), v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[c][j] += v[j];
                    }
                    if (USE == kStats || i < chunks - 1) release();
                }
                if (!ok) break;
                if constexpr (USE == kStats) {
                    largest(0, sum[0]);
                    largest(32, sum[1]);
                    if (plain) m2 = __fmul_ru(m2, a.sc);
                    take(0, sum[0]);
                    take(32, sum[1]);
                } else {
                    // the sums take the place of the last chunk, and are taken from there block by block: held in registers beside what follows they would spill
#pragma unroll
                    for (int c = 0; c < BLOCKS; ++c)
                        if (32 * c < half_w) tmem_st_32x32b_x32(tm_row + (uint32_t)(acc * ACC_COLS + 32 * c), sum[c]);
                    tmem_wait_st();
                }
            } else if (!wait_full()) break;
            if (!ADD_UP && rows <= 0) {                                     // (nothing of this warp's rows is asked for)
                release();
            } else if constexpr (USE == kStats && !ADD_UP) {
                // the largest first, then everything relative to it; two blocks of columns in turn (half_w is 64 or 128)
                const uint32_t at = tm_row + (uint32_t)(acc * ACC_COLS);
                float u[32], v[32];
                __syncwarp();
                tmem_ld32_start(at, u);
                for (int c0 = 0; c0 < half_w; c0 += 64) {
                    tmem_ld32_wait(u);
                    tmem_ld32_start(at + c0 + 32, v);
                    largest(c0, u);
                    tmem_ld32_wait(v);
                    tmem_ld32_start(at + (c0 + 64 < half_w ? c0 + 64 : 0), u);
                    largest(c0 + 32, v);
                }
                if (plain) m2 = __fmul_ru(m2, a.sc);
                for (int c0 = 0; c0 < half_w; c0 += 64) {
                    tmem_ld32_wait(u);
                    tmem_ld32_start(at + c0 + 32, v);
                    take(c0, u);
                    __syncwarp();
                    tmem_ld32_wait(v);
                    if (c0 + 64 < half_w) tmem_ld32_start(at + c0 + 64, u);
                    take(c0 + 32, v);
                    __syncwarp();
                }
                release();
            } else if constexpr (USE == kOut) {
                for (int c0 = 0; c0 < half_w; c0 += 32) {
                    float v[32];
                    __syncwarp();
                    tmem_ld32(tm_row + (uint32_t)(acc * ACC_COLS + c0), v);
                    take(c0, v);
                }
                release();
            }
            if (USE == kStats && rv) a.stats[(long long)(2 * t.n + half) * a.M + row] = make_float4(m2, s1, s2, dot);
        }
    }

    // Tear-down.  After a time-out, the leader gives loads that may still be in flight, its own and the other CTA's, a bounded chance to land before the shared
    // memory is released.  Neither CTA leaves while the other may still read its operands or arrive at its barriers.
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0 && rank == 0)
        for (int s = 0; s < CT_STAGES; ++s)
            for (uint32_t i = 0; i < 4096u; ++i)
                if (mbar_try_wait(full(s), 0) || mbar_try_wait(full(s), 1)) break;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_dealloc2(tmem_base, CT_TMEM);
    }
}

}  // namespace

}  // namespace gad
