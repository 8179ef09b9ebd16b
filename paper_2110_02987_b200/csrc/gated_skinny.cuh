// The products of the gated feed-forward block for few rows (skinny.cuh).  As the tiles of gated_gemm.cuh have it, 256 rows of x on the other side, a call of 48 rows mostly multiplies zeros and has too few
// tiles to read with.
//   kGate      a tile is up to 64 rows of Wg and the same of Wu: rows 0 .. 63 of the accumulator are g, 64 .. 127 u of the same units
//   kPlain     up to 128 rows of Wd
// Tiles have fewer rows where that deals them out more evenly (8192 units: 147 tiles of 56 instead of 128 of 64), and where there are too few for all SMs the reduction is cut into shares, whose sums
// skinny_join_kernel adds up.  The second product's first weights are loaded before the wait for the first product: they fill the time in which the last tiles in front are drained.
#pragma once

#include "gated_gemm.cuh"
#include "skinny.cuh"

namespace gad {

namespace {

struct SkinnyArgs {
    int rows, width;           // rows of x; rounded up to the instruction's N
    int N;                     // rows of the weights (kGate: of each)
    int per, tiles, nkb, shares, kb_share;   // per: rows of the weights a tile has (kGate: half of them of each), at most 128
    int stages;
    int chunk;                 // ADD_UP: blocks of the reduction that an accumulator has before its sums move to registers
    int early;                 // the weights are the caller's: they may be loaded before the kernel in front has ended
    int bf16, activation, clear;
    int32_t* err;
    void* out; long long ldo;  // h or y, or null: sums to parts
    float* parts;              // [shares x tiles][rows][128]
};

// A unit of work: a share of a tile.
struct SkinnyAt { int tile, kb0, nkb; };
__device__ __forceinline__ SkinnyAt skinny_at(const SkinnyArgs& a, int u) {
    const int share = u / a.tiles;
    SkinnyAt t;
    t.tile = u - share * a.tiles;
    t.kb0 = share * a.kb_share;
    t.nkb = min(a.kb_share, a.nkb - t.kb0);
    return t;
}

// ADD_UP: reductions longer than the tensor core may add up (kGatedChunk), in chunks whose sums the draining threads add up in registers and put back for what follows.
template <int USE, class T, bool ADD_UP>
__global__ void __launch_bounds__(SK_THREADS, 1)
skinny_kernel(const __grid_constant__ CUtensorMap tmW0, const __grid_constant__ CUtensorMap tmW1, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ SkinnyArgs a) {
    extern __shared__ uint8_t smem_raw[];
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
    float* xch = reinterpret_cast<float*>(sm + SK_RING + 512);

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

    const int units = a.tiles * a.shares;
    const uint32_t stage_bytes = SK_A + (uint32_t)a.width * (CT_K * 2), loaded = (uint32_t)(a.per + a.width) * (CT_K * 2);
    if (warp == 0) {
        if (lane == 0) {
            // ---------------- TMA producer ----------------
            const auto load_w = [&](int s, const SkinnyAt& t, int kb) {
                const uint32_t base = sm_addr + s * stage_bytes;
                mbar_expect_tx(full(s), loaded);
                if (USE == kGate) {
                    tma_load_3d(base, &tmW0, kb * CT_K, t.tile * (a.per / 2), 0, full(s));
                    tma_load_3d(base + SK_A / 2, &tmW1, kb * CT_K, t.tile * (a.per / 2), 0, full(s));
                } else {
                    tma_load_3d(base, &tmW0, kb * CT_K, t.tile * a.per, 0, full(s));
                }
            };
            const auto load_x = [&](int s, int kb) { tma_load_3d(sm_addr + s * stage_bytes + SK_A, &tmX, kb * CT_K, 0, 0, full(s)); };
            const SkinnyAt first = skinny_at(a, blockIdx.x);
            const int ahead = a.early ? min(a.stages, first.nkb) : 0;
            for (int i = 0; i < ahead; ++i) load_w(i, first, first.kb0 + i);
            pdl_wait();
            if (a.clear && blockIdx.x == 0) *a.err = 0;
            for (int i = 0; i < ahead; ++i) load_x(i, first.kb0 + i);
            int stage = ahead == a.stages ? 0 : ahead, done = ahead;
            uint32_t phase = ahead == a.stages ? 1u : 0u;
            bool ok = true;
            for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
                const SkinnyAt t = skinny_at(a, u);
                for (int kb = t.kb0 + done; kb < t.kb0 + t.nkb; ++kb) {
                    if (!(ok = mbar_wait(empty(stage), phase ^ 1u, abort_flag, a.err, 51))) break;
                    load_w(stage, t, kb);
                    load_x(stage, kb);
                    if (++stage == a.stages) { stage = 0; phase ^= 1u; }
                }
                done = 0;
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer: the whole warp runs the loop, one elected lane issues ----------------
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        const uint32_t idesc = instr_desc_f16(a.width, SK_M) | (a.bf16 ? (1u << 7) | (1u << 10) : 0u);
        bool ok = true;
        for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
            const int steps = skinny_at(a, u).nkb;
            int left = 0;                                          // stages until this accumulator is full
            for (int i = 0; i < steps; ++i) {
                const bool first = left == 0;
                if (first) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(tempty(acc), acc_phase ^ 1u, abort_flag, a.err, 52)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    left = ADD_UP ? min(a.chunk, steps - i) : steps;
                }
                const uint32_t d = tmem_base + (uint32_t)(acc * 256);
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(stage), phase, abort_flag, a.err, 53)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base = sm_addr + stage * stage_bytes;
                const uint64_t da = smem_desc(base), db = smem_desc(base + SK_A);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < CT_K / 16; ++ks) mma_f16_one(d, da + 2 * ks, db + 2 * ks, idesc, !first || ks != 0 ? 1u : 0u);
                    mma_commit(empty(stage));
                    if (left == 1) mma_commit(tfull(acc));
                }
                __syncwarp();
                if (++stage == a.stages) { stage = 0; phase ^= 1u; }
                if (--left == 0 && ++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else {
        // ---------------- drain: a row of the weights a lane, rows of x along the columns ----------------
        // (rows of the accumulator behind the tile's hold whatever the shared memory held: nothing of them is written)
        const int q = warp & 3, group = (warp - 2) >> 2, half = a.per / 2;
        float* xg = xch + group * 1024;
        float* xu = xg + 512;
        pdl_wait();
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int u = blockIdx.x; u < units; u += gridDim.x) {
            const SkinnyAt t = skinny_at(a, u);
            const uint32_t lanes = tmem_base + ((uint32_t)(q * 32) << 16);
            // all warps go on or none does: they meet at barriers below
            const auto wait_full = [&]() {
                const bool ok = all_drain(mbar_wait(tfull(acc), acc_phase, abort_flag, a.err, 56));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            const auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(tempty(acc));
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            };
            if (!wait_full()) break;
            if constexpr (ADD_UP) {
                constexpr int BLOCKS = SK_MOST_ROWS / (16 * SK_GROUPS);      // of 16 rows of x, a group
                float sum[BLOCKS][16];
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] = 0.f;
                bool ok = true;
                for (int left = t.nkb; ok; left -= a.chunk) {
#pragma unroll
                    for (int c = 0; c < BLOCKS; ++c) {
                        const int c0 = (c * SK_GROUPS + group) * 16;
                        if (c0 >= a.rows) break;
                        float v[16];
                        __syncwarp();
                        tmem_ld16(lanes + (uint32_t)(acc * 256 + c0), v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c][j] += v[j];
                    }
                    if (left <= a.chunk) break;
                    release();
                    ok = wait_full();
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c) {
                    const int c0 = (c * SK_GROUPS + group) * 16;
                    if (c0 < a.rows) tmem_st16(lanes + (uint32_t)(acc * 256 + c0), sum[c]);
                }
                tmem_wait_st();
            }
            const uint32_t at = lanes + (uint32_t)(acc * 256);
            const int local = USE == kGate ? (q & 1) * 32 + lane : q * 32 + lane;
            const int unit_row = USE == kGate ? t.tile * half + local : t.tile * a.per + local;
            const bool valid = local < (USE == kGate ? half : a.per) && unit_row < a.N;
            for (int c0 = group * 16; c0 < a.rows; c0 += SK_GROUPS * 16) {
                float v[16];
                __syncwarp();
                tmem_ld16(at + (uint32_t)c0, v);
                const int n = min(16, a.rows - c0);
                if (a.parts) {
                    float* out = a.parts + ((long long)u * a.rows + c0) * SK_M + q * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j < n) out[j * SK_M] = v[j];
                } else if (USE == kGate) {
                    // the threads that have g take the first eight rows, those that have u the others
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (q < 2) xg[j * 64 + local] = v[8 + j];
                        else xu[j * 64 + local] = v[j];
                    }
                    asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory");
                    const int first = q < 2 ? 0 : 8;
                    T* out = reinterpret_cast<T*>(a.out) + (long long)(c0 + first) * a.ldo + unit_row;
                    float g[8], d[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = q < 2 ? v[j] : xg[j * 64 + local];
                    activations(a.activation, g, d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (first + j < n && valid) *out = from_float<T>(g[j] * (q < 2 ? xu[j * 64 + local] : v[8 + j]));
                        out += a.ldo;
                    }
                    asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory");
                } else {
                    T* out = reinterpret_cast<T*>(a.out) + (long long)c0 * a.ldo + unit_row;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (j < n && valid) *out = from_float<T>(v[j]);
                        out += a.ldo;
                    }
                }
            }
            release();
        }
    }

    // Tear-down: after a time-out loads in flight get a bounded chance to land.
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0)
        for (int s = 0; s < a.stages; ++s)
            for (uint32_t i = 0; i < 4096u; ++i)
                if (mbar_try_wait(full(s), 0) || mbar_try_wait(full(s), 1)) break;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(CT_TMEM));
    }
}

// Sums of shares added up in order: for kGate g and u, and h of them.  A thread a value of h or y.
template <int USE, class T>
__global__ void __launch_bounds__(256) skinny_join_kernel(const __grid_constant__ SkinnyArgs a, void* out, long long ldo) {
    pdl_next();
    pdl_wait();
    const int c = blockIdx.x * 256 + threadIdx.x, n = blockIdx.y;
    if (c >= a.N) return;
    const int per = USE == kGate ? a.per / 2 : a.per;
    const float* p = a.parts + ((long long)(c / per) * a.rows + n) * SK_M + c % per;
    const long long share = (long long)a.tiles * a.rows * SK_M;
    float s = 0.f, v = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.shares; ++k) {
        s += p[k * share];
        if (USE == kGate) v += p[k * share + 64];
    }
    if (USE == kGate) {
        float g, d;
        activation(a.activation, s, g, d);
        s = g * v;
    }
    reinterpret_cast<T*>(out)[n * ldo + c] = from_float<T>(s);
}

}  // namespace

}  // namespace gad
