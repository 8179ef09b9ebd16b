// The matrix products of the gated feed-forward block on tcgen05, by pairs of CTAs, and what is done with a finished tile.  Used by gated.cu for
//   kGate      g = x Wg^T and u = x Wu^T side by side: h = act(g) u, and for a backward pass act(g) and u act'(g)
//   kHidden    dh = dy Wd: dg = dh u act'(g) and du = dh act(g)
//   kPlain     y = h Wd^T;  dx = dg Wg + du Wu;  dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// What bounds it (4096 x 2048 x 5504 bf16): the tensor pipe, 87 % busy in the three products of the backward pass (304 us), and in long runs the card's power; 75 to 83 % in kGate (132 us), whose drain
// writes three tensors; kHidden (84 us, 57 % of at most 95) shares the way to the L2 between operands, factors and results: without loading and storing those 66 us.
//
// The ring, the roles and the tiles are those of the output head's product (class_gemm.cuh): tiles of 256 rows by two CTAs (cta_group::2), 64 values of the reduction a
// stage, two accumulators of 256 columns, eight draining warps.  Of B each CTA of a pair holds half of the columns, so for kGate one CTA loads 128 rows of Wg and the
// other 128 rows of Wu: the accumulator has g in its left half and u, of the same units, in its right one, and no copy of the weights is laid out for it.
// The sum dg Wg + du Wu is one reduction over two segments with a B of its own each; dWg and dWu are one product over two planes of A with an output each; and the products that do not wait for
// one another (dx, both of these, dWd) are one launch, whose tiles are gone through one product behind the other.
#pragma once

#include "class_gemm.cuh"

namespace gad {

namespace {

enum GatedUse { kGate, kHidden, kPlain };
enum Activation { kSilu, kGelu, kRelu, kSigmoid };

struct GatedArgs {
    TileArgs t;                // tiles and shares (M rows of a plane)
    int parts, segs;           // operand parts; segments of the reduction
    int plane_tiles;           // row tiles of a plane
    int a_mn;                  // kAnyMN: A is MN-major
    int a_chunks, b_chunks;    // MN-major: the descriptor has chunks of 64 columns as a dimension (tc_make_chunk_map), so a box holds all that a CTA has of a stage
    int split;                 // kGate, kHidden: sums go to t.slots, whole tiles' too, and what is made of them is the join's
    int activation;
    int clear;                 // the call's first product: its first block sets the status to zero (blocks come up in order, and a wait takes 2^22 polls to run out)
    const float* factor;       // kPlain: of the results, or null
    void *C[2];                // kPlain: result of each plane; kGate with T = float: C[0] is h where it is kept, or null
    long long ldc[2];
    // kGate: h in the operand type, parts `h_part` values apart; act(g) and u act'(g), or null.  kHidden: those two read, dg and du written (C[0], parts and planes h_part apart)
    void *h, *act, *slope;
    long long ldh, h_part, ldact, ldslope;
};

// The products of a launch: one, or up to three.
constexpr int kGroup = 3;
template <int G>
struct GatedGroup {
    CUtensorMap A[G], B0[G], B1[G];
    GatedArgs p[G];
    int n;
    int first[G + 1];          // units of work in front of each, and of all
};
template <int G> __device__ __forceinline__ int product_of(const GatedGroup<G>& gr, int u) { return G > 1 && u >= gr.first[1] ? (u >= gr.first[2] ? 2 : 1) : 0; }
// Which operands are MN-major (the reduction runs over their rows): neither; B; B, and A as its product says (GatedArgs::a_mn).
enum Layout { kBothK, kBMN, kAnyMN };

// exp(-x^2 / 2) for 0 <= x <= 20: what the square and its product with log2(e) / 2 round off is put back.
__device__ __forceinline__ float exp_half_square(float x) {
    const float c = 0.72134752f, c_lo = 9.6298e-9f, q = x * x, a = q * c;
    const float lo = fmaf(q, c, -a) + fmaf(fmaf(x, x, -q), c, q * c_lo), e = exp2_fast(-a);
    return fmaf(e, -0.693147181f * lo, e);
}
// act(x) and act'(x).  The logistic function from exp2 and a reciprocal, each within 2 ulp, of an argument that is rounded: silu is off by 3 units of 2^-24 around 0 and by 16 at -12.9, where it is 3e-5.
// gelu: the normal distribution's tail is half of erfc(z), z = |x| / sqrt 2, by the Chebyshev fit of Press et al., Numerical Recipes ("erfcc"): erfc(z) = t exp(-z^2 + p(t)), t = 1 / (1 + z / 2), within
// 1.2e-7 of itself; in fp32 gelu is within 5.5e-7 of itself from -12.9 to 13.  (erfcf of -x / sqrt 2, whose rounding the square magnifies, is within 1.2e-5, and with it the drain of a tile took 13 us
// longer than relu's.)
__device__ __forceinline__ void activation(int kind, float x, float& a, float& d) {
    if (kind == kRelu) {
        a = x > 0.f || x != x ? x : 0.f;                   // (what is no number stays none)
        d = x > 0.f ? 1.f : 0.f;
    } else if (kind == kGelu) {
        const float y = fminf(fabsf(x), 20.f), t = __fdividef(1.f, fmaf(0.5f * 0.707106781f, y, 1.f)), e = exp_half_square(y);   // (behind 20 the tail is zero; what is no number comes back with x)
        float p = 0.17087277f;
        p = fmaf(p, t, -0.82215223f); p = fmaf(p, t, 1.48851587f); p = fmaf(p, t, -1.13520398f); p = fmaf(p, t, 0.27886807f); p = fmaf(p, t, -0.18628806f);
        p = fmaf(p, t, 0.09678418f); p = fmaf(p, t, 0.37409196f); p = fmaf(p, t, 1.00002368f); p = fmaf(p, t, -1.26551223f);
        const float tail = 0.5f * t * (e * exp2_fast(1.44269504f * p)), cdf = x < 0.f ? tail : 1.f - tail;
        a = x * cdf;
        d = fmaf(x, 0.398942280f * e, cdf);
    } else {
        const float e = exp2_fast(-1.44269504f * x), s = __fdividef(1.f, 1.f + e);
        const float r = e == INFINITY ? 1.f : e * s;           // 1 - s
        if (kind == kSigmoid) { a = s; d = s * r; }
        else {
            a = x * s;
            d = s * fmaf(x, r, 1.f);
        }
    }
}

// The same of N values, g becomes act(g), with the kind looked at once: value by value the steps of one wait for one another.  (One way through for calls that keep the slope and calls that
// do not: with code for each gelu took longer.)  4096 x 2048 x 5504 bf16, all kept: relu 187 us, silu and sigmoid 190, gelu 204.
template <int KIND, int N>
__device__ __forceinline__ void activations_of(float (&g)[N], float (&d)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float a;
        activation(KIND, g[j], a, d[j]);
        g[j] = a;
    }
}
template <int N>
__device__ __forceinline__ void activations(int kind, float (&g)[N], float (&d)[N]) {
    if (kind == kSilu) activations_of<kSilu>(g, d);
    else if (kind == kGelu) activations_of<kGelu>(g, d);
    else if (kind == kRelu) activations_of<kRelu>(g, d);
    else activations_of<kSigmoid>(g, d);
}

// 32 rows x 32 columns of a matrix on their way to the threads that have a row each: loaded as they lie, 64 bytes of eight rows at a time (a row a thread, the loads of a warp touched 32
// lines each), and turned through the warp's staging buffer when they are wanted.  Zeros behind the matrix.  wide: every row starts on 16 bytes.
template <class T> struct Block32 { uint4 u[2 * sizeof(T)]; };
template <class T>
__device__ __forceinline__ void load_block32(const T* __restrict__ src, long long ld, int rows, int cols, bool wide, int lane, Block32<T>& b) {
    constexpr int VEC = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
        const int r = (i & 3) * 8 + (lane >> 2), c = (i >> 2) * (4 * VEC) + (lane & 3) * VEC;
        const T* at = src + r * ld + c;
        if (wide && r < rows && c + VEC <= cols) b.u[i] = *reinterpret_cast<const uint4*>(at);
        else {
            union { uint4 u; T e[VEC]; } w;
#pragma unroll
            for (int j = 0; j < VEC; ++j) w.e[j] = r < rows && c + j < cols ? at[j] : from_float<T>(0.f);
            b.u[i] = w.u;
        }
    }
}
template <class T>
__device__ __forceinline__ void take_block32(uint8_t* buf, int lane, const Block32<T>& b, float (&v)[32]) {
    constexpr int VEC = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(staged(buf, i * 8 + (lane >> 2), lane & 3)) = b.u[4 * h + i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float w[VEC];
            unpack_vec<T, VEC>(*reinterpret_cast<const uint4*>(staged(buf, lane, i)), w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[(h * 4 + i) * VEC + j] = w[j];
        }
    }
}

// A lane's 32 values as operands: in the operand type, or (T = float) in three bfloat16 parts, each the nearest to what is left.
template <class T>
__device__ __forceinline__ void drain_operand(uint8_t* buf, int lane, float (&v)[32], void* out, long long at, long long part, long long ld, int rows, int cols) {
    if constexpr (sizeof(T) == 4) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) top = fmaxf(top, fabsf(v[j]));
        const bool large = top > 3.38e38f;                 // (a finite value that would round to infinity stays finite)
#pragma unroll 1
        for (int k = 0; k < 3; ++k) {
            uint32_t w[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                w[j] = Pair<__nv_bfloat16>::pack(v[2 * j], v[2 * j + 1]);
                if (large) {
                    if ((w[j] & 0x7FFFu) == 0x7F80u && !isinf(v[2 * j])) --w[j];
                    if ((w[j] & 0x7FFF0000u) == 0x7F800000u && !isinf(v[2 * j + 1])) w[j] -= 0x10000u;
                }
                const float2 f = Pair<__nv_bfloat16>::unpack(w[j]);
                v[2 * j] -= f.x;
                v[2 * j + 1] -= f.y;
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(staged(buf, lane, j)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
            __syncwarp();
            copy_out<16, __nv_bfloat16, false>(buf, lane, reinterpret_cast<__nv_bfloat16*>(out) + k * part + at, ld, rows, cols);
        }
    } else {
        drain_rows<T>(buf, lane, v, reinterpret_cast<T*>(out) + at, ld, rows, cols, 16);
    }
}

// USE as above; T: type of the tensors; ADD_UP: sums in chunks (t.chunk; of operands in parts, of one block of 64 terms each), as class_gemm_kernel takes them; G: products a launch may have.  (With the layouts of all products and their number known only
// at run time, in one kernel for all uses, 8192 x 2048 x 5504 took 428 us instead of 416, and the gradients of 16 384 x 4096 x 10 240 6.2 ms instead of 5.8.)
template <int USE, int LAYOUT, class T, bool ADD_UP, int G>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(CT_THREADS, 1)
gated_gemm_kernel(const __grid_constant__ GatedGroup<G> gr) {
    constexpr bool B_MN = LAYOUT != kBothK, PARTS = sizeof(T) == 4;   // PARTS: operands in three parts
    int32_t* const err = gr.p[0].t.err;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;   // the same in both CTAs
    uint8_t* sm = smem_raw + pad;
    const uint32_t sm_addr = raw_addr + pad;
    const uint32_t rank = cluster_rank();
    const uint32_t bars = sm_addr + CT_RING;
    constexpr int NACC = 2, ACC_COLS = CT_TMEM / NACC;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (CT_STAGES + s); };
    auto tfull = [&](int i) { return bars + 8u * (2 * CT_STAGES + i); };
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
    if (gr.p[0].clear && blockIdx.x == 0 && threadIdx.x == 0) *err = 0;

    const int ncl = gridDim.x >> 1, units = gr.first[G];

    if ((warp == 0 || warp == CT_LOADER_B) && lane == 0) {
        // ---------------- TMA producers, one for each operand: this CTA's rows of A, and half of the columns' rows of B; the leader's barrier counts both CTAs' bytes.  (One thread for
        // both was the bound of MN-major operands, whose stage has two boxes of 64 columns each: dx, dWg and dWu, dWd of 4096 x 2048 x 5504 in 325 us, with these 300.) ----------------
        const auto produce = [&](auto of_a) {
            constexpr bool OF_A = decltype(of_a)::value;
            const uint32_t leader = leader_address(full(0));
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int u = blockIdx.x >> 1; u < units && ok; u += ncl) {
                const int which = product_of(gr, u);
                const GatedArgs& ga = gr.p[which];
                const TileArgs& a = ga.t;
                const int half_w = a.width / 2;
                const bool mn = OF_A ? LAYOUT == kAnyMN && ga.a_mn : B_MN, chunks = OF_A ? ga.a_chunks : ga.b_chunks;
                const uint32_t bytes = 2u * (uint32_t)(CT_H + half_w) * (CT_K * 2);
                const TileAt t = tile_at(a, u - gr.first[which]);
                const int plane = t.m / ga.plane_tiles;
                // first row of the operand's share
                const int r = OF_A ? (t.m - plane * ga.plane_tiles) * CT_M + (int)rank * CT_H : USE == kGate ? t.n * half_w : t.n * a.width + (int)rank * half_w;
                const bool two = mn && !chunks && (OF_A || half_w > 64);      // two boxes of 64 columns a stage
                const auto load = [&](const CUtensorMap* map, int kb, int z) {
                    if (!(ok = mbar_wait(empty(stage), phase ^ 1u, abort_flag, err, OF_A ? 41 : 44))) return;
                    if (OF_A && rank == 0) mbar_expect_tx(full(stage), bytes);
                    const uint32_t to = sm_addr + stage * CT_STAGE + (OF_A ? 0 : CT_OPERAND), bar = leader + 8u * stage;
                    if (!mn) tma_load_3d_pair(to, map, kb * CT_K, r, z, bar);
                    else if (chunks) tma_load_4d_pair(to, map, kb * CT_K, r >> 6, z, bar);
                    else {
                        tma_load_3d_pair(to, map, r, kb * CT_K, z, bar);
                        if (two) tma_load_3d_pair(to + 8192, map, r + 64, kb * CT_K, z, bar);
                    }
                    if (++stage == CT_STAGES) { stage = 0; phase ^= 1u; }
                };
                const int group = ADD_UP && !PARTS ? a.chunk : t.nkb;
                for (int g = 0; g < t.nkb && ok; g += group)
                    for (int seg = 0; seg < ga.segs && ok; ++seg) {
                        const CUtensorMap* map = OF_A ? &gr.A[which] : (USE == kGate ? (int)rank : seg) ? &gr.B1[which] : &gr.B0[which];
                        const int last = t.kb0 + min(g + group, t.nkb), z = OF_A ? plane + seg : 0;
                        for (int kb = t.kb0 + g; kb < last && ok; ++kb) {
                            if constexpr (PARTS) {
                                // all parts of a block of the reduction, in the order in which the products let go of them
                                for (int p = 2; p >= 0 && ok; --p) load(map, kb, 3 * z + p);
                            } else load(map, kb, z);
                        }
                    }
            }
        };
        if (warp == 0) produce(std::true_type());
        else produce(std::false_type());
    } else if (warp == 1 && rank == 0) {
        // ---------------- MMA issuer (leader of the pair): the whole warp runs the loop, one elected lane issues ----------------
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (int u = blockIdx.x >> 1; u < units && ok; u += ncl) {
            const int which = product_of(gr, u);
            const GatedArgs& ga = gr.p[which];
            const TileArgs& a = ga.t;
            const bool a_mn = LAYOUT == kAnyMN && ga.a_mn;
            const uint32_t idesc = instr_desc_f16(a.width, CT_M) | (a.bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_mn ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
            const uint32_t stepA = a_mn ? 128 : 2;
            constexpr uint32_t stepB = B_MN ? 128 : 2;                        // 16 values of the reduction: 16 rows of 128 bytes, or 32 bytes of a row
            const uint64_t descA = a_mn ? operand_desc<true>(0) : operand_desc<false>(0);
            const int steps = tile_at(a, u - gr.first[which]).nkb * ga.segs, chunk = a.chunk * ga.segs;
            if constexpr (PARTS) {
                // the six products of the parts that reach 2^-24, the smallest first, in an accumulator of each block's own: what an addition cuts off is little, as the accumulator is small for
                // most of them, and each part comes from the L2 once.  (A stage a product, with each part loaded two or three times, was bound by the L2: 4345 x 4005 x 632 460 us, now 401.)
                for (int i = 0; i < steps; ++i) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(tempty(acc), acc_phase ^ 1u, abort_flag, err, 42)))) break;
                    uint32_t base[3], bar[3];
                    for (int p = 2; p >= 0 && ok; --p) {
                        ok = __all_sync(0xffffffffu, mbar_wait<true>(full(stage), phase, abort_flag, err, 43));
                        base[p] = sm_addr + stage * CT_STAGE;
                        bar[p] = empty(stage);
                        if (++stage == CT_STAGES) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem_base + (uint32_t)(acc * ACC_COLS);
                    if (elect_one()) {
                        const auto multiply = [&](int pa, int pb, bool first) {
                            const uint64_t da = descA | (base[pa] >> 4), db = operand_desc<B_MN>(base[pb] + CT_OPERAND);
#pragma unroll
                            for (int ks = 0; ks < CT_K / 16; ++ks) mma_f16_pair(d, da + stepA * ks, db + stepB * ks, idesc, !first || ks != 0 ? 1u : 0u);
                        };
                        multiply(0, 2, true);
                        multiply(2, 0, false);
                        mma_commit2(bar[2]);
                        multiply(1, 1, false);
                        multiply(0, 1, false);
                        multiply(1, 0, false);
                        mma_commit2(bar[1]);
                        multiply(0, 0, false);
                        mma_commit2(bar[0]);
                        mma_commit2(tfull(acc));
                    }
                    __syncwarp();
                    if (++acc == NACC) { acc = 0; acc_phase ^= 1u; }
                }
                continue;
            }
            int left = 0;                                          // stages until this accumulator is full
            for (int i = 0; i < steps; ++i) {
                const bool first = left == 0;
                if (first) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(tempty(acc), acc_phase ^ 1u, abort_flag, err, 42)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    left = ADD_UP ? min(chunk, steps - i) : steps;
                }
                const uint32_t d = tmem_base + (uint32_t)(acc * ACC_COLS);
                if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(full(stage), phase, abort_flag, err, 43)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base = sm_addr + stage * CT_STAGE;
                const uint64_t da = descA | (base >> 4), db = operand_desc<B_MN>(base + CT_OPERAND);
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
    } else if (warp >= CT_EPI_WARP0 && warp < CT_LOADER_B) {   // (warp 1 of the other CTA has nothing to do)
        // ---------------- drain: this warp's 32 rows (a row a lane) x half of the tile's columns (kGate: half of g and of u) ----------------
        const int ew = warp - CT_EPI_WARP0, q = warp & 3, half = ew >> 2;
        uint8_t* buf = sm + CT_RING + 256 + CT_BIAS + ew * 2048;
        int acc = 0;
        uint32_t acc_phase = 0;
        const auto store = [](const void* p, long long ld) { return store_bytes(p, ld * (long long)sizeof(T)); };
        for (int u = blockIdx.x >> 1; u < units; u += ncl) {
            const int which = product_of(gr, u);
            const GatedArgs& ga = gr.p[which];
            const TileArgs& a = ga.t;
            const int half_w = a.width / 2;
            const TileAt t = tile_at(a, u - gr.first[which]);
            const int plane = t.m / ga.plane_tiles, tm = t.m - plane * ga.plane_tiles;
            const int row0 = tm * CT_M + (int)rank * CT_H + q * 32, rows = a.M - row0;   // this warp's rows
            const uint32_t tm_row = tmem_base + ((uint32_t)(q * 32) << 16);
            const auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_leader_tmem(tempty(acc));
                if (++acc == NACC) { acc = 0; acc_phase ^= 1u; }
            };
            // kHidden: the factors of 32 columns are on their way before the product is waited for
            Block32<T> slope, act;
            const auto load_factors = [&](int col) {
                load_block32<T>(reinterpret_cast<const T*>(ga.slope) + (long long)row0 * ga.ldslope + col, ga.ldslope, rows, a.N - col, store(ga.slope, ga.ldslope) == 16, lane, slope);
                load_block32<T>(reinterpret_cast<const T*>(ga.act) + (long long)row0 * ga.ldact + col, ga.ldact, rows, a.N - col, store(ga.act, ga.ldact) == 16, lane, act);
            };
            if (USE == kHidden && !ADD_UP) load_factors(t.n * a.width + half * half_w);   // (the sums of chunks leave no registers for them: those forms spill 0.6 KB a thread as it is, in fp32 1.2)
            bool ok = true;
            const auto wait_full = [&]() {
                ok = __all_sync(0xffffffffu, mbar_wait(tfull(acc), acc_phase, abort_flag, err, 46));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            // this warp's columns of the accumulator: blocks of 32, for kGate one or two of g and the same of u behind them
            const int blocks = half_w / 32, of_g = blocks / 2;
            const auto block_at = [&](int c) { return USE != kGate ? half * half_w + 32 * c : c < of_g ? half * (half_w / 2) + 32 * c : half_w + half * (half_w / 2) + 32 * (c - of_g); };
            if constexpr (ADD_UP) {
                const int chunks = PARTS ? t.nkb * ga.segs : (t.nkb + a.chunk - 1) / a.chunk;
                float sum[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[c][j] = 0.f;
                for (int i = 0; i < chunks; ++i) {
                    if (!wait_full()) break;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c >= blocks) break;
                        float v[32];
                        tmem_ld32(tm_row + (uint32_t)(acc * ACC_COLS + block_at(c)), v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[c][j] += v[j];
                    }
                    if (i < chunks - 1) release();
                }
                if (!ok) break;
                // the sums take the place of the last chunk, and are taken from there block by block: held in registers beside what follows they would spill
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c < blocks) tmem_st_32x32b_x32(tm_row + (uint32_t)(acc * ACC_COLS + block_at(c)), sum[c]);
                tmem_wait_st();
            } else if (!wait_full()) break;
            const uint32_t at = tm_row + (uint32_t)(acc * ACC_COLS);
            const int slot = USE != kPlain && ga.split && t.slot < 0 ? u - gr.first[which] : t.slot;
            if (slot >= 0) {
                // (this warp's own blocks: those of the other half may not have been put back yet)
                for (int c = 0; c < blocks; ++c) {
                    if (rows <= 0) break;
                    float v[32];
                    __syncwarp();
                    tmem_ld32(at + (uint32_t)block_at(c), v);
                    drain_rows<float>(buf, lane, v, a.slots + (long long)slot * CT_M * a.width + (long long)((int)rank * CT_H + q * 32) * a.width + block_at(c), a.width, 32, 32, 16);
                }
                release();
            } else if constexpr (USE == kGate) {
                for (int c = 0; c < of_g; ++c) {
                    const int col = t.n * half_w + half * (half_w / 2) + 32 * c, cols = a.N - col;
                    if (rows <= 0 || cols <= 0) break;
                    float g[32], v[32];
                    __syncwarp();
                    tmem_ld32_start(at + (uint32_t)block_at(c), g);
                    tmem_ld32_start(at + (uint32_t)block_at(c + of_g), v);
                    tmem_ld32_wait(g);
                    tmem_ld32_wait(v);
                    float d[32];
                    activations(ga.activation, g, d);
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        d[j] *= v[j];
                        v[j] *= g[j];
                    }
                    if (ga.act) {
                        drain_rows<T>(buf, lane, d, reinterpret_cast<T*>(ga.slope) + (long long)row0 * ga.ldslope + col, ga.ldslope, rows, cols, store(ga.slope, ga.ldslope));
                        drain_rows<T>(buf, lane, g, reinterpret_cast<T*>(ga.act) + (long long)row0 * ga.ldact + col, ga.ldact, rows, cols, store(ga.act, ga.ldact));
                        if (sizeof(T) == 4) drain_rows<T>(buf, lane, v, reinterpret_cast<T*>(ga.C[0]) + (long long)row0 * ga.ldc[0] + col, ga.ldc[0], rows, cols, store(ga.C[0], ga.ldc[0]));
                    }
                    drain_operand<T>(buf, lane, v, ga.h, (long long)row0 * ga.ldh + col, ga.h_part, ga.ldh, rows, cols);
                }
                release();
            } else if constexpr (USE == kHidden) {
                for (int c0 = 0; c0 < half_w; c0 += 32) {
                    const int col = t.n * a.width + half * half_w + c0, cols = a.N - col;
                    if (rows <= 0 || cols <= 0) break;
                    if (ADD_UP && c0 == 0) load_factors(col);
                    float dh[32], v[32];
                    __syncwarp();
                    tmem_ld32(at + (uint32_t)(half * half_w + c0), dh);
                    take_block32<T>(buf, lane, slope, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= dh[j];
                    drain_operand<T>(buf, lane, v, ga.C[0], (long long)row0 * ga.ldh + col, ga.h_part, ga.ldh, rows, cols);
                    take_block32<T>(buf, lane, act, v);
                    if (c0 + 32 < half_w) load_factors(col + 32);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= dh[j];
                    drain_operand<T>(buf, lane, v, ga.C[0], (long long)ga.parts * ga.h_part + (long long)row0 * ga.ldh + col, ga.h_part, ga.ldh, rows, cols);
                }
                release();
            } else {
                for (int c0 = 0; c0 < half_w; c0 += 32) {
                    const int col = t.n * a.width + half * half_w + c0, cols = a.N - col;
                    if (rows <= 0 || cols <= 0) break;
                    float v[32];
                    __syncwarp();
                    tmem_ld32(at + (uint32_t)(half * half_w + c0), v);
                    if (ga.factor) {
                        const float f = *ga.factor;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= f;
                    }
                    drain_rows<T>(buf, lane, v, reinterpret_cast<T*>(ga.C[plane]) + (long long)row0 * ga.ldc[plane] + col, ga.ldc[plane], rows, cols, store(ga.C[plane], ga.ldc[plane]));
                }
                release();
            }
        }
    }

    // Tear-down, as in class_gemm_kernel: after a time-out loads in flight get a bounded chance to land; neither CTA leaves while the other may still read its operands or arrive at its barriers.
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
