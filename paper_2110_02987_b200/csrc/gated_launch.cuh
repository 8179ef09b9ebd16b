// Products of gated_gemm.cuh on the host: their sizes, how their tiles are cut, descriptors, launches.  For gated.cu, and for the fp32 gradients of the policy loss in class_loss.cu.
#pragma once

#include <algorithm>
#include <atomic>

#include "gated_gemm.cuh"

namespace gad {

namespace {

constexpr int kPairs = 74;                               // pairs of CTAs that run at once

// The shares of the tiles that were cut along their reduction, added up in order: four columns a thread, 1024 values a block.  first: blocks in front of each product's, and of all.
struct JoinArgs { GatedArgs p[kGroup]; int first[kGroup + 1]; };
template <class T>
__global__ void __launch_bounds__(256) gated_join_kernel(const __grid_constant__ JoinArgs j) {
    const int which = (int)blockIdx.x >= j.first[1] ? (int)blockIdx.x >= j.first[2] ? 2 : 1 : 0;
    const GatedArgs& ga = j.p[which];
    const TileArgs& a = ga.t;
    const int b = blockIdx.x - j.first[which];
    const int per_row = a.width / 4, rows = 256 / per_row, per_tile = CT_M / rows;
    const int i = b / per_tile, r = b % per_tile * rows + threadIdx.x / per_row, x = threadIdx.x % per_row * 4;
    pdl_next();
    pdl_wait();
    const TileAt t = tile_at(a, a.whole + (long long)i * a.shares);
    const int plane = t.m / ga.plane_tiles, row = (t.m - plane * ga.plane_tiles) * CT_M + r, c = t.n * a.width + x;
    if (row >= a.M || c >= a.N) return;
    const float* slot = a.slots + ((long long)i * a.shares * CT_M + r) * a.width + x;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < a.shares; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(slot + (long long)k * CT_M * a.width);
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
    }
    const float f = ga.factor ? *ga.factor : 1.f;
    T* out = reinterpret_cast<T*>(ga.C[plane]) + (long long)row * ga.ldc[plane] + c;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < a.N) out[k] = from_float<T>(f * s[k]);
}

// Four values as operands, at most `cols` of them: in the operand type, or in three bfloat16 parts.
template <class T>
__device__ __forceinline__ void store_operand4(const float (&v)[4], void* out, long long at, long long part, int cols) {
    if constexpr (sizeof(T) == 4) {
        union { uint2 u; __nv_bfloat16 h[4]; } w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            __nv_bfloat16 p[3];
            split3(v[j], p);
            for (int k = 0; k < 3; ++k) w[k].h[j] = p[k];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(out) + k * part + at;
            if (cols >= 4) *reinterpret_cast<uint2*>(to) = w[k].u;
            else for (int j = 0; j < cols; ++j) to[j] = w[k].h[j];
        }
    } else {
        T* to = reinterpret_cast<T*>(out) + at;
        if (cols >= 4) *reinterpret_cast<uint2*>(to) = make_uint2(Pair<T>::pack(v[0], v[1]), Pair<T>::pack(v[2], v[3]));
        else for (int j = 0; j < cols; ++j) to[j] = from_float<T>(v[j]);
    }
}
// The sums of kGate and kHidden that went to slots, joined, and what those kernels make of a tile: four columns of a row a thread, all of the GPU at once.  With fewer tiles than pairs of CTAs a
// tile's drain has nothing to hide behind, and in fp32 (three parts of h, dg and du each) it takes as long as 60 to 100 stages of the reduction.
template <int USE, class T>
__global__ void __launch_bounds__(256) gated_hidden_join_kernel(const __grid_constant__ GatedArgs ga) {
    const TileArgs& a = ga.t;
    const int wide = USE == kGate ? a.width / 2 : a.width;            // columns of h (dg, du) a tile has
    const int per_row = wide / 4, rows = 256 / per_row, per_tile = CT_M / rows;
    const int i = blockIdx.x / per_tile, r = blockIdx.x % per_tile * rows + threadIdx.x / per_row, x = threadIdx.x % per_row * 4;
    pdl_next();
    pdl_wait();
    const TileAt t = tile_at(a, (long long)i * a.shares);             // (all tiles are cut, or none)
    const int row = t.m * CT_M + r, c = t.n * wide + x, cols = a.N - c;
    if (row >= a.M || cols <= 0) return;
    const float* slot = a.slots + ((long long)i * a.shares * CT_M + r) * a.width + x;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int k = 0; k < a.shares; ++k) {
        const float4 p = *reinterpret_cast<const float4*>(slot + (long long)k * CT_M * a.width);
        s[0] += p.x; s[1] += p.y; s[2] += p.z; s[3] += p.w;
        if (USE == kGate) {
            const float4 q = *reinterpret_cast<const float4*>(slot + (long long)k * CT_M * a.width + wide);
            v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
        }
    }
    if (USE == kGate) {
        float d[4];
        activations(ga.activation, s, d);
#pragma unroll
        for (int j = 0; j < 4; ++j) { d[j] *= v[j]; v[j] *= s[j]; }
        if (ga.act) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >= cols) break;
                reinterpret_cast<T*>(ga.act)[(long long)row * ga.ldact + c + j] = from_float<T>(s[j]);
                reinterpret_cast<T*>(ga.slope)[(long long)row * ga.ldslope + c + j] = from_float<T>(d[j]);
                if (sizeof(T) == 4) reinterpret_cast<T*>(ga.C[0])[(long long)row * ga.ldc[0] + c + j] = from_float<T>(v[j]);
            }
        }
        store_operand4<T>(v, ga.h, (long long)row * ga.ldh + c, ga.h_part, cols);
    } else {
        const T *act = reinterpret_cast<const T*>(ga.act) + (long long)row * ga.ldact + c, *slope = reinterpret_cast<const T*>(ga.slope) + (long long)row * ga.ldslope + c;
        float g[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] = j < cols ? s[j] * to_float(slope[j]) : 0.f;
            v[j] = j < cols ? s[j] * to_float(act[j]) : 0.f;
        }
        store_operand4<T>(g, ga.C[0], (long long)row * ga.ldh + c, ga.h_part, cols);
        store_operand4<T>(v, ga.C[0], (long long)ga.parts * ga.h_part + (long long)row * ga.ldh + c, ga.h_part, cols);
    }
}

// The kernels of a call: the first waits for all that is in front of it on the stream, the others for the one in front; the first product clears the status.
struct Sequence {
    cudaStream_t s;
    bool first = true, clear = true;
    template <class... P, class... Args>
    cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, Args&&... args) {
        const bool f = first;
        first = false;
        return chain(kernel, grid, block, smem, s, f, std::forward<Args>(args)...);
    }
};

// Blocks of 64 terms that the tensor core adds up before the sum moves to registers: it cuts its accumulator off at every addition, 2^-23 of the sum every 16 terms at most (see
// class_gemm_kernel).  As for the head's gradients, as many as cost an eighth of the results' rounding at most.  (fp32: one.)
template <class T> constexpr int kGatedChunk = 1;
template <> constexpr int kGatedChunk<__half> = 128;
template <> constexpr int kGatedChunk<__nv_bfloat16> = 1024;

// ---- sizes of products, and how their tiles are cut: the same for the workspace and the launches ----

// One product: planes of M x N over K, in segs segments and pairs products of parts.
struct Shape { int64_t M; int N; int64_t K; int planes, segs; };
struct Cut {
    int width, tiles_m, tiles_n, nkb, whole, shares, kb_share;
    bool split;                        // kGate, kHidden: all sums to slots
    int64_t tiles() const { return (int64_t)tiles_m * tiles_n; }
};

// Tiles are 256 columns wide; narrow: 128, which take about three quarters of the time (their operands come from L2 half as fast again).
Cut whole_tiles(const Shape& s, bool narrow) {
    Cut c{};
    c.width = narrow || s.N <= 128 ? 128 : 256;
    c.tiles_m = s.planes * (int)((s.M + CT_M - 1) / CT_M);
    c.tiles_n = (s.N + c.width - 1) / c.width;
    c.nkb = (int)((s.K + CT_K - 1) / CT_K);
    c.shares = 1;
    c.kb_share = c.nkb;
    c.whole = (int)c.tiles();
    return c;
}
// Products whose results go as they are.  With three rounds of tiles and more, tiles that take long are cut along their reduction where the pair of CTAs with most work finishes sooner so (pairs take units
// in turn: the 16 tiles of dx of 64 x 4096 x 11 000, 344 stages each, would be 16 pairs' alone: 226 us, cut 150; a unit that is cut costs about ten stages more, and its sums' way through the L2), and those of the last product that are left over when all pairs have had the same number are cut along their
// reduction, down to 8 ring stages a share; with fewer, every tile is cut into shares of about the same number of stages, the number that lets the pair with most work finish first.
constexpr int kMostUnits = 4 * kPairs;                    // of a launch whose tiles are cut
double cut_group(const Shape* s, int n, int pairs, Cut* c) {
    const auto stages = [&](int i, int kb) { return (int64_t)kb * pairs * s[i].segs; };
    int64_t tiles = 0, units = 0;
    for (int i = 0; i < n; ++i) {
        c[i] = whole_tiles(s[i], false);
        tiles += c[i].tiles();
        units += c[i].tiles() * std::max<int64_t>(1, stages(i, c[i].nkb) / 8);
    }
    if (units < kPairs) {                                 // not even cut are there enough
        tiles = 0;
        for (int i = 0; i < n; ++i) { c[i] = whole_tiles(s[i], true); tiles += c[i].tiles(); }
    }
    const auto share = [&](int i, int want) {
        c[i].kb_share = (c[i].nkb + want - 1) / want;
        c[i].shares = (c[i].nkb + c[i].kb_share - 1) / c[i].kb_share;
    };
    if (tiles >= 3 * kPairs) {
        int64_t all = 0;
        for (int i = 0; i < n; ++i) all += c[i].tiles() * stages(i, c[i].nkb);
        const auto share_over = [&](int64_t most) {        // tiles of more than so many stages
            for (int i = 0; i < n; ++i) {
                const int64_t one = stages(i, c[i].nkb);
                share(i, most && one > most ? (int)std::min((one + most - 1) / most, std::max<int64_t>(1, one / 8)) : 1);
            }
        };
        double least = 1e30;
        int64_t best = 0;
        for (int k = 0; k < 5; ++k) {
            const int64_t most = k ? std::max<int64_t>(8, (all / kPairs) >> (k - 1)) : 0;
            share_over(most);
            int64_t load[kPairs] = {}, at = 0, cut = 0;
            for (int i = 0; i < n; ++i) {
                // the pairs' turns go on from one product to the next
                const int64_t units = c[i].tiles() * c[i].shares, one = stages(i, c[i].kb_share) + (c[i].shares > 1 ? 10 : 2);
                for (int x = 0; x < kPairs; ++x) load[(at + x) % kPairs] += (units / kPairs + (x < units % kPairs)) * one;
                at = (at + units) % kPairs;
                if (c[i].shares > 1) cut += units;
            }
            const double cost = (double)*std::max_element(load, load + kPairs) + (cut ? 15 + 0.3 * (double)cut : 0.0);
            if (cost < 0.97 * least) { least = cost; best = most; }
        }
        share_over(best);
        for (int i = 0; i < n; ++i)
            if (c[i].shares > 1) c[i].whole = 0;
        const int i = n - 1;
        const int64_t rest = std::min<int64_t>(tiles % kPairs, c[i].tiles());
        if (!rest || c[i].shares > 1) return 0.0;
        const int want = (int)std::min<int64_t>(kPairs / rest, stages(i, c[i].nkb) / 8);
        if (want < 2) return 0.0;
        share(i, want);
        if (c[i].shares > 1) c[i].whole = (int)(c[i].tiles() - rest);
        return 0.0;
    }
    int64_t longest = 0;
    for (int i = 0; i < n; ++i) longest = std::max(longest, stages(i, c[i].nkb));
    const auto share_all = [&](int64_t most) {             // units of at most so many stages; their number
        int64_t units = 0;
        for (int i = 0; i < n; ++i) {
            share(i, (int)std::max<int64_t>(1, std::min<int64_t>((stages(i, c[i].nkb) + most - 1) / most, stages(i, c[i].nkb) / 8)));
            units += c[i].tiles() * c[i].shares;
        }
        return units;
    };
    double least = 1e30;
    int64_t best = longest;
    for (int64_t most = longest; most >= 8; most = most * 3 / 4) {
        if (share_all(most) > kMostUnits) break;
        int load[kPairs] = {}, at = 0, top = 0;
        for (int i = 0; i < n; ++i)
            for (int64_t k = 0; k < c[i].tiles(); ++k)
                for (int x = 0; x < c[i].shares; ++x) {
                    load[at] += (int)stages(i, std::min(c[i].kb_share, c[i].nkb - x * c[i].kb_share)) + 4;
                    top = std::max(top, load[at]);
                    if (++at == kPairs) at = 0;
                }
        const double cost = top + (most < longest ? 12 : 0);
        if (cost < least) { least = cost; best = most; }
    }
    share_all(best);
    for (int i = 0; i < n; ++i)
        if (c[i].shares > 1) c[i].whole = 0;
    return least;
}
int64_t slot_bytes(const Cut& c) { return c.split ? c.tiles() * c.shares * CT_M * c.width * 4 : (c.tiles() - c.whole) * (c.shares > 1 ? c.shares : 0) * CT_M * c.width * 4; }

// kGate and kHidden: what is made of a finished tile is not additive, so tiles are whole and drained where they lie (`drain`: that of the last tile, in stages), or all sums go
// to slots, of shares of the reduction where that helps, for a kernel that makes h (dg and du) of them: with few tiles.  Narrow tiles where their rounds are shorter all the same (22 wide tiles on
// 74 pairs: 44 narrow ones).
Cut cut_hidden(const Shape& s, int pairs, int drain) {
    const Cut wide = whole_tiles(s, false), narrow = whole_tiles(s, true);
    const auto rounds = [](const Cut& c) { return (double)((c.tiles() + kPairs - 1) / kPairs); };
    const bool is_narrow = 0.75 * rounds(narrow) < rounds(wide) && wide.tiles() < 8 * kPairs;
    Cut best = is_narrow ? narrow : wide;
    if (wide.tiles() > 2 * kPairs) return best;
    const double stages = (double)best.nkb * pairs, factor = is_narrow ? 0.75 : 1.0;
    const double here = rounds(best) * factor * std::max(stages, (double)drain) + factor * drain;
    Cut cut;
    const double there = cut_group(&s, 1, pairs, &cut) + 16;
    if (there >= here) return best;
    cut.whole = cut.shares > 1 ? 0 : cut.whole;
    cut.split = true;
    return cut;
}

// The same for an operand whose columns are what the result has rows or columns of (the reduction runs over its rows), `box` of them a CTA and stage: with chunks of 64 columns as a dimension
// where rows have whole chunks.
cudaError_t map_mn(CUtensorMap& m, const void* base, int64_t ld, int64_t rows, int cols, int planes, int box, int& chunks) {
    chunks = cols % 64 == 0;
    const bool ok = chunks ? tc_make_chunk_map(&m, base, (uint64_t)cols / 64, (uint64_t)rows, (uint64_t)planes, (uint64_t)ld * 2, (uint64_t)(ld * 2 * rows), (uint32_t)box / 64)
                           : tc_make_map(&m, base, (uint64_t)cols, (uint64_t)rows, (uint64_t)planes, (uint64_t)ld * 2, (uint64_t)(ld * 2 * rows), CT_K, false, true);
    return ok ? cudaSuccess : cudaErrorInvalidValue;
}
GatedArgs product(const Shape& s, const Cut& c, int dtype, bool a_mn, int group, int32_t* status) {
    GatedArgs g{};
    g.parts = dtype == GAD_F32 ? 3 : 1;
    g.segs = s.segs;
    g.a_mn = a_mn;
    g.split = c.split;
    g.plane_tiles = (int)((s.M + CT_M - 1) / CT_M);
    g.t.M = (int)s.M; g.t.N = s.N;
    g.t.tiles_m = c.tiles_m; g.t.tiles_n = c.tiles_n; g.t.width = c.width;
    g.t.nkb = c.nkb; g.t.whole = c.whole; g.t.shares = c.shares; g.t.kb_share = c.kb_share;
    g.t.group = group;
    g.t.bf16 = dtype != GAD_F16;
    g.t.err = status;
    return g;
}

template <int USE, int LAYOUT, class T, bool ADD_UP, int G>
cudaError_t launch_gated(const GatedGroup<G>& g, Sequence& q) {
    const auto kernel = gated_gemm_kernel<USE, LAYOUT, T, ADD_UP, G>;
    cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), CT_SMEM, false);
    if (e != cudaSuccess) return e;
    static std::atomic<int> known{0};
    if (known.load() <= 0) known.store(max_active_pairs(reinterpret_cast<const void*>(kernel), CT_THREADS, CT_SMEM, 2 * kPairs));
    return q.launch(kernel, dim3((unsigned)(2 * std::min(g.first[G], known.load()))), CT_THREADS, CT_SMEM, g);
}

// A launch of g.n products, and the join of the tiles that were cut.
template <int USE, int LAYOUT, class T, int G>
cudaError_t go(GatedGroup<G>& g, Sequence& q) {
    bool add_up = sizeof(T) == 4;
    int64_t u = 0;
    JoinArgs j{};
    for (int i = 0; i < kGroup; ++i) {
        if (i < g.n) {
            g.first[i] = (int)u;
            TileArgs& a = g.p[i].t;
            a.chunk = kGatedChunk<T>;
            if (sizeof(T) == 2) {
                // a sum that is no longer than a chunk is one
                const int64_t most = (int64_t)(a.whole > 0 ? a.nkb : a.kb_share) * g.p[i].segs;
                if (most > a.chunk) { add_up = true; a.chunk = std::max(1, a.chunk / g.p[i].segs); } else a.chunk = a.nkb;
            }
            u += a.whole + ((int64_t)a.tiles_m * a.tiles_n - a.whole) * a.shares;
            j.p[i] = g.p[i];
            j.first[i + 1] = j.first[i] + (a.shares > 1 ? (int)(((int64_t)a.tiles_m * a.tiles_n - a.whole) * (CT_M * a.width / 1024)) : 0);
        } else j.first[i + 1] = j.first[i];
    }
    if (u > INT32_MAX) return cudaErrorInvalidValue;
    for (int i = g.n; i <= G; ++i) g.first[i] = (int)u;
    g.p[0].clear = q.clear;
    q.clear = false;
    const cudaError_t e = add_up ? launch_gated<USE, LAYOUT, T, true>(g, q) : launch_gated<USE, LAYOUT, T, sizeof(T) == 4>(g, q);
    if constexpr (USE != kPlain) {
        if (e != cudaSuccess || !g.p[0].split) return e;
        const TileArgs& a = g.p[0].t;
        const int wide = USE == kGate ? a.width / 2 : a.width;
        return q.launch(gated_hidden_join_kernel<USE, T>, dim3((unsigned)((int64_t)a.tiles_m * a.tiles_n * (CT_M * wide / 1024))), 256, 0, g.p[0]);
    }
    if (e != cudaSuccess || j.first[kGroup] == 0) return e;
    return q.launch(gated_join_kernel<T>, dim3((unsigned)j.first[kGroup]), 256, 0, j);
}

}  // namespace

}  // namespace gad
