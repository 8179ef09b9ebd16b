// Gated feed-forward block and its backward pass:
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T            x [N x D], Wg, Wu [F x D], Wd [D x F]
//   dh = dy Wd,  dg = dh u act'(g),  du = dh act(g);   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h.
//
// Forward, two products: kGate leaves h (g and u never leave the chip), kPlain y.  For a backward pass kGate also leaves the two factors that dh is multiplied by there, act(g) and
// u act'(g), instead of g and u: one rounding to the tensors' type each where g and u would bring theirs into every factor, and the backward pass has no activation to take again.
// Backward: kHidden leaves dg and du, and one launch of kPlain takes dx (one reduction over both), dWg and dWu, and dWd.
//
// Operands as in class_loss.cu: fp16 and bfloat16 as they are, fp32 in three bfloat16 parts with six products.  h, dg and du are operands of a second product, so they are rounded to
// fp16 or bfloat16 (fp32: 24 bits): in norm the results' error grows by the square root of two over their own rounding.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "gated_few.cuh"
#include "gated_gemm.cuh"
#include "gated_launch.cuh"
#include "gated_skinny.cuh"
#include "operand_pack.cuh"

namespace gad {

namespace {

// Matrices to be copied to operands, in one launch: a warp has up to 512 columns of a row.
constexpr int kPackRun = 512;
struct PackJob { const void* src; long long ld; int rows, cols; void* dst; long long ldp, part_stride; };
struct PackJobs { PackJob job[6]; long long first[7]; int n; };   // first: runs in front of each
template <class T>
__global__ void __launch_bounds__(256) gated_pack_kernel(const __grid_constant__ PackJobs a) {
    const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_next();
    pdl_wait();
    if (i >= a.first[a.n]) return;
    int j = 0;
    while (i >= a.first[j + 1]) ++j;
    const PackJob& k = a.job[j];
    const int runs = (k.cols + kPackRun - 1) / kPackRun;
    const long long row = (i - a.first[j]) / runs;
    const int c = (int)(i - a.first[j] - row * runs) * kPackRun;
    pack_row<T>(reinterpret_cast<const T*>(k.src) + row * k.ld + c, min(kPackRun, k.cols - c), true, k.dst, row * k.ldp + c, k.part_stride, threadIdx.x & 31, 32);
}

template <class T>
__global__ void __launch_bounds__(256) gated_zero_kernel(T* __restrict__ p, int64_t ld, int64_t rows, int cols) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_float<T>(0.f);
}
__global__ void gated_empty_kernel(int32_t* status) { *status = 0; }

// ---------------------------------------------------------------------------------------------
// How a call is cut up; the same for the workspace and the launches.
// ---------------------------------------------------------------------------------------------

// An operand matrix [rows x cols] as a descriptor reaches it: where it lies, or a copy in the workspace.
struct Operand {
    const void* src; int64_t ld; int64_t rows; int cols;
    bool pack; int64_t at, ldp;        // of the copy
};

struct Room {
    int64_t at = 0;
    int64_t take(int64_t bytes) { const int64_t o = at; at += round_up(bytes, 256); return o; }
};

Operand operand(const void* p, int64_t ld, int64_t rows, int cols, int dtype, Room& room) {
    Operand o{p, ld, rows, cols, false, 0, round_up(cols, 8)};
    if (rows == 1 && dtype != GAD_F32) o.ld = o.ldp;                                      // (one row has no stride)
    o.pack = dtype == GAD_F32 || ((uintptr_t)p & 15) != 0 || o.ld == 0 || (o.ld * 2) % 16 != 0;
    if (o.pack) o.at = room.take((dtype == GAD_F32 ? 6 : 2) * rows * o.ldp);
    return o;
}

cudaError_t map_mn(CUtensorMap& m, const Operand& o, uint8_t* ws, int parts, int box, int& chunks) {
    return map_mn(m, o.pack ? ws + o.at : o.src, o.pack ? o.ldp : o.ld, o.rows, o.cols, parts, box, chunks);
}

template <class T>
cudaError_t pack(std::initializer_list<const Operand*> all, uint8_t* ws, Sequence& q) {
    PackJobs p{};
    for (const Operand* o : all)
        if (o->pack && o->src && o->rows > 0) {
            p.job[p.n] = {o->src, o->ld, (int)o->rows, o->cols, ws + o->at, o->ldp, o->rows * o->ldp};
            p.first[p.n + 1] = p.first[p.n] + o->rows * ((o->cols + kPackRun - 1) / kPackRun);
            ++p.n;
        }
    if (!p.n) return cudaSuccess;
    return q.launch(gated_pack_kernel<T>, dim3((unsigned)((p.first[p.n] + 7) / 8)), 256, 0, p);
}

#define GAD_TRY(x) do { const cudaError_t e_ = (x); if (e_ != cudaSuccess) return e_; } while (0)

// Descriptor of an operand; `box` rows at a time (64 where the reduction runs over its rows).
cudaError_t map_of(CUtensorMap& m, const Operand& o, uint8_t* ws, int parts, uint32_t box) {
    const void* base = o.pack ? ws + o.at : o.src;
    const int64_t ld = o.pack ? o.ldp : o.ld;
    return tc_make_map(&m, base, (uint64_t)o.cols, (uint64_t)o.rows, (uint64_t)parts, (uint64_t)ld * 2, (uint64_t)(ld * 2 * o.rows), box, false, true) ? cudaSuccess : cudaErrorInvalidValue;
}

// Few rows: how a product is cut.  In units of the time in which HBM gives every SM 16 KB (0.37 us): all weights once; or, where more, the stages of the SM that has most (0.45 each with few
// rows, about 0.17 us: the latency of its loads over the stages of the ring; some of it shows in any case), or what all SMs take from the L2, rows of x or h again in every stage (at 1.7 times
// HBM's rate).  To that a unit to change over, and four for a join beside its sums' way through the L2.  Fitted to a sweep of per and shares (512 x 1408 to 4096 x 16 384, 1 to 200 rows), where it stays within 5 % of
// the best.  per: a multiple of 8 rows of a matrix, the swizzle's period (kGate: of two matrices).
struct SkinnyCut { int per, tiles, nkb, shares, kb_share; };
SkinnyCut skinny_cut(int64_t rows, int n, bool gate, int64_t K) {
    const int sms = 2 * kPairs, nkb = (int)((K + CT_K - 1) / CT_K), each = gate ? 2 : 1;
    const double width = (double)round_up(rows, 16);
    SkinnyCut best{};
    double least = 1e30;
    for (int per = SK_M; per >= SK_M / 2; per -= 16) {
        const int tiles = (n + per / each - 1) / (per / each);
        const double stages = (double)tiles * nkb / sms / SK_M;
        for (int want = 1; want <= std::min(nkb, 64); want += 1 + want / 8) {
            const int kb = (nkb + want - 1) / want, shares = (nkb + kb - 1) / kb;
            if (tiles * shares > 4 * sms && shares > 1) break;
            const double waves = (double)((tiles * shares + sms - 1) / sms);
            const double one = waves * kb * 0.45 * (1 + width / 256);
            const double cost = std::max({stages * per, one, 0.6 * stages * (per + width)}) + 0.15 * one + waves + (shares > 1 ? 4.0 + (double)shares * tiles * rows / (sms * 32) : 0.0);
            if (cost < least) { least = cost; best = {per, tiles, nkb, shares, kb}; }
        }
    }
    return best;
}
bool is_skinny(const gad_gated_args& a) { return a.dtype != GAD_F32 && !a.act && a.rows <= SK_MOST_ROWS; }

// Few rows of weights that the tensor cores could only read as copies (gated_few.cuh): both products of fp32, and of 16-bit types that of Wg and Wu with one or two rows.
bool few_gate(const gad_gated_args& a) {
    const auto off = [](const void* p, int64_t ld, int64_t rows) { return ((uintptr_t)p & 15) != 0 || (rows > 1 && ld % 8 != 0); };
    if (a.act || few_group(a.rows, a.cols) == 0) return false;
    return a.dtype == GAD_F32 ? a.rows <= FEW_ROWS : a.rows <= 2 && (off(a.w_gate, a.ldwg, a.inner) || off(a.w_up, a.ldwu, a.inner));
}
bool few_down(const gad_gated_args& a) { return a.dtype == GAD_F32 && !a.act && a.rows <= FEW_ROWS && few_group(a.rows, a.inner) > 0; }
bool is_few(const gad_gated_args& a) { return a.dtype == GAD_F32 && few_gate(a) && few_down(a); }

struct ForwardPlan {
    Operand x, wg, wu, wd, h;
    SkinnyCut gate, down;
    bool gate_few;
    Cut hidden, out;
    int64_t o_slots, o_gate, total;
};
// (a tile of kGate has g and u of half as many units as it is wide)
Shape gate_shape(const gad_gated_args& a) { return {a.rows, 2 * a.inner, a.cols, 1, 1}; }
Shape out_shape(const gad_gated_args& a) { return {a.rows, a.cols, a.inner, 1, 1}; }
ForwardPlan plan_forward(const gad_gated_args& a) {
    ForwardPlan p{};
    Room room;
    if (is_few(a)) {                                     // h as it is
        p.h = {nullptr, 0, a.rows, a.inner, true, 0, round_up(a.inner, 4)};
        p.h.at = room.take(4 * a.rows * p.h.ldp);
        p.total = room.at;
        return p;
    }
    p.gate_few = is_skinny(a) && few_gate(a);
    if (!p.gate_few) {
        p.x = operand(a.x, a.ldx, a.rows, a.cols, a.dtype, room);
        p.wg = operand(a.w_gate, a.ldwg, a.inner, a.cols, a.dtype, room);
        p.wu = operand(a.w_up, a.ldwu, a.inner, a.cols, a.dtype, room);
    }
    p.wd = operand(a.w_down, a.ldwd, a.cols, a.inner, a.dtype, room);
    // h: kept where the caller wants it and a descriptor reaches it, else in the workspace
    const bool kept = a.h && a.dtype != GAD_F32;
    p.h = {kept ? a.h : nullptr, a.rows == 1 ? round_up(a.inner, 8) : a.ldh, a.rows, a.inner, !kept, 0, round_up(a.inner, 8)};
    if (!kept) p.h.at = room.take((a.dtype == GAD_F32 ? 6 : 2) * a.rows * p.h.ldp);
    if (is_skinny(a)) {
        p.gate = skinny_cut(a.rows, a.inner, true, a.cols);
        p.down = skinny_cut(a.rows, a.cols, false, a.inner);
        const auto parts = [&](const SkinnyCut& c) { return c.shares > 1 ? (int64_t)c.shares * c.tiles * a.rows * SK_M * 4 : 0; };
        p.o_gate = room.take(parts(p.gate));
        p.o_slots = room.take(parts(p.down));
    } else {
        p.hidden = cut_hidden(gate_shape(a), a.dtype == GAD_F32 ? 6 : 1, a.dtype == GAD_F32 ? (a.act ? 90 : 60) : a.act ? 25 : 15);
        p.o_gate = room.take(slot_bytes(p.hidden));
        const Shape s = out_shape(a);
        cut_group(&s, 1, a.dtype == GAD_F32 ? 6 : 1, &p.out);
        p.o_slots = room.take(slot_bytes(p.out));
    }
    p.total = room.at;
    return p;
}

template <int USE, class T>
cudaError_t go_skinny(const CUtensorMap& W0, const CUtensorMap& W1, const CUtensorMap& X, SkinnyArgs k, const SkinnyCut& c, float* parts, void* out, int64_t ldo, Sequence& q) {
    // (with shares no longer than a chunk instead, the sums of 256 rows would take an eighth of the weights' bytes to HBM and back)
    k.chunk = kGatedChunk<T>;
    const auto kernel = c.kb_share > k.chunk ? skinny_kernel<USE, T, true> : skinny_kernel<USE, T, false>;
    const cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), SK_SMEM, false);
    if (e != cudaSuccess) return e;
    k.per = c.per; k.tiles = c.tiles; k.nkb = c.nkb; k.shares = c.shares; k.kb_share = c.kb_share;
    k.stages = std::min<int>(SK_MOST_STAGES, SK_RING / (SK_A + k.width * (CT_K * 2)));
    k.clear = q.clear;
    q.clear = false;
    k.parts = c.shares > 1 ? parts : nullptr;
    k.out = out; k.ldo = ldo;
    GAD_TRY(q.launch(kernel, dim3((unsigned)std::min(2 * kPairs, c.tiles * c.shares)), SK_THREADS, SK_SMEM, W0, W1, X, k));
    if (c.shares == 1) return cudaSuccess;
    return q.launch(skinny_join_kernel<USE, T>, dim3((unsigned)((k.N + 255) / 256), (unsigned)k.rows), 256, 0, k, out, (long long)ldo);
}

// Few rows of weights as they lie.
template <int USE, int NR, class T>
cudaError_t launch_few(const FewRowsArgs& k, Sequence& q) {
    const auto on = [](const void* p, int64_t ld, int64_t rows) { return ((uintptr_t)p & 15) == 0 && (rows == 1 || ld * (int64_t)sizeof(T) % 16 == 0); };
    const bool wide = on(k.w0, k.ldw0, k.n) && (USE != kGate || on(k.w1, k.ldw1, k.n));
    const auto kernel = wide ? few_rows_kernel<USE, NR, true, T> : few_rows_kernel<USE, NR, false, T>;
    const cudaError_t e = configure_kernel_once(reinterpret_cast<const void*>(kernel), FEW_SMEM, false);
    if (e != cudaSuccess) return e;
    const size_t smem = 4 * (size_t)NR * (size_t)round_up(k.cols, 8);
    const int per = (FEW_THREADS / 32) * (USE == kGate ? 2 : 4), groups = (k.rows + NR - 1) / NR;
    // (as many blocks as run at once where shared memory allows more than one an SM)
    const int blocks = std::min((k.n + per - 1) / per, 2 * kPairs * std::max(1, std::min(4, (int)(FEW_SMEM / smem))));
    return q.launch(kernel, dim3((unsigned)blocks, (unsigned)groups), FEW_THREADS, smem, k);
}
template <int USE, class T>
cudaError_t go_few(FewRowsArgs k, Sequence& q) {
    k.clear = q.clear;
    q.clear = false;
    const int nr = few_group(k.rows, k.cols);
    return nr == 4 ? launch_few<USE, 4, T>(k, q) : nr == 2 ? launch_few<USE, 2, T>(k, q) : launch_few<USE, 1, T>(k, q);
}
template <class T>
cudaError_t few_gate_product(const gad_gated_args& a, void* h, int64_t ldh, Sequence& q) {
    return go_few<kGate, T>({a.x, a.ldx, a.w_gate, a.w_up, a.ldwg, a.ldwu, (int)a.rows, a.cols, a.inner, h, ldh, a.activation, 0, a.status}, q);
}
template <class T>
cudaError_t few_down_product(const gad_gated_args& a, const void* h, int64_t ldh, Sequence& q) {
    return go_few<kPlain, T>({h, ldh, a.w_down, nullptr, a.ldwd, 0, (int)a.rows, a.inner, a.cols, a.y, a.ldy, a.activation, 0, a.status}, q);
}

// Few rows of 16-bit operands.
template <class T>
cudaError_t run_skinny(const gad_gated_args& a, const ForwardPlan& p, uint8_t* ws, Sequence& q) {
    CUtensorMap W0, W1, X;
    SkinnyArgs k{};
    k.rows = (int)a.rows; k.width = (int)round_up(a.rows, 16); k.bf16 = a.dtype != GAD_F16; k.activation = a.activation; k.err = a.status;
    if (p.gate_few) GAD_TRY(few_gate_product<T>(a, ws + p.h.at, p.h.ldp, q));
    else {
        k.N = a.inner;
        k.early = !p.wg.pack && !p.wu.pack;
        GAD_TRY(map_of(X, p.x, ws, 1, (uint32_t)k.width));
        GAD_TRY(map_of(W0, p.wg, ws, 1, (uint32_t)p.gate.per / 2));
        GAD_TRY(map_of(W1, p.wu, ws, 1, (uint32_t)p.gate.per / 2));
        GAD_TRY((go_skinny<kGate, T>(W0, W1, X, k, p.gate, reinterpret_cast<float*>(ws + p.o_gate), ws + p.h.at, p.h.ldp, q)));
    }
    k.N = a.cols;
    k.early = !p.wd.pack;
    GAD_TRY(map_of(X, p.h, ws, 1, (uint32_t)k.width));
    GAD_TRY(map_of(W0, p.wd, ws, 1, (uint32_t)p.down.per));
    return go_skinny<kPlain, T>(W0, W0, X, k, p.down, reinterpret_cast<float*>(ws + p.o_slots), a.y, a.ldy, q);
}

template <class T>
cudaError_t run_forward(const gad_gated_args& a, const ForwardPlan& p, uint8_t* ws, cudaStream_t s) {
    const int parts = a.dtype == GAD_F32 ? 3 : 1;
    Sequence q{s};
    GAD_TRY(pack<T>({&p.x, &p.wg, &p.wu, &p.wd}, ws, q));
    if constexpr (sizeof(T) == 4) {
        if (is_few(a)) {
            GAD_TRY(few_gate_product<float>(a, ws + p.h.at, p.h.ldp, q));
            GAD_TRY(few_down_product<float>(a, ws + p.h.at, p.h.ldp, q));
            return cudaGetLastError();
        }
    }
    if constexpr (sizeof(T) == 2) {
        if (is_skinny(a)) { GAD_TRY(run_skinny<T>(a, p, ws, q)); return cudaGetLastError(); }
    }
    GatedGroup<1> r{};
    r.n = 1;
    GatedArgs& g = r.p[0];
    g = product(gate_shape(a), p.hidden, a.dtype, false, 16, a.status);
    g.t.N = a.inner;
    g.activation = a.activation;
    g.h = p.h.pack ? ws + p.h.at : const_cast<void*>(p.h.src);
    g.ldh = p.h.pack ? p.h.ldp : p.h.ld;
    g.h_part = a.rows * g.ldh;
    g.act = a.act; g.ldact = a.ldact; g.slope = a.slope; g.ldslope = a.ldslope;
    g.C[0] = a.dtype == GAD_F32 ? a.h : nullptr; g.ldc[0] = a.ldh;
    g.t.slots = reinterpret_cast<float*>(ws + p.o_gate);
    GAD_TRY(map_of(r.A[0], p.x, ws, parts, CT_H));
    GAD_TRY(map_of(r.B0[0], p.wg, ws, parts, (uint32_t)g.t.width / 2));
    GAD_TRY(map_of(r.B1[0], p.wu, ws, parts, (uint32_t)g.t.width / 2));
    GAD_TRY((go<kGate, kBothK, T>(r, q)));
    g = product(out_shape(a), p.out, a.dtype, false, 8, a.status);
    g.C[0] = a.y; g.ldc[0] = a.ldy;
    g.t.slots = reinterpret_cast<float*>(ws + p.o_slots);
    GAD_TRY(map_of(r.A[0], p.h, ws, parts, CT_H));
    GAD_TRY(map_of(r.B0[0], p.wd, ws, parts, (uint32_t)g.t.width / 2));
    GAD_TRY((go<kPlain, kBothK, T>(r, q)));
    return cudaGetLastError();
}

struct BackwardPlan {
    Operand dy, x, wg, wu, wd, h;
    Cut hidden, cut[kGroup];
    Shape shape[kGroup];
    int n, at_x, at_gu, at_d;          // products behind dg and du, and which is which (-1: not wanted)
    int64_t o_dg, ldg, o_hidden, o_slots[kGroup], total;
};
bool wants_hidden(const gad_gated_grad_args& a) { return a.dx || a.dw_gate || a.dw_up; }
Shape hidden_shape(const gad_gated_grad_args& a) { return {a.rows, a.inner, a.cols, 1, 1}; }
BackwardPlan plan_backward(const gad_gated_grad_args& a) {
    BackwardPlan p{};
    Room room;
    const bool hidden = wants_hidden(a);
    const auto maybe = [&](bool wanted, const void* ptr, int64_t ld, int64_t rows, int cols) { return wanted ? operand(ptr, ld, rows, cols, a.dtype, room) : Operand{}; };
    p.dy = maybe(hidden || a.dw_down, a.dy, a.lddy, a.rows, a.cols);
    p.wd = maybe(hidden, a.w_down, a.ldwd, a.cols, a.inner);
    p.wg = maybe(a.dx, a.w_gate, a.ldwg, a.inner, a.cols);
    p.wu = maybe(a.dx, a.w_up, a.ldwu, a.inner, a.cols);
    p.x = maybe(a.dw_gate || a.dw_up, a.x, a.ldx, a.rows, a.cols);
    p.h = maybe(a.dw_down, a.h, a.ldh, a.rows, a.inner);
    p.ldg = round_up(a.inner, 8);
    if (hidden) {
        p.o_dg = room.take((a.dtype == GAD_F32 ? 12 : 4) * a.rows * p.ldg);
        p.hidden = cut_hidden(hidden_shape(a), a.dtype == GAD_F32 ? 6 : 1, a.dtype == GAD_F32 ? 80 : 15);
        p.o_hidden = room.take(slot_bytes(p.hidden));
    }
    p.at_x = p.at_gu = p.at_d = -1;
    if (a.dx) { p.at_x = p.n; p.shape[p.n++] = {a.rows, a.cols, a.inner, 1, 2}; }
    if (a.dw_gate || a.dw_up) { p.at_gu = p.n; p.shape[p.n++] = {a.inner, a.cols, a.rows, a.dw_gate && a.dw_up ? 2 : 1, 1}; }
    if (a.dw_down) { p.at_d = p.n; p.shape[p.n++] = {a.cols, a.inner, a.rows, 1, 1}; }
    cut_group(p.shape, p.n, a.dtype == GAD_F32 ? 6 : 1, p.cut);
    for (int i = 0; i < p.n; ++i) p.o_slots[i] = room.take(slot_bytes(p.cut[i]));
    p.total = room.at;
    return p;
}

template <class T>
cudaError_t run_backward(const gad_gated_grad_args& a, const BackwardPlan& p, uint8_t* ws, cudaStream_t s) {
    const int parts = a.dtype == GAD_F32 ? 3 : 1;
    const int64_t N = a.rows;
    Sequence q{s};
    GAD_TRY(pack<T>({&p.dy, &p.wd, &p.wg, &p.wu, &p.x, &p.h}, ws, q));
    uint8_t* dg = ws + p.o_dg;
    const int64_t part = N * p.ldg;                       // values of a part of dg; du lies behind all of dg's
    if (wants_hidden(a)) {
        GatedGroup<1> r{};
        r.n = 1;
        GatedArgs& g = r.p[0];
        g = product(hidden_shape(a), p.hidden, a.dtype, false, 16, a.status);
        g.act = const_cast<void*>(a.act); g.ldact = a.ldact; g.slope = const_cast<void*>(a.slope); g.ldslope = a.ldslope;
        g.C[0] = dg; g.ldh = p.ldg; g.h_part = part;
        g.t.slots = reinterpret_cast<float*>(ws + p.o_hidden);
        GAD_TRY(map_of(r.A[0], p.dy, ws, parts, CT_H));
        GAD_TRY(map_mn(r.B0[0], p.wd, ws, parts, g.t.width / 2, g.b_chunks));
        GAD_TRY((go<kHidden, kBMN, T>(r, q)));
    }
    GatedGroup<kGroup> r{};
    r.n = p.n;
    for (int i = 0; i < p.n; ++i) {
        r.p[i] = product(p.shape[i], p.cut[i], a.dtype, i != p.at_x, 8, a.status);
        r.p[i].t.slots = reinterpret_cast<float*>(ws + p.o_slots[i]);
    }
    if (p.at_x >= 0) {
        const int i = p.at_x;
        r.p[i].C[0] = a.dx; r.p[i].ldc[0] = a.lddx;
        if (!tc_make_map(&r.A[i], dg, (uint64_t)a.inner, (uint64_t)N, (uint64_t)(2 * parts), (uint64_t)p.ldg * 2, (uint64_t)part * 2, CT_H, false, true)) return cudaErrorInvalidValue;
        GAD_TRY(map_mn(r.B0[i], p.wg, ws, parts, r.p[i].t.width / 2, r.p[i].b_chunks));
        GAD_TRY(map_mn(r.B1[i], p.wu, ws, parts, r.p[i].t.width / 2, r.p[i].b_chunks));
    }
    if (p.at_gu >= 0) {
        const int i = p.at_gu;
        r.p[i].C[0] = a.dw_gate ? a.dw_gate : a.dw_up; r.p[i].ldc[0] = a.dw_gate ? a.lddwg : a.lddwu;
        r.p[i].C[1] = a.dw_up; r.p[i].ldc[1] = a.lddwu;
        GAD_TRY(map_mn(r.A[i], dg + (a.dw_gate ? 0 : 1) * parts * part * 2, p.ldg, N, a.inner, p.shape[i].planes * parts, CT_H, r.p[i].a_chunks));
        GAD_TRY(map_mn(r.B0[i], p.x, ws, parts, r.p[i].t.width / 2, r.p[i].b_chunks));
    }
    if (p.at_d >= 0) {
        const int i = p.at_d;
        r.p[i].C[0] = a.dw_down; r.p[i].ldc[0] = a.lddwd;
        GAD_TRY(map_mn(r.A[i], p.dy, ws, parts, CT_H, r.p[i].a_chunks));
        GAD_TRY(map_mn(r.B0[i], p.h, ws, parts, r.p[i].t.width / 2, r.p[i].b_chunks));
    }
    GAD_TRY((go<kPlain, kAnyMN, T>(r, q)));
    return cudaGetLastError();
}
#undef GAD_TRY

template <class T> int zero(void* p, int64_t ld, int64_t rows, int cols, cudaStream_t s) {
    if (!p) return 0;
    gated_zero_kernel<T><<<592, 256, 0, s>>>((T*)p, ld, rows, cols);
    ++g_kernel_launches;
    return 0;
}
int empty(int32_t* status, cudaStream_t s) {
    gated_empty_kernel<<<1, 1, 0, s>>>(status);
    ++g_kernel_launches;
    return cudaGetLastError() == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
}
// No rows: gradients of the weights are zero.
template <class T>
int run_no_rows(const gad_gated_grad_args& a, cudaStream_t s) {
    zero<T>(a.dw_gate, a.lddwg, a.inner, a.cols, s);
    zero<T>(a.dw_up, a.lddwu, a.inner, a.cols, s);
    zero<T>(a.dw_down, a.lddwd, a.cols, a.inner, s);
    return empty(a.status, s);
}

bool sizes_ok(int dtype, int64_t rows, int cols, int inner) { return dtype >= GAD_F32 && dtype <= GAD_BF16 && rows >= 0 && cols >= 1 && inner >= 1; }
bool in_range(int64_t rows, int cols, int inner) { return rows <= (1 << 30) && cols <= (1 << 20) && inner <= (1 << 20); }

// Any of them off the elements of its type (null is on).
bool off_elements(int dtype, std::initializer_list<const void*> all, const int32_t* status) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= (uintptr_t)p;
    return (bits & (dtype == GAD_F32 ? 3 : 1)) != 0 || ((uintptr_t)status & 3) != 0;
}
int check_forward(const gad_gated_args* a) {
    if (!a || !sizes_ok(a->dtype, a->rows, a->cols, a->inner)) return GAD_ERR_ARG;
    if (!in_range(a->rows, a->cols, a->inner)) return GAD_ERR_RANGE;
    if (a->activation < GAD_SILU || a->activation > GAD_SIGMOID) return GAD_ERR_ARG;
    if ((a->rows > 1 && a->ldx != 0 && a->ldx < a->cols) || a->ldwg < a->cols || a->ldwu < a->cols || a->ldwd < a->inner || (a->rows > 1 && a->ldy < a->cols)) return GAD_ERR_ARG;
    const int kept = (a->act != nullptr) + (a->slope != nullptr) + (a->h != nullptr);
    if (kept != 0 && kept != 3) return GAD_ERR_ARG;
    if (kept && a->rows > 1 && (a->ldact < a->inner || a->ldslope < a->inner || a->ldh < a->inner)) return GAD_ERR_ARG;
    // h is an operand of the second product where it lies
    if (kept && a->dtype != GAD_F32 && (((uintptr_t)a->h & 15) != 0 || (a->rows > 1 && a->ldh % 8 != 0))) return GAD_ERR_ARG;
    return GAD_OK;
}
int check_backward(const gad_gated_grad_args* a) {
    if (!a || !sizes_ok(a->dtype, a->rows, a->cols, a->inner)) return GAD_ERR_ARG;
    if (!in_range(a->rows, a->cols, a->inner)) return GAD_ERR_RANGE;
    if (a->rows > 1 && ((a->lddy != 0 && a->lddy < a->cols) || (a->ldx != 0 && a->ldx < a->cols) || (a->dx && a->lddx < a->cols) || a->ldact < a->inner || a->ldslope < a->inner || a->ldh < a->inner))
        return GAD_ERR_ARG;
    if (a->ldwg < a->cols || a->ldwu < a->cols || a->ldwd < a->inner || (a->dw_gate && a->lddwg < a->cols) || (a->dw_up && a->lddwu < a->cols) || (a->dw_down && a->lddwd < a->inner)) return GAD_ERR_ARG;
    return GAD_OK;
}

}  // namespace
}  // namespace gad

extern "C" int gad_gated_feed_forward_workspace_bytes(const gad_gated_args* args, size_t* bytes) {
    const int rc = gad::check_forward(args);
    if (rc != GAD_OK) return rc;
    if (!bytes) return GAD_ERR_ARG;
    *bytes = args->rows == 0 ? 0 : (size_t)gad::plan_forward(*args).total;
    return GAD_OK;
}

extern "C" int gad_gated_feed_forward(const gad_gated_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace gad;
    const int rc = check_forward(args);
    if (rc != GAD_OK) return rc;
    const gad_gated_args& a = *args;
    if (!a.status || off_elements(a.dtype, {a.x, a.w_gate, a.w_up, a.w_down, a.y, a.act, a.slope, a.h}, a.status)) return GAD_ERR_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    if (a.rows == 0) return empty(a.status, s);
    if (!a.x || !a.w_gate || !a.w_up || !a.w_down || !a.y) return GAD_ERR_ARG;
    const ForwardPlan p = plan_forward(a);
    const size_t need = (size_t)p.total;
    if (need && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need)) return GAD_ERR_OOM;
    try {
        uint8_t* ws = (uint8_t*)workspace;
        const cudaError_t e = a.dtype == GAD_F32 ? run_forward<float>(a, p, ws, s) : a.dtype == GAD_F16 ? run_forward<__half>(a, p, ws, s) : run_forward<__nv_bfloat16>(a, p, ws, s);
        return e == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
    } catch (...) {   // (the table of configured kernels could not grow)
        return GAD_ERR_OOM;
    }
}

extern "C" int gad_gated_feed_forward_backward_workspace_bytes(const gad_gated_grad_args* args, size_t* bytes) {
    const int rc = gad::check_backward(args);
    if (rc != GAD_OK) return rc;
    if (!bytes) return GAD_ERR_ARG;
    *bytes = args->rows == 0 ? 0 : (size_t)gad::plan_backward(*args).total;
    return GAD_OK;
}

extern "C" int gad_gated_feed_forward_backward(const gad_gated_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace gad;
    const int rc = check_backward(args);
    if (rc != GAD_OK) return rc;
    const gad_gated_grad_args& a = *args;
    if (!a.status || off_elements(a.dtype, {a.dy, a.x, a.w_gate, a.w_up, a.w_down, a.act, a.slope, a.h, a.dx, a.dw_gate, a.dw_up, a.dw_down}, a.status)) return GAD_ERR_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    if (a.rows == 0) return a.dtype == GAD_F32 ? run_no_rows<float>(a, s) : a.dtype == GAD_F16 ? run_no_rows<__half>(a, s) : run_no_rows<__nv_bfloat16>(a, s);
    if (!a.dy || !a.x || !a.w_gate || !a.w_up || !a.w_down || !a.act || !a.slope || !a.h) return GAD_ERR_ARG;
    if (!a.dx && !a.dw_gate && !a.dw_up && !a.dw_down) return empty(a.status, s);
    const BackwardPlan p = plan_backward(a);
    const size_t need = (size_t)p.total;
    if (need && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need)) return GAD_ERR_OOM;
    try {
        uint8_t* ws = (uint8_t*)workspace;
        const cudaError_t e = a.dtype == GAD_F32 ? run_backward<float>(a, p, ws, s) : a.dtype == GAD_F16 ? run_backward<__half>(a, p, ws, s) : run_backward<__nv_bfloat16>(a, p, ws, s);
        return e == cudaSuccess ? GAD_OK : GAD_ERR_CUDA;
    } catch (...) {
        return GAD_ERR_OOM;
    }
}
