// C ABI of the layers in front of a loss: argument checks and kernel launches.  Declarations and contracts are in include/kimad.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "operators_host.h"
#include "k_dropout.h"
#include "k_gemm.h"
#include "k_linear.h"
#include "k_xent.h"

namespace {

using namespace kimad;

static_assert(ACT_NONE == KIMAD_ACT_NONE && ACT_RELU == KIMAD_ACT_RELU && ACT_GELU == KIMAD_ACT_GELU && ACT_SILU == KIMAD_ACT_SILU, "header and kernel constants");

constexpr uint64_t FEW_MOST = 96;                        // products of so many rows may go by k_gemm_few (FEW_ROWS of the binding)
constexpr uint64_t LD_MOST = 1ull << 22;                 // operands: 256 rows are reached by 32-bit offsets
constexpr uint64_t OUT_LD_MOST = 1ull << 24;             // results: 32 rows
constexpr uint64_t ROWS_MOST = 65535ull * SUM_ROWS;      // 4194240: the column sums' grid
constexpr uint64_t MATRIX_MOST = 1ull << 33;             // elements of a matrix are fewer: the grid of what lays two of them out

typedef GemmTile<256, 256, 2, 4> Gemm256;
typedef GemmTile<128, 128, 2, 2> Gemm128;
typedef GemmTile<64, 64, 2, 2> Gemm64;

template <class F>
int with_half_type(uint32_t type, F f) {
    if (type == KIMAD_VALUES_F16) return f(std::integral_constant<uint32_t, TYPE_F16>{});
    return f(std::integral_constant<uint32_t, TYPE_BF16>{});
}

// A workspace is handed out from its beginning, in pieces that begin at multiples of 256 bytes; without an address it is only measured.
struct Room {
    uint8_t* base;
    uint64_t used;
    template <class T>
    T* take(uint64_t count) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += (count * sizeof(T) + 255) & ~255ull;
        return p;
    }
};

// How a product is shared out: by the least of the times below, which are fits (us) to measurements of each tile alone: rounds of as many tiles as compute units hold, and a
// last one that costs less the fewer of them it has.  The tiles of a last round may be shared out along the sum too (`splits` parts, which are of fp32 and are added by a
// second launch).  Measured into 16 bits (us; each tile without parts, and the best way of all that were tried; the choice comes within 7 % of it but at 2048 x 2048 x 2048, 14 %):
//                   M      N      K        256     128     64      best                 M      N      K        256     128     64      best
//   both along K    77     1000   520      21      12      8.1     7.4 few rows         1024   4096   4096     101     60      57      52  256, 4 parts
//                   64     8192   8192     184     102     64      27  64, 4 parts      2048   5632   2048     56      67      80      56  256
//                   256    768    768      25      13      8.7     8.7 64               4096   768    16384    369     208     156     105 256, 5 parts
//                   2048   2048   2048     56      29      33      29  128              8192   5632   2048     174     200     295     174 256
//   B across K      299    3683   9456     240     135     88      45  128, 5 parts     4096   768    50304    1431    859     604     342 256, 5 parts
//                   300    1000   1000     30      17      10      10  64               8192   2048   5632     158     189     299     158 256
//   both across K   1000   520    104      15      8.9     6.1     6.1 64               50257  768    4096     395     411     832     353 256, 3 parts of the last
//                   768    768    8192     194     112     71      26  64, 5 parts      5632   2048   8192     196     230     347     196 256
struct GemmPlan {
    enum { FEW, T64, T128, T256 } kind;
    uint64_t tiles_m, tiles_n, whole;
    uint32_t splits, share;
    double us;
    uint32_t strip() const { return kind == FEW ? 16 : kind == T64 ? Gemm64::STRIP : kind == T128 ? Gemm128::STRIP : Gemm256::STRIP; }
    uint64_t edge() const { return kind == T256 ? 256 : kind == T128 ? 128 : 64; }
    uint64_t shared() const { return kind == FEW ? 0 : tiles_m * tiles_n - whole; }
    uint64_t parts_count() const { return shared() * splits * edge() * edge(); }
};
GemmPlan gemm_plan(uint64_t M, uint64_t N, uint64_t K, bool wide, bool may_split, uint32_t few) {
    GemmPlan best{};
    best.splits = 1;
    const uint64_t stages = (K + GEMM_STAGE_K - 1) / GEMM_STAGE_K;
    best.share = (uint32_t)stages;
    // k_gemm_few, whose waves read all of A each; rows that begin off 16-byte addresses cost it nearly twice as much, and the tiles a copy.
    const double copy = few == 2 ? 4.0 + (double)((M + N) * K) * 4.0 / 4.5e6 : 0.0;
    if (few && M <= FEW_MOST) {
        best.kind = GemmPlan::FEW;
        best.us = 2.5 + (double)(N * K) * (0.26e-6 + 1.5e-8 * (double)M) * (few == 2 ? 1.8 : 1.0) - copy;
        if (best.us <= 0) best.us = 1e-3;
    }
    const double read = 2.0 + (double)((M + N) * K) * 2.0 / 4.5e6;            // both operands from memory
    // of one tile: a stage with nothing beside it on its compute unit, and a unit's time for one among others; its end in 16 bits and in 32; the launch; tiles that
    // a compute unit holds
    struct { decltype(best.kind) kind; uint64_t edge; double alone, stage, end16, end32, launch; uint64_t held; } const kinds[] = {
        {GemmPlan::T256, 256, 1.5, 1.65, 6.0, 8.0, 4.0, 1}, {GemmPlan::T128, 128, 0.87, 0.56, 1.0, 1.5, 5.0, 2}, {GemmPlan::T64, 64, 0.5, 0.21, 0.35, 0.35, 4.5, 4}};
    for (const auto& k : kinds) {
        const uint64_t tm = (M + k.edge - 1) / k.edge, tn = (N + k.edge - 1) / k.edge, tiles = tm * tn, slots = UNITS * k.held, full = tiles / slots * slots, rest = tiles - full;
        auto rounds = [&](uint64_t items, uint64_t each, double end) {        // of `each` stages a tile
            const uint64_t left = (items % slots + UNITS - 1) / UNITS;
            const double whole = (double)(items / slots * k.held) * ((double)each * k.stage + end);
            return left ? whole + (double)each * std::max(k.alone, (double)left * k.stage) + (double)left * end : whole;
        };
        for (uint64_t splits = 1; splits == 1 || (may_split && rest && splits <= 256 && 4 * splits <= stages && (splits <= 4 || rest * splits <= 2 * slots)); splits += splits < 16 ? 1 : splits / 4) {
            const uint64_t share = (stages + splits - 1) / splits, parts = (stages + share - 1) / share;
            if (parts != splits) continue;
            const double end = wide ? k.end32 : k.end16;
            double us = k.launch + rounds(full, stages, end) + rounds(rest * parts, share, parts > 1 ? k.end32 : end);
            if (parts > 1) us += 6.5 + 0.1 * (double)parts + (double)(rest * parts * k.edge * k.edge) * 8.0 / 8e6;   // 4 bytes written and read, much of them beyond memory
            us = std::max(us, read);
            if (best.us == 0 || us < best.us) {
                best.us = us;
                best.kind = k.kind; best.tiles_m = tm; best.tiles_n = tn; best.whole = parts > 1 ? full : tiles;
                best.splits = (uint32_t)parts; best.share = (uint32_t)share;
            }
        }
    }
    return best;
}

// Rows of tiles in a band: about as many as columns among the tiles that an XCD has at a time, so that these share most of what they read.
uint32_t band_rows(const GemmPlan& p) {
    const uint64_t run = std::min<uint64_t>(UNITS / 8, (p.tiles_m * p.tiles_n * p.splits + 7) / 8);
    const uint64_t across = std::max<uint64_t>(1, std::min(p.tiles_n, (uint64_t)std::sqrt((double)run)));
    return (uint32_t)std::min(p.tiles_m, (run + across - 1) / across);
}

template <uint32_t TYPE, class T, bool XA, bool XB, uint32_t END>
int launch_tile(GemmArgs g, const GemmPlan& p, hipStream_t s) {
    const uint64_t items = p.whole + p.shared() * p.splits;                   // (below 2^28 for matrices of fewer than 2^33 elements)
    constexpr uint64_t slots = UNITS * ((160 * 1024) / T::LDS);
    g.tiles_m = (uint32_t)p.tiles_m; g.tiles_n = (uint32_t)p.tiles_n; g.band = band_rows(p); g.whole = (uint32_t)p.whole; g.splits = p.splits; g.share = p.share;
    hipLaunchKernelGGL((k_gemm_tile<TYPE, T, XA, XB, END>), dim3((uint32_t)std::min<uint64_t>(items, slots)), dim3(64 * T::WAVES), 0, s, g);
    if constexpr (END != END_SOFTMAX)
        if (p.splits > 1) {
            const uint64_t units = p.shared() * (T::WAVES * T::TI);
            if (const int rc = launched()) return rc;
            hipLaunchKernelGGL((k_gemm_join<TYPE, T, END>), dim3((uint32_t)((units + 3) / 4)), dim3(256), 0, s, g);
        }
    return launched();
}
template <uint32_t TYPE, uint32_t END>
int launch_few(const GemmArgs& g, hipStream_t s) {
    const uint32_t groups = (uint32_t)((g.N + 15) / 16);
    const bool shifted = !aligned(g.a, 16) || !aligned(g.b, 16) || (g.lda % 8 && g.M > 1) || (g.ldb % 8 && g.N > 1);
    auto go = [&](auto mt) {
        if (shifted) hipLaunchKernelGGL((k_gemm_few<TYPE, decltype(mt)::value, END, true>), dim3(groups), dim3(256), 0, s, g);
        else hipLaunchKernelGGL((k_gemm_few<TYPE, decltype(mt)::value, END, false>), dim3(groups), dim3(256), 0, s, g);
        return launched();
    };
    if (g.M <= 16) return go(std::integral_constant<uint32_t, 1>{});
    if (g.M <= 32) return go(std::integral_constant<uint32_t, 2>{});
    if (g.M <= 64) return go(std::integral_constant<uint32_t, 4>{});
    return go(std::integral_constant<uint32_t, 6>{});
}
template <uint32_t TYPE, bool XA, bool XB, uint32_t END>
int launch_kind(const GemmArgs& g, const GemmPlan& p, hipStream_t s) {
    if constexpr (!XA && !XB)
        if (p.kind == GemmPlan::FEW) return launch_few<TYPE, END>(g, s);
    if (p.kind == GemmPlan::T256) return launch_tile<TYPE, Gemm256, XA, XB, END>(g, p, s);
    if (p.kind == GemmPlan::T128) return launch_tile<TYPE, Gemm128, XA, XB, END>(g, p, s);
    return launch_tile<TYPE, Gemm64, XA, XB, END>(g, p, s);
}
// A product and its end; parts: room for the plan's parts_count() numbers.
template <uint32_t TYPE, bool XA, bool XB>
int launch_gemm(GemmArgs g, const GemmPlan& p, bool out32, float* parts, hipStream_t s) {
    g.parts = parts;
    return out32 ? launch_kind<TYPE, XA, XB, END_F32>(g, p, s) : launch_kind<TYPE, XA, XB, END_TYPE>(g, p, s);
}

// A sum over nothing, and its end.
template <uint32_t TYPE>
int launch_none(uint64_t M, uint64_t N, const GemmEnd& end, bool out32, hipStream_t s) {
    const uint32_t wgs = (uint32_t)std::min<uint64_t>((M * N + 255) / 256, 65536);
    if (wgs == 0) return KIMAD_OK;
    if (out32) hipLaunchKernelGGL((k_gemm_none<TYPE, true>), dim3(wgs), dim3(256), 0, s, M, N, end);
    else hipLaunchKernelGGL((k_gemm_none<TYPE, false>), dim3(wgs), dim3(256), 0, s, M, N, end);
    return launched();
}
int zeros(void* out, uint32_t type, uint64_t rows, uint64_t cols, uint64_t ld, hipStream_t s) {
    GemmEnd end{};
    end.out = out; end.ld = ld;
    return launch_none<TYPE_BF16>(rows, cols, end, type == KIMAD_VALUES_F32, s);
}

// Whether the tiles' loads reach an operand as it lies: rows at 16-byte addresses, and for one that is stored along K rows that end at one.
bool lies_well(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, bool along) { return aligned(p, 16) && (ld % 8 == 0 || rows <= 1) && (!along || cols % 8 == 0); }
// Two matrices (either may stay where it is: `to` null) laid out anew; the first one's rows that do not count become zeros.  scale: as k_rows_copy makes it.
struct CopyOf {
    const void* from;
    uint64_t ld, rows, cols;
    void* to;
};
int copy_rows(const CopyOf& first, const CopyOf& second, const int32_t* target, uint64_t vocab, const float* weight, float* scale, float largest, hipStream_t s) {
    CopyArgs a{};
    const CopyOf* of[2] = {&first, &second};
    uint64_t wgs[2];
    for (uint32_t i = 0; i < 2; ++i) {
        a.from[i] = of[i]->from; a.to[i] = of[i]->to; a.ld[i] = of[i]->ld; a.rows[i] = of[i]->rows; a.cols[i] = of[i]->cols; a.pitch[i] = pitch_of(of[i]->cols);
        wgs[i] = of[i]->to ? (of[i]->rows * (a.pitch[i] / 8) + 255) / 256 : 0;
    }
    if (wgs[0] + wgs[1] == 0 && !scale) return KIMAD_OK;
    a.scale = scale; a.largest = largest;
    a.wgs0 = (uint32_t)wgs[0]; a.target = target; a.weight = weight; a.vocab = (uint32_t)vocab;
    hipLaunchKernelGGL(k_rows_copy, dim3((uint32_t)(wgs[0] + wgs[1] + (scale ? 1 : 0))), dim3(256), 0, s, a);
    return launched();
}
// an operand: its address and leading dimension, copied or in place
struct Operand {
    const void* p;
    uint64_t ld;
};
Operand operand(const void* copy, const void* p, uint64_t ld, uint64_t rows, uint64_t cols) { return copy ? Operand{copy, pitch_of(cols)} : Operand{p, stage_ld(rows, cols, ld)}; }

bool matrix_ok(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t bytes, uint64_t most) {
    return ld >= cols && ld <= most && (rows == 0 || cols == 0 || (p && aligned(p, bytes)));
}
bool fits(uint64_t rows, uint64_t cols) { return cols == 0 || rows < MATRIX_MOST / cols; }
bool half_type(uint32_t type) { return type == KIMAD_VALUES_F16 || type == KIMAD_VALUES_BF16; }

// ---- linear ----

struct LinearRoom {
    uint16_t *x, *w;
    float* parts;
    GemmPlan plan;
};
LinearRoom linear_room(Room& room, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint64_t M, uint64_t N, uint64_t K) {
    LinearRoom r{};
    const bool x_well = lies_well(x, ld_x, M, K, true), w_well = lies_well(w, ld_w, N, K, true);
    r.plan = gemm_plan(M, N, K, true, true, x_well && w_well ? 1 : 2);
    if (r.plan.kind == GemmPlan::FEW) return r;
    if (!x_well) r.x = room.take<uint16_t>(M * pitch_of(K));
    if (!w_well) r.w = room.take<uint16_t>(N * pitch_of(K));
    r.parts = room.take<float>(r.plan.parts_count());
    return r;
}
bool linear_sizes_ok(uint64_t M, uint64_t N, uint64_t K) { return M <= ROWS_MOST && N <= LD_MOST && K <= LD_MOST && fits(M, N + 7) && fits(M, K + 7) && fits(N, K + 7); }

// ---- gradient of a linear layer ----

struct LinearGradRoom {
    bool dz_made;                // else dy itself is dz
    uint16_t *dz, *x, *w;
    float *sums, *parts;
    uint64_t sum_rows, sum_parts;
    GemmPlan dx, dw;
};
LinearGradRoom linear_grad_room(Room& room, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint64_t M, uint64_t N, uint64_t K, uint32_t act,
                                uint32_t wants) {
    LinearGradRoom r{};
    const bool dx = wants & KIMAD_WANT_DX, dw = wants & KIMAD_WANT_DW;
    r.dz_made = (dx || dw) && (act != KIMAD_ACT_NONE || !lies_well(dy, ld_dy, M, N, true));
    if (r.dz_made) r.dz = room.take<uint16_t>(M * pitch_of(N));
    if (dw && !lies_well(x, ld_x, M, K, false)) r.x = room.take<uint16_t>(M * pitch_of(K));
    if (dx && !lies_well(w, ld_w, N, K, false)) r.w = room.take<uint16_t>(N * pitch_of(K));
    r.sum_rows = M <= 2 * SUM_ROWS ? 2 * SUM_ROWS : SUM_ROWS;
    r.sum_parts = (M + r.sum_rows - 1) / r.sum_rows;
    if ((wants & KIMAD_WANT_DB) && r.sum_parts > 1) r.sums = room.take<float>(r.sum_parts * N);
    uint64_t parts = 0;
    if (dx) {
        r.dx = gemm_plan(M, K, pitch_of(N), false, true, 0);
        parts = std::max(parts, r.dx.parts_count());
    }
    if (dw) {
        r.dw = gemm_plan(N, K, M, true, true, 0);
        parts = std::max(parts, r.dw.parts_count());
    }
    r.parts = room.take<float>(parts);
    return r;
}

// ---- cross entropy ----

// Of the exponentials that a gradient's piece of rows keeps: 8192 rows of 50257, width 768, in one piece 2398 us, in two 2536, in four (which the memory-side cache would hold)
// 2821, for every piece adds to all of dw.
constexpr uint64_t PIECE_BYTES = 1ull << 30;
struct XentRoom {
    uint64_t piece, pieces, pitch;
    uint16_t *x, *w, *e;
    f32x2* strips;
    f32x4* rows_out;
    float *picked, *scale, *sum, *parts;
    struct { GemmPlan z, dx, dw; } plans[2];             // of a piece, and of the last one, which may have fewer rows
};
XentRoom xent_room(Room& room, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint64_t rows, uint64_t vocab, uint64_t dim, uint32_t wants, uint32_t dw_type) {
    XentRoom r{};
    const bool dx = wants & KIMAD_WANT_DX, dw = wants & KIMAD_WANT_DW, grad = dx || dw;
    r.pitch = (vocab + 63) / 64 * 64;
    const uint64_t row_bytes = grad ? 2 * r.pitch : r.pitch / 4;               // (without a gradient the strips' 8 bytes of 32 columns)
    uint64_t most = std::max<uint64_t>(PIECE_BYTES / row_bytes / 256 * 256, 256);
    r.pieces = (rows + most - 1) / most;
    r.piece = r.pieces <= 1 ? rows : std::min(most, ((rows + r.pieces - 1) / r.pieces + 255) / 256 * 256);
    r.pieces = (rows + r.piece - 1) / r.piece;
    const bool x_well = lies_well(x, ld_x, rows, dim, true), w_well = lies_well(w, ld_w, vocab, dim, true);
    uint64_t parts = 0, strips = 0;
    for (uint32_t last = 0; last < 2; ++last) {
        const uint64_t n = last ? rows - (r.pieces - 1) * r.piece : r.piece;
        auto& p = r.plans[last];
        p.z = gemm_plan(n, vocab, dim, false, false, grad ? 0 : x_well && w_well ? 1 : 2);
        strips = std::max(strips, n * ((vocab + p.z.strip() - 1) / p.z.strip()));
        if (dx) p.dx = gemm_plan(n, dim, r.pitch, false, true, 0);
        if (dw) p.dw = gemm_plan(vocab, dim, n, r.pieces > 1, true, 0);
        parts = std::max(parts, std::max(dx ? p.dx.parts_count() : 0, dw ? p.dw.parts_count() : 0));
    }
    const bool few = r.plans[0].z.kind == GemmPlan::FEW && r.plans[1].z.kind == GemmPlan::FEW;
    if (grad || (!few && !x_well)) r.x = room.take<uint16_t>(rows * pitch_of(dim));
    if (!few && !w_well) r.w = room.take<uint16_t>(vocab * pitch_of(dim));
    r.strips = room.take<f32x2>(strips);
    r.picked = room.take<float>(r.piece);
    if (!grad) return r;
    r.rows_out = room.take<f32x4>(r.piece);
    r.scale = room.take<float>(2);
    r.e = room.take<uint16_t>(r.piece * r.pitch);
    if (dw && r.pieces > 1 && dw_type != KIMAD_VALUES_F32) r.sum = room.take<float>(vocab * dim);
    r.parts = room.take<float>(parts);
    return r;
}
bool xent_sizes_ok(uint64_t rows, uint64_t vocab, uint64_t dim) { return rows <= ROWS_MOST && vocab && vocab <= LD_MOST - 64 && dim && dim <= LD_MOST && fits(rows, dim + 7) && fits(vocab, dim + 7); }

}  // namespace

extern "C" {

uint64_t kimad_linear_workspace_bytes(const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint64_t M, uint64_t N, uint64_t K) {
    if (!linear_sizes_ok(M, N, K) || M == 0 || N == 0 || K == 0) return 0;
    Room room{nullptr, 0};
    linear_room(room, x, ld_x, w, ld_w, M, N, K);
    return room.used;
}

int kimad_linear(const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint32_t type, uint64_t M, uint64_t N, uint64_t K, const void* bias, const void* residual,
                 uint64_t ld_residual, uint32_t act, void* z, uint64_t ld_z, void* out, uint32_t out_type, uint64_t ld_out, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!half_type(type) || (out_type != type && out_type != KIMAD_VALUES_F32) || act > KIMAD_ACT_SILU || !linear_sizes_ok(M, N, K)) return KIMAD_ERR_INVALID_ARG;
    if (!matrix_ok(x, M, K, ld_x, 2, LD_MOST) || !matrix_ok(w, N, K, ld_w, 2, LD_MOST) || !matrix_ok(out, M, N, ld_out, type_bytes(out_type), OUT_LD_MOST)) return KIMAD_ERR_INVALID_ARG;
    if ((residual && !matrix_ok(residual, M, N, ld_residual, 2, OUT_LD_MOST)) || (z && !matrix_ok(z, M, N, ld_z, 2, OUT_LD_MOST)) || !aligned(bias, 2)) return KIMAD_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return KIMAD_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GemmArgs g{};
    g.M = M; g.N = N; g.K = K;
    g.end.out = out; g.end.ld = ld_out; g.end.bias = bias; g.end.residual = residual; g.end.ld_res = ld_residual; g.end.z = z; g.end.ld_z = ld_z; g.end.act = act;
    const bool out32 = out_type == KIMAD_VALUES_F32;
    if (K == 0) return with_half_type(type, [&](auto t) { return launch_none<decltype(t)::value>(M, N, g.end, out32, s); });
    Room room{static_cast<uint8_t*>(workspace), 0};
    const LinearRoom r = linear_room(room, x, ld_x, w, ld_w, M, N, K);
    if (room.used && (!workspace || workspace_bytes < room.used || !aligned(workspace, 16))) return KIMAD_ERR_WORKSPACE_TOO_SMALL;
    if (const int rc = copy_rows({x, ld_x, M, K, r.x}, {w, ld_w, N, K, r.w}, nullptr, 0, nullptr, nullptr, 0.f, s)) return rc;
    const Operand ox = operand(r.x, x, ld_x, M, K), ow = operand(r.w, w, ld_w, N, K);
    g.a = static_cast<const uint8_t*>(ox.p); g.lda = ox.ld; g.b = static_cast<const uint8_t*>(ow.p); g.ldb = ow.ld;
    if (r.plan.kind != GemmPlan::FEW) g.K = pitch_of(K);
    return with_half_type(type, [&](auto t) { return launch_gemm<decltype(t)::value, false, false>(g, r.plan, out32, r.parts, s); });
}

uint64_t kimad_linear_grad_workspace_bytes(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint64_t M, uint64_t N, uint64_t K, uint32_t act,
                                           uint32_t wants) {
    if (!linear_sizes_ok(M, N, K) || M == 0 || N == 0) return 0;
    Room room{nullptr, 0};
    linear_grad_room(room, dy, ld_dy, x, ld_x, w, ld_w, M, N, K, act, wants);
    return room.used;
}

int kimad_linear_grad(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, const void* z, uint64_t ld_z, uint32_t type, uint64_t M, uint64_t N,
                      uint64_t K, uint32_t act, void* dx, uint64_t ld_dx, void* dw, uint32_t dw_type, uint64_t ld_dw, float* db, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!half_type(type) || (dw && dw_type != type && dw_type != KIMAD_VALUES_F32) || act > KIMAD_ACT_SILU || !linear_sizes_ok(M, N, K)) return KIMAD_ERR_INVALID_ARG;
    if (!matrix_ok(dy, M, N, ld_dy, 2, LD_MOST) || (act != KIMAD_ACT_NONE && !matrix_ok(z, M, N, ld_z, 2, LD_MOST)) || !aligned(db, 4)) return KIMAD_ERR_INVALID_ARG;
    if (dx && (!matrix_ok(w, N, K, ld_w, 2, LD_MOST) || !matrix_ok(dx, M, K, ld_dx, 2, OUT_LD_MOST))) return KIMAD_ERR_INVALID_ARG;
    if (dw && (!matrix_ok(x, M, K, ld_x, 2, LD_MOST) || !matrix_ok(dw, N, K, ld_dw, type_bytes(dw_type), OUT_LD_MOST))) return KIMAD_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (M == 0 || N == 0) {                                                   // (sums over nothing)
        int rc = dx ? zeros(dx, type, M, K, ld_dx, s) : KIMAD_OK;
        if (!rc && dw) rc = zeros(dw, dw_type, N, K, ld_dw, s);
        return !rc && db ? zeros(db, KIMAD_VALUES_F32, 1, N, N, s) : rc;
    }
    if (K == 0) dx = dw = nullptr;
    Room room{static_cast<uint8_t*>(workspace), 0};
    const uint32_t wants = (dx ? KIMAD_WANT_DX : 0u) | (dw ? KIMAD_WANT_DW : 0u) | (db ? KIMAD_WANT_DB : 0u);
    const LinearGradRoom r = linear_grad_room(room, dy, ld_dy, x, ld_x, w, ld_w, M, N, K, act, wants);
    if (room.used && (!workspace || workspace_bytes < room.used || !aligned(workspace, 16))) return KIMAD_ERR_WORKSPACE_TOO_SMALL;
    if (const int rc = copy_rows({x, ld_x, M, K, r.x}, {w, ld_w, N, K, r.w}, nullptr, 0, nullptr, nullptr, 0.f, s)) return rc;
    const Operand odz = operand(r.dz, dy, ld_dy, M, N);
    const Operand ox = operand(r.x, x, ld_x, M, K), ow = operand(r.w, w, ld_w, N, K);
    if (r.dz_made || db) {
        ActGradArgs a{};
        a.dy = dy; a.z = act == KIMAD_ACT_NONE ? nullptr : z; a.dz = r.dz; a.M = M; a.N = N; a.ld_dy = ld_dy; a.ld_z = ld_z; a.pitch = pitch_of(N); a.act = act; a.rows = (uint32_t)r.sum_rows;
        a.lanes = 1;
        while (a.lanes < 64 && 8 * a.lanes < a.pitch) a.lanes *= 2;
        a.sums = db ? (r.sum_parts > 1 ? r.sums : db) : nullptr;
        const uint64_t gx = (a.pitch + SUM_COLS - 1) / SUM_COLS;
        const int rc = with_half_type(type, [&](auto t) {
            hipLaunchKernelGGL(k_act_grad<decltype(t)::value>, dim3((uint32_t)gx, (uint32_t)r.sum_parts), dim3(256), 0, s, a);
            return launched();
        });
        if (rc) return rc;
        if (r.sums) {
            hipLaunchKernelGGL(k_sum_join, dim3((uint32_t)((N + 63) / 64)), dim3(1024), 0, s, r.sums, r.sum_parts, N, db);
            if (const int rc2 = launched()) return rc2;
        }
    }
    if (dx) {
        GemmArgs g{};
        g.a = static_cast<const uint8_t*>(odz.p); g.lda = odz.ld; g.b = static_cast<const uint8_t*>(ow.p); g.ldb = ow.ld;
        g.M = M; g.N = K; g.K = pitch_of(N); g.k_rows_b = N;
        g.end.out = dx; g.end.ld = ld_dx;
        const int rc = with_half_type(type, [&](auto t) { return launch_gemm<decltype(t)::value, false, true>(g, r.dx, false, r.parts, s); });
        if (rc) return rc;
    }
    if (dw) {
        GemmArgs g{};
        g.a = static_cast<const uint8_t*>(odz.p); g.lda = odz.ld; g.b = static_cast<const uint8_t*>(ox.p); g.ldb = ox.ld;
        g.M = N; g.N = K; g.K = M; g.k_rows_a = M; g.k_rows_b = M;
        g.end.out = dw; g.end.ld = ld_dw;
        return with_half_type(type, [&](auto t) { return launch_gemm<decltype(t)::value, true, true>(g, r.dw, dw_type == KIMAD_VALUES_F32, r.parts, s); });
    }
    return KIMAD_OK;
}

uint64_t kimad_linear_xent_workspace_bytes(const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint32_t /* both types take the same */, uint64_t rows, uint64_t vocab, uint64_t dim, uint32_t wants,
                                           uint32_t dw_type) {
    if (!xent_sizes_ok(rows, vocab, dim) || rows == 0) return 0;
    Room room{nullptr, 0};
    xent_room(room, x, ld_x, w, ld_w, rows, vocab, dim, wants, dw_type);
    return room.used;
}

int kimad_linear_xent(const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, uint32_t type, uint64_t rows, uint64_t vocab, uint64_t dim, const int32_t* target,
                      const float* row_weight, float* loss, float* lse, void* dx, uint64_t ld_dx, void* dw, uint32_t dw_type, uint64_t ld_dw, void* workspace,
                      uint64_t workspace_bytes, void* stream) {
    if (!half_type(type) || (dw && dw_type != type && dw_type != KIMAD_VALUES_F32) || !xent_sizes_ok(rows, vocab, dim)) return KIMAD_ERR_INVALID_ARG;
    if (!matrix_ok(x, rows, dim, ld_x, 2, LD_MOST) || !matrix_ok(w, vocab, dim, ld_w, 2, LD_MOST)) return KIMAD_ERR_INVALID_ARG;
    if ((dx && !matrix_ok(dx, rows, dim, ld_dx, 2, OUT_LD_MOST)) || (dw && !matrix_ok(dw, vocab, dim, ld_dw, type_bytes(dw_type), OUT_LD_MOST))) return KIMAD_ERR_INVALID_ARG;
    if (!aligned(target, 4) || !aligned(row_weight, 4) || !aligned(loss, 4) || !aligned(lse, 4)) return KIMAD_ERR_INVALID_ARG;
    if (rows && (!target || (!loss && !lse && !dx && !dw))) return KIMAD_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t wants = (dx ? KIMAD_WANT_DX : 0u) | (dw ? KIMAD_WANT_DW : 0u);
    if (rows == 0) return dw ? zeros(dw, dw_type, vocab, dim, ld_dw, s) : KIMAD_OK;
    Room room{static_cast<uint8_t*>(workspace), 0};
    const XentRoom r = xent_room(room, x, ld_x, w, ld_w, rows, vocab, dim, wants, dw_type);
    if (!workspace || workspace_bytes < room.used || !aligned(workspace, 16)) return KIMAD_ERR_WORKSPACE_TOO_SMALL;
    if (const int rc = copy_rows({x, ld_x, rows, dim, r.x}, {w, ld_w, vocab, dim, r.w}, target, vocab, row_weight, r.scale, type == KIMAD_VALUES_F16 ? 4096.f : 1.f, s)) return rc;
    const Operand ox = operand(r.x, x, ld_x, rows, dim), ow = operand(r.w, w, ld_w, vocab, dim);
    const bool dw32 = dw_type == KIMAD_VALUES_F32;
    return with_half_type(type, [&](auto t) {
        constexpr uint32_t TYPE = decltype(t)::value;
        for (uint64_t p = 0; p < r.pieces; ++p) {
            const uint64_t row = p * r.piece, n = std::min(r.piece, rows - row);
            const auto& plan = r.plans[p + 1 == r.pieces];
            const uint32_t strip = plan.z.strip(), strips_row = (uint32_t)((vocab + strip - 1) / strip);
            GemmArgs g{};
            g.a = static_cast<const uint8_t*>(ox.p) + row * ox.ld * 2; g.lda = ox.ld; g.b = static_cast<const uint8_t*>(ow.p); g.ldb = ow.ld;
            g.M = n; g.N = vocab; g.K = plan.z.kind == GemmPlan::FEW ? dim : pitch_of(dim);
            g.soft.strips = r.strips; g.soft.e = r.e; g.soft.target = target + row; g.soft.picked = r.picked; g.soft.pitch = r.pitch; g.soft.strips_row = strips_row;
            if (const int rc = launch_kind<TYPE, false, false, END_SOFTMAX>(g, plan.z, s)) return rc;
            XentArgs a{};
            a.strips = r.strips; a.picked = r.picked; a.target = target + row; a.weight = row_weight ? row_weight + row : nullptr;
            a.loss = loss ? loss + row : nullptr; a.lse = lse ? lse + row : nullptr; a.rows_out = r.rows_out; a.e = r.e; a.scale = r.scale;
            a.rows = n; a.pitch = r.pitch; a.vocab = (uint32_t)vocab; a.strips_row = strips_row; a.strip = strip;
            hipLaunchKernelGGL(k_xent_rows, dim3((uint32_t)n), dim3(256), 0, s, a);
            if (const int rc = launched()) return rc;
            if (!wants) continue;
            const uint64_t chunks = (r.pitch + 2047) / 2048;
            hipLaunchKernelGGL(k_xent_gradient<TYPE>, dim3((uint32_t)(n * chunks)), dim3(256), 0, s, a, (uint32_t)chunks);
            if (const int rc = launched()) return rc;
            if (dx) {
                GemmArgs d{};
                d.a = reinterpret_cast<const uint8_t*>(r.e); d.lda = r.pitch; d.b = static_cast<const uint8_t*>(ow.p); d.ldb = ow.ld;
                d.M = n; d.N = dim; d.K = r.pitch; d.k_rows_b = vocab;
                d.end.out = static_cast<uint8_t*>(dx) + row * ld_dx * 2; d.end.ld = ld_dx; d.end.scale = r.scale + 1;
                if (const int rc = launch_gemm<TYPE, false, true>(d, plan.dx, false, r.parts, s)) return rc;
            }
            if (dw) {
                GemmArgs d{};
                d.a = reinterpret_cast<const uint8_t*>(r.e); d.lda = r.pitch; d.b = static_cast<const uint8_t*>(ox.p) + row * ox.ld * 2; d.ldb = ox.ld;
                d.M = vocab; d.N = dim; d.K = n; d.k_rows_a = n; d.k_rows_b = n;
                d.end.scale = r.scale + 1;
                // the pieces' sums in fp32, in dw itself where it is
                void* sum = dw32 ? dw : r.sum;
                const uint64_t ld_sum = dw32 ? ld_dw : dim;
                const bool last = p + 1 == r.pieces;
                if (p) { d.end.residual = sum; d.end.ld_res = ld_sum; d.end.res32 = 1; }
                d.end.out = last ? dw : sum; d.end.ld = last ? ld_dw : ld_sum;
                if (const int rc = launch_gemm<TYPE, true, true>(d, plan.dw, dw32 || !last, r.parts, s)) return rc;
            }
        }
        return (int)KIMAD_OK;
    });
}

int kimad_dropout(const void* x, uint32_t type, uint64_t rows, uint64_t cols, uint64_t ld, const void* residual, uint64_t ld_residual, double p, uint64_t seed, uint64_t offset, void* out,
                  uint64_t ld_out, void* stream) {
    if (type > KIMAD_VALUES_BF16 || rows > MOST || cols > MOST || (cols && rows > MOST / cols) || !(p >= 0.0 && p <= 1.0)) return KIMAD_ERR_INVALID_ARG;
    const uint64_t bytes = type_bytes(type);
    if (!matrix_ok(x, rows, cols, ld, bytes, MOST) || !matrix_ok(out, rows, cols, ld_out, bytes, MOST) || (residual && !matrix_ok(residual, rows, cols, ld_residual, bytes, MOST)))
        return KIMAD_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return KIMAD_OK;
    DropoutArgs a{};
    a.x = x; a.residual = residual; a.out = out; a.rows = rows; a.cols = cols; a.ld = ld; a.ld_res = ld_residual; a.ld_out = ld_out;
    a.key[0] = (uint32_t)seed; a.key[1] = (uint32_t)(seed >> 32); a.offset[0] = (uint32_t)offset; a.offset[1] = (uint32_t)(offset >> 32);
    a.border = (uint32_t)std::floor(65536.0 * p + 0.5);
    a.scale = a.border == 65536 ? 0.f : (float)(65536.0 / (65536.0 - (double)a.border));
    const bool flat = rows == 1 || (ld == cols && ld_out == cols && (!residual || ld_residual == cols));
    if (flat) { a.cols *= a.rows; a.rows = 1; }
    const uint64_t wgs = ((rows * cols + 7) / 8 + 255) / 256;
    if (!grid_ok(wgs, 256)) return KIMAD_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto go = [&](auto t) {
        constexpr uint32_t TYPE = decltype(t)::value;
        if (flat) hipLaunchKernelGGL((k_dropout<TYPE, false>), dim3((uint32_t)wgs), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_dropout<TYPE, true>), dim3((uint32_t)wgs), dim3(256), 0, s, a);
        return launched();
    };
    return type == KIMAD_VALUES_F32 ? go(std::integral_constant<uint32_t, TYPE_F32>{}) : with_half_type(type, go);
}

}  // extern "C"
