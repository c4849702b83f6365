// C ABI of the operators beside a round: argument checks and kernel launches.  Declarations and contracts are in include/kimad.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "operators_host.h"
#include "k_mx4_quantise.h"
#include "k_mx4_matmul.h"
#include "k_mx4_update.h"
#include "k_distill.h"

namespace {

using namespace kimad;

static_assert(TYPE_F32 == KIMAD_VALUES_F32 && TYPE_F16 == KIMAD_VALUES_F16 && TYPE_BF16 == KIMAD_VALUES_BF16, "header and kernel constants");

static_assert(UPDATE_MAX_WORKERS == KIMAD_MAX_WORKERS, "header and kernel constants");

constexpr uint64_t FEW_ROWS = 32;                        // products of so many rows may go by k_mx4_matmul_few
constexpr uint64_t MATMUL_MOST_K = 1ull << 25, MATMUL_MOST_LD = 1ull << 24;     // eight rows of codes and 32 rows of the result are reached by 32-bit offsets
constexpr uint32_t UPDATE_MOST_L = 0x7FFFFFFFu;          // layers of an update: the kernels count them, and search among them, in 32 bits
inline uint64_t words_of(uint64_t cols) { return (cols + MX4_WORD - 1) / MX4_WORD; }
// codes and scales are both given or both missing
inline bool pair_ok(const void* codes, const uint32_t* scales) {
    return !codes == !scales && (!codes || (aligned(codes, 16) && aligned(scales, 4)));
}

// Calls f with the type as a compile-time constant.
template <class F>
inline int with_type(uint32_t type, F f) {
    if (type == KIMAD_VALUES_F32) return f(std::integral_constant<uint32_t, TYPE_F32>{});
    if (type == KIMAD_VALUES_F16) return f(std::integral_constant<uint32_t, TYPE_F16>{});
    return f(std::integral_constant<uint32_t, TYPE_BF16>{});
}

// Workgroups and the run of words that each of them takes: runs of at least 16, and at most eight workgroups a compute unit.
inline uint32_t update_grid(uint64_t words, uint64_t& share) {
    const uint64_t wgs = std::min<uint64_t>((words + 15) / 16, 2048);
    share = ((words + wgs - 1) / wgs + 15) / 16 * 16;
    return (uint32_t)((words + share - 1) / share);
}

}  // namespace

namespace {

// Rows that no workgroup's registers hold go by chunks, in two launches.  (Shorter ones do not, however few they are: one row of 9000 elements 11 us by chunks
// and 7 whole, of 32000 10 and 9.6, of 50257 10.4 and 11.9, the loss alone 9.1 and 6.6 to 8.2; 64 rows of 32000 12 and 10.5, of 50257 13.5 and 13.2.)
constexpr uint64_t DISTILL_ROW_MOST = 65536 - 7;         // (a row that begins off a 16-byte address takes a group more)
inline uint32_t distill_chunks(uint64_t vocab) { return (uint32_t)((vocab + 7 + 8 * DISTILL_CHUNK - 1) / (8 * DISTILL_CHUNK)); }
inline bool distill_by_chunks(uint64_t vocab) { return vocab > DISTILL_ROW_MOST; }

int distill_args(DistillArgs& a, const void* logits, uint32_t type, uint64_t rows, uint64_t vocab, uint64_t ld, const uint32_t* t_idx,
                 const float* t_val, uint32_t k, float temperature, const float* row_weight, const float* loss, const float* stats, const void* grad,
                 uint64_t ld_grad) {
    if (type > KIMAD_VALUES_BF16 || vocab == 0 || vocab >= (1ull << 31) || rows > GRID_MOST || ld < vocab || k > DISTILL_MAX_K) return KIMAD_ERR_INVALID_ARG;
    if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return KIMAD_ERR_INVALID_ARG;
    if (rows && (!logits || !aligned(logits, type_bytes(type)) || (k && (!t_idx || !t_val)))) return KIMAD_ERR_INVALID_ARG;
    if (!aligned(t_idx, 4) || !aligned(t_val, 4) || !aligned(row_weight, 4) || !aligned(loss, 4) || !aligned(stats, 4)) return KIMAD_ERR_INVALID_ARG;
    if (grad && (ld_grad < vocab || !aligned(grad, type_bytes(type)))) return KIMAD_ERR_INVALID_ARG;
    if (distill_by_chunks(vocab) && !grid_ok(rows * distill_chunks(vocab), CHUNK_NT)) return KIMAD_ERR_INVALID_ARG;
    a.z = logits; a.idx = t_idx; a.val = t_val; a.weight = row_weight; a.grad = const_cast<void*>(grad);
    a.rows = rows; a.vocab = (uint32_t)vocab; a.ld = ld; a.ld_grad = ld_grad; a.k = k; a.bloom = distill_bloom(k);
    a.T = temperature; a.c = (float)(1.4426950408889634 / (double)temperature);
    a.chunks = distill_chunks(vocab);
    return KIMAD_OK;
}

template <uint32_t TYPE, uint32_t NT, uint32_t NV>
int launch_row(const DistillArgs& a, hipStream_t s) {
    if (!grid_ok(a.rows, NT)) return KIMAD_ERR_INVALID_ARG;
    if (a.grad) hipLaunchKernelGGL((k_distill_row<TYPE, NT, NV, true>), dim3((uint32_t)a.rows), dim3(NT), distill_lds(a.k), s, a);
    else hipLaunchKernelGGL((k_distill_row<TYPE, NT, NV, false>), dim3((uint32_t)a.rows), dim3(NT), distill_lds(a.k), s, a);
    return launched();
}

typedef MatmulTile<256, 256, 2, 4> Tile256;
typedef MatmulTile<128, 128, 2, 2> Tile128;
typedef MatmulTile<64, 64, 2, 2> Tile64;

// How a product is shared out: by the least of the times below, which are fits (us) to measurements of each tile alone on products of 256 to 50257 rows, 768 to
// 50257 columns and 6 to 128 words, most of them good to a tenth: rounds of as many tiles as compute units, of `stages` stages (pairs of words) each, and a last
// one that costs less the fewer units it fills.  Measured, and in the end here, into 32 bits (into 16):
//   M      N      K        256            128            64             here
//   512    2048   2048     20  (19)       11  (11)       7.1 (7.1)      7.1 (7.0)
//   1024   4096   4096     31  (30)       20  (18)       21  (20)       19  (17)
//   4096   768    16384    91  (91)       51  (50)       48  (48)       49  (48)
//   2048   5632   2048     24  (23)       32  (23)       28  (28)       25  (22)
//   8192   5632   2048     73  (62)       75  (69)       102 (100)      72  (62)
//   50257  768    8192     195 (182)      222 (205)      309 (296)      195 (182)
//   1000   50257  768      55  (44)       51  (43)       65  (63)       48  (43)
// Products of up to 32 rows (B's codes and scales not used just before, us; few: k_mx4_matmul_few, whose waves read all of A each):
//   M      N      K        few   64    128       M      N      K        few   64    128
//   8      32000  2048     10.0  11.6  14.1      8      50257  8192     49    52    52
//   16     32000  2048     11.0  11.7  14.1      16     50257  8192     58    52    52
//   32     32000  2048     14.8  11.9  14.3      32     50257  8192     83    55    53
//   32     5632   2048     5.9   7.8   11.1      32     8192   8192     15.2  17.7  17.8
// With few tiles and long sums the stages are shared out as well (64 x 8192 x 8192 19.6 and 15.1 us, 48 x 4096 x 16384 34 and 14.9),
// and the parts, which are of 32 bits, added by a second launch.  wide: a result of 32 bits.
struct MatmulPlan {
    enum { FEW, T64, T128, T256 } kind;
    uint64_t tiles_m, tiles_n;
    uint32_t splits, share;
    double us;
};
MatmulPlan matmul_plan(uint64_t M, uint64_t N, uint64_t W, bool wide, bool may_split) {
    MatmulPlan best{};
    best.splits = 1;
    const uint64_t stages = (W + 1) / 2;
    best.share = (uint32_t)stages;
    if (W == 0) return best;                                                  // (nothing to share out; such a product goes by none of these)
    const double read = 2.0 + (double)((M + N) * W) * 68.0 / 4.5e6;           // both operands from memory
    if (M <= FEW_ROWS) {
        best.kind = MatmulPlan::FEW;
        best.us = std::max(read, 2.2 + (double)(N * W) * 68.0 / 7.2e6 * (1.0 + (double)M / 28.0) + (double)(N * M) * 1.2e-6);
    }
    // of one tile: a stage with nothing beside it on its compute unit, what comes from beyond the L2; among others, where few units have one and where all do;
    // its end in 16 bits and in 32; the launch
    struct { decltype(best.kind) kind; uint64_t edge; double alone, lone, stage, end16, end32, launch; } const kinds[] = {
        {MatmulPlan::T256, 256, 1.3, 1.3, 1.95, 3.0, 6.0, 5.0}, {MatmulPlan::T128, 128, 0.69, 0.64, 0.64, 1.0, 1.5, 5.0}, {MatmulPlan::T64, 64, 0.45, 0.24, 0.24, 0.35, 0.35, 4.5}};
    for (const auto& k : kinds) {
        const uint64_t tm = (M + k.edge - 1) / k.edge, tn = (N + k.edge - 1) / k.edge;
        for (uint64_t splits = 1; splits == 1 || (may_split && splits <= 16 && 4 * splits <= stages && tm * tn * splits <= 4 * UNITS); splits *= 2) {
            const uint64_t share = (stages + splits - 1) / splits, parts = (stages + share - 1) / share;
            const uint64_t items = tm * tn * parts, rounds = items / UNITS;
            const double part = (double)(items % UNITS) / UNITS, end = wide || parts > 1 ? k.end32 : k.end16;
            double us = (double)rounds * ((double)share * k.stage + end) + k.launch;
            if (part > 0) us += (double)share * (k.lone + part * (k.stage - k.lone)) + end;
            if (parts > 1) us += 4.0 + (double)(parts * M * N) * 8.0 / 4e6;     // 4 bytes written and read, at 4 TB/s
            us = std::max(std::max(us, k.launch + (double)share * k.alone + end), read);
            if (best.us == 0 || us < best.us) {
                best.us = us;
                best.kind = k.kind; best.tiles_m = tm; best.tiles_n = tn;
                best.splits = (uint32_t)parts; best.share = (uint32_t)share;
            }
        }
    }
    return best;
}
// Tiles of 256 rows that leave at least three quarters of the compute units without work in their last round: so many of A's rows make whole rounds, the rest
// goes by a second launch, if both together are expected to take less (8704 x 4096 x 8192, an eighth of the units in the last round: 180 and 160 us; 9216, a
// quarter: 182 and 170; but 50257 x 768 x 8192, a third: 195 and 208).  0: one launch.
inline uint64_t matmul_first_rows(const MatmulPlan& p, uint64_t M, uint64_t N, uint64_t W, bool wide, MatmulPlan& rest) {
    const uint64_t tiles = p.tiles_m * p.tiles_n, rounds = tiles / UNITS;
    if (p.kind != MatmulPlan::T256 || p.splits != 1 || rounds == 0 || tiles % UNITS > UNITS / 4) return 0;
    const uint64_t rows = rounds * UNITS / p.tiles_n * 256;
    if (rows == 0 || rows >= M) return 0;
    rest = matmul_plan(M - rows, N, W, wide, false);
    const MatmulPlan first = matmul_plan(rows, N, W, wide, false);
    return first.kind == MatmulPlan::T256 && first.us + rest.us < p.us ? rows : 0;
}
inline uint64_t matmul_parts_bytes(const MatmulPlan& p, uint64_t M, uint64_t N) { return p.splits > 1 ? 4 * p.splits * M * N : 0; }

template <uint32_t TYPE, class T>
int launch_tile(MatmulArgs g, const MatmulPlan& p, hipStream_t s) {
    const uint64_t items = p.tiles_m * p.tiles_n * p.splits;
    if (items > GRID_MOST) return KIMAD_ERR_INVALID_ARG;
    constexpr uint64_t slots = UNITS * ((160 * 1024) / T::LDS);
    g.tiles_m = (uint32_t)p.tiles_m; g.tiles_n = (uint32_t)p.tiles_n; g.splits = p.splits; g.share = p.share;
    hipLaunchKernelGGL((k_mx4_matmul_tile<TYPE, T>), dim3((uint32_t)std::min<uint64_t>(items, slots)), dim3(64 * T::WAVES), 0, s, g);
    return launched();
}

// Sixteen rows of B by a wave where that makes a wave a SIMD and the sum is short, else by four (32000 rows, 16 words: 8.3 and 9.6 us; 16384 rows,
// 128 words: 33.7 and 27.5).
template <uint32_t TYPE, uint32_t MT>
int launch_few(const MatmulArgs& g, uint64_t groups, hipStream_t s) {
    if (groups >= 4 * UNITS && g.W <= 32) hipLaunchKernelGGL((k_mx4_matmul_few<TYPE, MT, false>), dim3((uint32_t)((groups + 3) / 4)), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((k_mx4_matmul_few<TYPE, MT, true>), dim3((uint32_t)groups), dim3(256), 0, s, g);
    return launched();
}

template <uint32_t TYPE>
int launch_kind(const MatmulArgs& g, const MatmulPlan& p, hipStream_t s) {
    if (p.kind == MatmulPlan::FEW) {
        const uint64_t groups = (g.N + 15) / 16;
        if (!grid_ok(groups, 256)) return KIMAD_ERR_INVALID_ARG;
        return g.M <= 16 ? launch_few<TYPE, 1>(g, groups, s) : launch_few<TYPE, 2>(g, groups, s);
    }
    if (p.kind == MatmulPlan::T256) return launch_tile<TYPE, Tile256>(g, p, s);
    if (p.kind == MatmulPlan::T128) return launch_tile<TYPE, Tile128>(g, p, s);
    return launch_tile<TYPE, Tile64>(g, p, s);
}

}  // namespace

extern "C" {

int kimad_mx4_quantise(const void* x, uint32_t type, uint64_t rows, uint64_t cols, uint64_t ld, void* codes, uint32_t* scales,
                       void* codes_t, uint32_t* scales_t, void* stream) {
    if (type > KIMAD_VALUES_BF16 || rows > MOST || cols > MOST || ld < cols || !pair_ok(codes, scales) || !pair_ok(codes_t, scales_t))
        return KIMAD_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return KIMAD_OK;
    if ((!codes && !codes_t) || !x || !aligned(x, type_bytes(type))) return KIMAD_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint64_t W = words_of(cols), WT = words_of(rows);
    if (codes_t) {
        if (!grid_ok(W, 256) || WT > GRID_Y_MOST) return KIMAD_ERR_INVALID_ARG;
        return with_type(type, [&](auto t) {
            hipLaunchKernelGGL(k_mx4_quantise_both<decltype(t)::value>, dim3((uint32_t)W, (uint32_t)WT), dim3(256), 0, s, x, rows, cols, ld, W, WT,
                               static_cast<uint32_t*>(codes), scales, static_cast<uint32_t*>(codes_t), scales_t);
            return launched();
        });
    }
    const uint64_t gx = (rows + QROWS - 1) / QROWS, gy = (W + QWORDS - 1) / QWORDS;
    if (!grid_ok(gx, 256) || gy > GRID_Y_MOST) return KIMAD_ERR_INVALID_ARG;
    return with_type(type, [&](auto t) {
        hipLaunchKernelGGL(k_mx4_quantise_rows<decltype(t)::value>, dim3((uint32_t)gx, (uint32_t)gy), dim3(256), 0, s, x, rows, cols, ld, W,
                           static_cast<uint32_t*>(codes), scales);
        return launched();
    });
}

int kimad_mx4_dequantise(const void* codes, const uint32_t* scales, uint64_t rows, uint64_t cols, void* out, uint32_t type,
                         uint64_t ld, void* stream) {
    if (type > KIMAD_VALUES_BF16 || rows > MOST || cols > MOST || ld < cols) return KIMAD_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return KIMAD_OK;
    if (!codes || !pair_ok(codes, scales) || !out || !aligned(out, type_bytes(type))) return KIMAD_ERR_INVALID_ARG;
    const uint64_t W = words_of(cols), gx = (rows + QROWS - 1) / QROWS, gy = (W + QWORDS - 1) / QWORDS;
    if (!grid_ok(gx, 256) || gy > GRID_Y_MOST) return KIMAD_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_type(type, [&](auto t) {
        hipLaunchKernelGGL(k_mx4_dequantise<decltype(t)::value>, dim3((uint32_t)gx, (uint32_t)gy), dim3(256), 0, s,
                           static_cast<const uint32_t*>(codes), scales, rows, cols, W, out, ld);
        return launched();
    });
}

uint64_t kimad_mx4_matmul_workspace_bytes(uint64_t M, uint64_t N, uint64_t K) {
    if (M > MOST || N > MOST || K > MATMUL_MOST_K || M == 0 || N == 0) return 0;
    return matmul_parts_bytes(matmul_plan(M, N, words_of(K), true, true), M, N);
}

int kimad_mx4_matmul(const void* a_codes, const uint32_t* a_scales, uint64_t M, const void* b_codes, const uint32_t* b_scales,
                     uint64_t N, uint64_t K, void* out, uint32_t type, uint64_t ld, void* workspace, uint64_t workspace_bytes,
                     void* stream) {
    if (type > KIMAD_VALUES_BF16 || M > MOST || N > MOST || K > MATMUL_MOST_K || ld < N || ld > MATMUL_MOST_LD) return KIMAD_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return KIMAD_OK;
    if (!out || !aligned(out, type_bytes(type))) return KIMAD_ERR_INVALID_ARG;
    if (K && (!a_codes || !b_codes || !pair_ok(a_codes, a_scales) || !pair_ok(b_codes, b_scales))) return KIMAD_ERR_INVALID_ARG;
    if (workspace && !aligned(workspace, 16)) return KIMAD_ERR_INVALID_ARG;
    MatmulArgs g{};
    g.a = static_cast<const uint8_t*>(a_codes); g.b = static_cast<const uint8_t*>(b_codes);
    MatmulPlan p = matmul_plan(M, N, words_of(K), type == KIMAD_VALUES_F32, true);
    if (matmul_parts_bytes(p, M, N) > (workspace ? workspace_bytes : 0)) p = matmul_plan(M, N, words_of(K), type == KIMAD_VALUES_F32, false);
    g.sa = a_scales; g.sb = b_scales; g.out = out; g.M = M; g.N = N; g.W = words_of(K); g.ld = ld; g.scale_rows = M;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_type(type, [&](auto t) {
        constexpr uint32_t TYPE = decltype(t)::value;
        if (K == 0) {
            if (M > MOST / N * 256 || !grid_ok((M * N + 255) / 256, 256)) return (int)KIMAD_ERR_INVALID_ARG;
            hipLaunchKernelGGL(k_mx4_matmul_none<TYPE>, dim3((uint32_t)((M * N + 255) / 256)), dim3(256), 0, s, out, M, N, ld);
            return launched();
        }
        MatmulPlan rest{};
        if (const uint64_t rows = matmul_first_rows(p, M, N, g.W, type == KIMAD_VALUES_F32, rest)) {
            MatmulArgs first = g;
            first.M = rows;
            MatmulPlan fp = p;
            fp.tiles_m = rows / 256;
            const int rc = launch_kind<TYPE>(first, fp, s);
            if (rc) return rc;
            g.a += rows * g.W * 64; g.sa += rows; g.M = M - rows;
            g.out = static_cast<uint8_t*>(out) + rows * ld * type_bytes(type);
            return launch_kind<TYPE>(g, rest, s);
        }
        if (p.splits == 1) return launch_kind<TYPE>(g, p, s);
        g.out = workspace; g.ld = N;
        const int rc = launch_kind<TYPE_F32>(g, p, s);
        if (rc) return rc;
        const uint64_t wgs = (M * N + 255) / 256;
        if (!grid_ok(wgs, 256)) return (int)KIMAD_ERR_INVALID_ARG;
        hipLaunchKernelGGL(k_mx4_matmul_join<TYPE>, dim3((uint32_t)wgs), dim3(256), 0, s, static_cast<const float*>(workspace), p.splits, M, N, out, ld);
        return launched();
    });
}

uint64_t kimad_mx4_update_words(uint32_t L, uint64_t d) { return d / MX4_WORD + L; }

int kimad_mx4_compress_ef(const float* g, float* h, const uint64_t* layer_start, uint32_t L, uint64_t d, void* codes,
                          uint32_t* scales, int32_t* status_out, void* stream) {
    if (!g || !h || !layer_start || L == 0 || L > UPDATE_MOST_L || d == 0 || d > MOST || !codes || !pair_ok(codes, scales) || !aligned(g, 4) || !aligned(h, 4) ||
        !aligned(layer_start, 8) || !aligned(status_out, 4))
        return KIMAD_ERR_INVALID_ARG;
    Mx4CompressArgs a{};
    a.g = g; a.h = h; a.layer_start = layer_start; a.L = L; a.d = d;
    a.codes = static_cast<uint16_t*>(codes); a.scales = scales;
    a.words = kimad_mx4_update_words(L, d);
    a.streams = aligned(g, 128) && aligned(h, 128) && update_streams(8 * d);
    const uint32_t wgs = update_grid(a.words, a.share);
    hipLaunchKernelGGL(k_mx4_compress, dim3(wgs), dim3(256), 0, static_cast<hipStream_t>(stream), a, status_out, (int32_t)KIMAD_ERR_BAD_OFFSETS);
    return launched();
}

int kimad_mx4_server_apply(const kimad_mx4_update_t* updates, float* const* u_hat, const double* weights, uint32_t M,
                           const uint64_t* layer_start, uint32_t L, uint64_t d, float* x, double gamma, int32_t* status_out,
                           void* stream) {
    if (!updates || !u_hat || !weights || !layer_start || M == 0 || M > KIMAD_MAX_WORKERS || L == 0 || L > UPDATE_MOST_L || d == 0 || d > MOST ||
        !aligned(x, 4) || !aligned(layer_start, 8) || !aligned(status_out, 4))
        return KIMAD_ERR_INVALID_ARG;
    Mx4ServerArgs a{};
    bool lined = true;
    for (uint32_t m = 0; m < M; ++m) {
        if (!updates[m].codes || !pair_ok(updates[m].codes, updates[m].scales) || !u_hat[m] || !aligned(u_hat[m], 4)) return KIMAD_ERR_INVALID_ARG;
        a.codes[m] = static_cast<const uint16_t*>(updates[m].codes);
        a.scales[m] = updates[m].scales;
        a.u_hat[m] = u_hat[m];
        a.w[m] = weights[m];
        lined = lined && aligned(u_hat[m], 128);
    }
    a.M = M; a.L = L; a.d = d; a.layer_start = layer_start; a.x = x; a.gamma = gamma;
    a.streams = lined && aligned(x, 128) && update_streams(4 * (M + 1) * d);
    a.words = kimad_mx4_update_words(L, d);
    const uint32_t wgs = update_grid(a.words, a.share);
    hipLaunchKernelGGL(k_mx4_server, dim3(wgs), dim3(256), 0, static_cast<hipStream_t>(stream), a, status_out, (int32_t)KIMAD_ERR_BAD_OFFSETS);
    return launched();
}

uint64_t kimad_distill_workspace_bytes(uint64_t rows, uint64_t vocab, uint32_t k) {
    return distill_by_chunks(vocab) ? 4 * rows * (2ull * distill_chunks(vocab) + k) : 0;
}

int kimad_distill(const void* logits, uint32_t type, uint64_t rows, uint64_t vocab, uint64_t ld, const uint32_t* t_idx,
                  const float* t_val, uint32_t k, float temperature, const float* row_weight, float* loss, float* stats,
                  void* grad, uint64_t ld_grad, void* workspace, uint64_t workspace_bytes, void* stream) {
    DistillArgs a{};
    const int rc = distill_args(a, logits, type, rows, vocab, ld, t_idx, t_val, k, temperature, row_weight, loss, stats, grad, ld_grad);
    if (rc || rows == 0) return rc;
    if (!loss && !stats && !grad) return KIMAD_ERR_INVALID_ARG;
    a.loss = loss; a.stats = stats;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint64_t need = kimad_distill_workspace_bytes(rows, vocab, k);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 4))) return KIMAD_ERR_WORKSPACE_TOO_SMALL;
    if (need) {
        a.parts = static_cast<float*>(workspace);
        a.zj = a.parts + 2 * rows * a.chunks;
        return with_type(type, [&](auto t) {
            constexpr uint32_t TYPE = decltype(t)::value;
            hipLaunchKernelGGL(k_distill_part<TYPE>, dim3((uint32_t)(rows * a.chunks)), dim3(CHUNK_NT), 0, s, a);
            if (hipGetLastError() != hipSuccess) return (int)KIMAD_ERR_HIP;
            if (a.grad) hipLaunchKernelGGL((k_distill_rest<TYPE, true, true>), dim3((uint32_t)(rows * a.chunks)), dim3(CHUNK_NT), distill_lds(k), s, a, a.chunks);
            else hipLaunchKernelGGL((k_distill_rest<TYPE, true, false>), dim3((uint32_t)rows), dim3(CHUNK_NT), distill_lds(k), s, a, 1u);
            return launched();
        });
    }
    return with_type(type, [&](auto t) {
        constexpr uint32_t TYPE = decltype(t)::value;
        const uint64_t groups = (vocab + 7 + 7) / 8;
        // Small workgroups with many groups a thread, for more of a row's phases run beside one another, as long as the registers leave two
        // workgroups a compute unit: loss and gradient, us, rows of 4000 elements by 64, 128 and 256 threads 35, 41, 51 (16 bits; 32 bits 62, 68, 69), of 8000
        // by 128 and 256 61, 64 (129, 114), of 12000 by 128 and 256 98, 87 (182, 167), of 32000 by 256 and 512 116, 109 (219, 208), of 50257 by 512 and
        // 1024 335, 402 (by 512 with 32 bits: scratch memory).  By 512 threads, up to ten groups a thread leave registers for a third workgroup, which
        // helps shorter rows: with room for 10 and for 16 groups a thread 8192 rows of 34000 elements 222, 249, of 36000 231, 250, of 38000 250, 266, of 40953 264, 273;
        // with room for 13 and for 16 of 42000 279, 279, of 44000 293, 287, of 48000 319, 309, of 53241 353, 330.
        constexpr bool WIDE = TYPE == TYPE_F32;
        if (groups <= 64) return launch_row<TYPE, 64, 1>(a, s);
        if (groups <= 128) return launch_row<TYPE, 64, 2>(a, s);
        if (groups <= 256) return launch_row<TYPE, 64, 4>(a, s);
        if (groups <= 512) return launch_row<TYPE, 64, 8>(a, s);
        if (groups <= 1024) return launch_row<TYPE, WIDE ? 256 : 128, WIDE ? 4 : 8>(a, s);
        if (groups <= 2048) return launch_row<TYPE, 256, 8>(a, s);
        if (groups <= 4096) return launch_row<TYPE, 512, 8>(a, s);
        if (!WIDE && groups <= 512 * 10) return launch_row<TYPE, WIDE ? 1024 : 512, WIDE ? 8 : 10>(a, s);
        return launch_row<TYPE, WIDE ? 1024 : 512, WIDE ? 8 : 16>(a, s);
    });
}

int kimad_distill_grad(const void* logits, uint32_t type, uint64_t rows, uint64_t vocab, uint64_t ld, const uint32_t* t_idx,
                       const float* t_val, uint32_t k, float temperature, const float* row_weight, const float* stats, void* grad,
                       uint64_t ld_grad, void* stream) {
    DistillArgs a{};
    const int rc = distill_args(a, logits, type, rows, vocab, ld, t_idx, t_val, k, temperature, row_weight, nullptr, stats, grad, ld_grad);
    if (rc || rows == 0) return rc;
    if (!stats || !grad || !grid_ok(rows * a.chunks, CHUNK_NT)) return KIMAD_ERR_INVALID_ARG;
    a.stats = const_cast<float*>(stats);
    return with_type(type, [&](auto t) {
        hipLaunchKernelGGL((k_distill_rest<decltype(t)::value, false, true>), dim3((uint32_t)(rows * a.chunks)), dim3(CHUNK_NT), distill_lds(k),
                           static_cast<hipStream_t>(stream), a, a.chunks);
        return launched();
    });
}

}  // extern "C"
