// A linear layer's products beside the tiles of k_gemm.h: few rows, rows laid out anew, and what its gradient is made of.
#pragma once
#include "k_distill.h"
#include "k_gemm.h"

namespace kimad {

// Eight 16-bit elements at a time of a row that may begin at any of them.  SHIFTED: from the one or two whole 16 bytes that they lie in, by selections and shifts; loads from
// addresses off 16 bytes take longer (one row by 32000 x 2049 64 us, so 36, and 20 where rows lie at such addresses).  (Whole 16 bytes with an element of the row are never of another page.)
template <bool SHIFTED>
struct RowReader {
    const uint8_t* at;
    uint32_t shift;              // bytes from a 16-byte address to the row's first element
    __device__ __forceinline__ void begin(const uint8_t* p) {
        shift = SHIFTED ? (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) : 0u;
        at = p - shift;
    }
    struct Raw {
        u32x4 v[SHIFTED ? 2 : 1];
    };
    __device__ __forceinline__ Raw load(uint64_t i) const {                   // i: a multiple of 8
        Raw r;
        const u32x4* q = reinterpret_cast<const u32x4*>(at + 2 * i);
        r.v[0] = q[0];
        if constexpr (SHIFTED) r.v[1] = q[shift ? 1 : 0];
        return r;
    }
    __device__ __forceinline__ u32x4 words(const Raw& r) const {
        if constexpr (!SHIFTED) return r.v[0];
        else {
            // (by masks: of selections the compiler makes addresses)
            const uint32_t by4 = shift & 4u ? ~0u : 0u, by8 = shift & 8u ? ~0u : 0u;
            uint32_t d[8], t[7], u[5];
            u32x4 out;
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) d[k] = r.v[k / 4][k % 4];
#pragma unroll
            for (uint32_t k = 0; k < 7; ++k) t[k] = (d[k + 1] & by4) | (d[k] & ~by4);
#pragma unroll
            for (uint32_t k = 0; k < 5; ++k) u[k] = (t[k + 2] & by8) | (t[k] & ~by8);
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) out[k] = __builtin_amdgcn_alignbyte(u[k + 1], u[k], shift & 2u);
            return out;
        }
    }
    __device__ __forceinline__ u32x4 first(uint64_t i, int64_t n) const {     // the first n of them, the others zeros
        const Raw8<TYPE_BF16> v = load8_first<TYPE_BF16>(at + shift, i, n);
        return u32x4{v.r[0], v.r[1], v.r[2], v.r[3]};
    }
};

// Few rows of A (16 MT at most): sixteen rows of B by a workgroup, whose waves take a quarter of K each, straight from memory to registers, U times 32 of K
// under way.  SHIFTED: rows may begin anywhere.  Bound by the reads of B.
template <uint32_t TYPE, uint32_t MT, uint32_t END, bool SHIFTED>
__global__ __launch_bounds__(256) void k_gemm_few(GemmArgs g) {
    __shared__ f32x4 s_part[3][MT][64];
    constexpr uint32_t U = MT == 1 ? 8 : MT == 2 ? 4 : 2;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, blk = lane >> 4;
    const uint64_t n0 = (uint64_t)blockIdx.x * 16, n = n0 + r < g.N ? n0 + r : g.N - 1;
    // (whole cache lines)
    const uint64_t quarter = (g.K + 255) / 256 * 64, begin = wave * quarter < g.K ? wave * quarter : g.K, end = begin + quarter < g.K ? begin + quarter : g.K;
    RowReader<SHIFTED> b, a[MT];
    b.begin(g.b + 2 * n * g.ldb);
    f32x4 acc[MT];
#pragma unroll
    for (uint32_t t = 0; t < MT; ++t) {
        a[t].begin(g.a + 2 * (16 * t + r < g.M ? 16 * t + r : g.M - 1) * g.lda);
        acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    uint64_t k = begin;
    for (; k + 32 * U <= end; k += 32 * U) {
        typename RowReader<SHIFTED>::Raw vb[U], va[U][MT];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            vb[u] = b.load(k + 32 * u + 8 * blk);
#pragma unroll
            for (uint32_t t = 0; t < MT; ++t) va[u][t] = a[t].load(k + 32 * u + 8 * blk);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t t = 0; t < MT; ++t) acc[t] = mfma16<TYPE>(a[t].words(va[u][t]), b.words(vb[u]), acc[t]);
    }
    for (; k < end; k += 32) {
        const int64_t left = (int64_t)(end - k) - 8 * blk;
        const u32x4 vb = b.first(k + 8 * blk, left);
#pragma unroll
        for (uint32_t t = 0; t < MT; ++t) acc[t] = mfma16<TYPE>(a[t].first(k + 8 * blk, left), vb, acc[t]);
    }
    if (wave)
#pragma unroll
        for (uint32_t t = 0; t < MT; ++t) s_part[wave - 1][t][lane] = acc[t];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (uint32_t t = 0; t < MT; ++t) {
        acc[t] = acc[t] + s_part[0][t][lane] + s_part[1][t][lane] + s_part[2][t][lane];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint64_t m = 16 * t + 4 * blk + i;
            const bool in = m < g.M && n0 + r < g.N;
            if constexpr (END == END_SOFTMAX) {
                // sixteen lanes have a row's strip of sixteen columns
                const SoftmaxEnd& o = g.soft;
                if (in && (uint64_t)(int64_t)o.target[m] == n0 + r) o.picked[m] = acc[t][i];
                const float x = in ? acc[t][i] : -INFINITY;
                Softmax v = {x, x == -INFINITY ? 0.f : 1.f + (x - x)};            // (of +Inf and NaN a NaN)
#pragma unroll
                for (uint32_t h = 1; h < 16; h <<= 1) v = join(v, Softmax{__shfl_xor(v.m, h), __shfl_xor(v.s, h)}, LOG2E);
                if (r == 0 && m < g.M) o.strips[m * o.strips_row + blockIdx.x] = f32x2{v.m, v.s};
            } else if (in) {
                const GemmEnd& o = g.end;
                float v = acc[t][i] + (o.bias ? load1<TYPE>(o.bias, n) : 0.f);
                if (o.z) store1<TYPE>(o.z, m * o.ld_z + n, v);
                v = act_of(v, o.act);
                if (o.residual) v += load1<TYPE>(o.residual, m * o.ld_res + n);
                store1<END == END_F32 ? TYPE_F32 : TYPE>(o.out, m * o.ld + n, v);
            }
        }
    }
}

// A product over nothing: its end alone.
template <uint32_t TYPE, bool OUT32>
__global__ __launch_bounds__(256) void k_gemm_none(uint64_t M, uint64_t N, GemmEnd o) {
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < M * N; i += (uint64_t)gridDim.x * 256) {
        const uint64_t m = i / N, n = i % N;
        float v = o.bias ? load1<TYPE>(o.bias, n) : 0.f;
        if (o.z) store1<TYPE>(o.z, m * o.ld_z + n, v);
        v = act_of(v, o.act);
        if (o.residual) v += load1<TYPE>(o.residual, m * o.ld_res + n);
        store1<OUT32 ? TYPE_F32 : TYPE>(o.out, m * o.ld + n, v);
    }
}

// Rows of 16-bit elements laid out anew, `pitch` (a multiple of 8) apart and filled up with zeros: for operands whose rows do not begin at 16-byte addresses or
// end inside 16 bytes.  Rows that do not count (weight 0, no target) become zeros: a NaN there would reach every sum over rows.  Two matrices in one launch.
struct CopyArgs {
    const void* from[2];
    void* to[2];                 // or null
    uint64_t ld[2], rows[2], cols[2], pitch[2];
    uint32_t wgs0;               // workgroups of the first
    const int32_t* target;       // of the first matrix's rows, or null
    const float* weight;
    uint32_t vocab;
    float* scale;                // two numbers, or null
    float largest;               // what the largest weight is to become
};
// The cross entropy's G in 16 bits holds w / max |w| times `largest`: equal weights, however many rows share one, then cost no rounding that is the same for all rows, and
// fp16's small numbers reach further.  (By one workgroup; weights that are not finite leave nothing finite anyway.)
__device__ __forceinline__ void scale_of_weights(const CopyArgs& a) {
    __shared__ float s_max[4];
    float m = 0.f;
#pragma unroll 8
    for (uint64_t r = threadIdx.x; r < a.rows[0]; r += 256) {
        const float w = a.weight ? fabsf(a.weight[r]) : 1.f;
        m = fmaxf(m, (uint32_t)a.target[r] < a.vocab && w < INFINITY ? w : 0.f);
    }
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if ((threadIdx.x & 63u) == 0) s_max[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x) return;
    m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    m = m == 0.f ? 1.f : fmaxf(m, 0x1p-100f);
    a.scale[0] = a.largest / m;
    a.scale[1] = m / a.largest;
}
__global__ __launch_bounds__(256) void k_rows_copy(CopyArgs a) {
    if (a.scale && blockIdx.x + 1 == gridDim.x) {
        scale_of_weights(a);
        return;
    }
    const uint32_t which = blockIdx.x >= a.wgs0;
    const uint64_t each = a.pitch[which] / 8, i = (uint64_t)(blockIdx.x - (which ? a.wgs0 : 0)) * 256 + threadIdx.x;
    if (i >= a.rows[which] * each) return;
    const uint64_t r = i / each, c = i % each * 8;
    const bool live = which || ((!a.target || (uint32_t)a.target[r] < a.vocab) && (!a.weight || a.weight[r] != 0.f));
    const Raw8<TYPE_BF16> v = load8_first<TYPE_BF16>(a.from[which], r * a.ld[which] + c, live ? (int64_t)(a.cols[which] - c) : 0);
    reinterpret_cast<u32x4*>(a.to[which])[i] = u32x4{v.r[0], v.r[1], v.r[2], v.r[3]};
}

// dz = dy act'(z), rounded to the type, and the sums of its columns in fp32 (of what was not rounded): of 64 rows a workgroup (128, if there are no more), 512 columns.  Bound by memory.
// (Rounded for dw in fp32 too: the matrix cores take 16 bits, and a second product of what the rounding leaves would double both.  8192 x 5632 x 2048 in bfloat16 against 64 bits: 0.0023 of the
// gradients' norm, 0.0017 with dz in fp32.)
constexpr uint32_t SUM_ROWS = 64, SUM_COLS = 512;
struct ActGradArgs {
    const void *dy, *z;          // z null: no activation
    void* dz;                    // or null; pitch elements from row to row, filled up with zeros
    float* sums;                 // [ceil(M / rows)][N], or null
    uint64_t M, N, ld_dy, ld_z, pitch;
    uint32_t act, rows, lanes;   // rows of a workgroup; lanes of a row, a power of two, 8 columns each
};
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_act_grad(ActGradArgs a) {
    __shared__ float s_sum[4 * SUM_COLS];
    // (a wave takes 64 / lanes rows at a time: of narrow matrices several)
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, per = 64u / a.lanes, group = wave * per + lane / a.lanes, at = lane % a.lanes;
    const uint64_t c = (uint64_t)blockIdx.x * SUM_COLS + 8 * at, m0 = (uint64_t)blockIdx.y * a.rows, m1 = m0 + a.rows < a.M ? m0 + a.rows : a.M;
    const int64_t n = (int64_t)a.N - (int64_t)c;
    float sum[8] = {};
    constexpr uint32_t U = 4;                            // rows of a lane under way together
    if (c < a.pitch)
        with_act(a.z ? a.act : (uint32_t)ACT_NONE, [&](auto kind) {
            constexpr uint32_t ACT = decltype(kind)::value;
            for (uint64_t m = m0 + group; m < m1; m += 4 * per * U) {
                Raw8<TYPE> g[U], z[U];
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) {
                    const uint64_t r = m + 4 * per * u < m1 ? m + 4 * per * u : m;
                    g[u] = load8_first<TYPE>(a.dy, r * a.ld_dy + c, n);
                    if (ACT != ACT_NONE) z[u] = load8_first<TYPE>(a.z, r * a.ld_z + c, n);
                }
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) {
                    if (m + 4 * per * u >= m1) break;
                    float v[8];
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k) v[k] = ACT == ACT_NONE ? g[u].at(k) : (int64_t)k < n ? g[u].at(k) * slope_as<ACT>(z[u].at(k)) : 0.f;
                    if (a.dz) store8<TYPE>(a.dz, (m + 4 * per * u) * a.pitch + c, v);
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k) sum[k] += v[k];
                }
            }
        });
    if (!a.sums) return;
    const uint32_t cols = 8 * a.lanes;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) s_sum[group * cols + 8 * at + k] = sum[k];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < cols; i += 256) {
        const uint64_t col = (uint64_t)blockIdx.x * SUM_COLS + i;
        float v = 0.f;
        for (uint32_t q = 0; q < 4 * per; ++q) v += s_sum[q * cols + i];
        if (col < a.N) a.sums[blockIdx.y * a.N + col] = v;
    }
}
// The sums of all rows from the workgroups': 64 columns a workgroup, whose sixteen waves take every sixteenth part.
__global__ __launch_bounds__(1024) void k_sum_join(const float* __restrict__ sums, uint64_t parts, uint64_t N, float* __restrict__ out) {
    __shared__ float s_sum[16][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t n = (uint64_t)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (n < N)
#pragma unroll 8
        for (uint64_t p = wave; p < parts; p += 16) v += sums[p * N + n];
    s_sum[wave][lane] = v;
    __syncthreads();
    if (wave || n >= N) return;
#pragma unroll
    for (uint32_t i = 1; i < 16; ++i) v += s_sum[i][lane];
    out[n] = v;
}

}  // namespace kimad
