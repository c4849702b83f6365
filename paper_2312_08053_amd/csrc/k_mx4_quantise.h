// Quantisation to microscaled 4-bit floats along rows, or along rows and columns at once, and reading back.
// x [R, C] -> codes [R, 64 W] bytes, scales [W, R] words, W = ceil(C / 128); the columns' form is that of the transpose.
#pragma once
#include "mx4.h"

namespace kimad {

constexpr uint32_t QROWS = 16, QWORDS = 8;    // rows and words of a workgroup's share
constexpr uint32_t QU = 4;                   // words of a lane under way together

// Along rows: a workgroup takes 16 rows of up to eight words.  Its sixteen groups of sixteen lanes walk row by row through the share, so
// that reads and codes run on without gaps; the scale words, whose neighbours in memory are other rows' words, are collected in LDS
// and leave in runs of 16.  Bound by memory: 50257 x 768
// in fp32 40 us, 4.4 TB/s, 8192 x 2048 in bfloat16 9.7 us.  (Shares of 4, 8, 16 and 64 words, 256 x 2048: 3.0, 5.4, 6.8 and 6.8 us; 8192 x 2048: 11.2, 9.7, 10.0, 10.0.)
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_quantise_rows(const void* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ld,
                                                           uint64_t W, uint32_t* __restrict__ codes, uint32_t* __restrict__ scales) {
    __shared__ uint32_t s_scale[QWORDS * QROWS];
    const uint64_t row0 = (uint64_t)blockIdx.x * QROWS, word0 = (uint64_t)blockIdx.y * QWORDS;
    const uint32_t nr = (uint32_t)(rows - row0 < QROWS ? rows - row0 : QROWS), nw = (uint32_t)(W - word0 < QWORDS ? W - word0 : QWORDS);
    const uint32_t lane16 = threadIdx.x & 15u, units = nr * nw;
    for (uint32_t u0 = threadIdx.x >> 4; u0 < units; u0 += 16u * QU) {
        Raw8<TYPE> raw[QU];
#pragma unroll
        for (uint32_t i = 0; i < QU; ++i) {
            const uint32_t u = u0 + 16u * i, r = u / nw, w = u - r * nw;
            const uint64_t col = (word0 + w) * MX4_WORD + 8u * lane16;
            raw[i] = load8_first<TYPE>(x, (row0 + r) * ld + col, u < units ? (int64_t)cols - (int64_t)col : 0);
        }
#pragma unroll
        for (uint32_t i = 0; i < QU; ++i) {
            const uint32_t u = u0 + 16u * i, r = u / nw, w = u - r * nw;
            if (u >= units) break;
            float v[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) v[k] = raw[i].at(k);
            uint32_t byte;
            const uint32_t c = mx4_encode8(v, byte);
            codes[((row0 + r) * W + word0 + w) * 16u + lane16] = c;
            const uint32_t sw = mx4_scale_word(byte, lane16);
            if (lane16 == 0) s_scale[w * QROWS + r] = sw;
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < nw * QROWS; i += 256u) {
        const uint32_t w = i / QROWS, r = i % QROWS;
        if (r < nr) scales[(word0 + w) * rows + row0 + r] = s_scale[i];
    }
}

// Along columns, and along rows from the same read where `codes` is given: a workgroup holds a tile of 128 by 128 in LDS.  Behind every 32
// rows sixteen words are left out: a wave then reads sixteen columns of four blocks of rows from 64 different banks, and
// writes the 64 bytes of a column's word side by side.  Bound by memory: 50257 x 768 in fp32, both ways, 48 us, 4.1 TB/s.
constexpr uint32_t QT_PITCH = 128;
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_quantise_both(const void* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t W,
                                                           uint64_t WT, uint32_t* __restrict__ codes, uint32_t* __restrict__ scales,
                                                           uint32_t* __restrict__ codes_t, uint32_t* __restrict__ scales_t) {
    using E = std::conditional_t<TYPE == TYPE_F32, uint32_t, uint16_t>;
    constexpr uint32_t SKEW = 64 / sizeof(E);
    __shared__ __attribute__((aligned(16))) E tile[128 * QT_PITCH + 4 * SKEW];
    __shared__ uint32_t s_scale[128];
    const uint64_t w = blockIdx.x, wt = blockIdx.y;
    const uint64_t row0 = wt * 128, col0 = w * 128;
    const uint32_t lane16 = threadIdx.x & 15u, g = threadIdx.x >> 4;
    Raw8<TYPE> raw[8];
    const int64_t have = (int64_t)cols - (int64_t)(col0 + 8u * lane16);
#pragma unroll
    for (uint32_t p = 0; p < 8; ++p) {
        const uint64_t row = row0 + 16u * p + g;
        raw[p] = load8_first<TYPE>(x, row * ld + col0 + 8u * lane16, row < rows ? have : 0);
    }
#pragma unroll
    for (uint32_t p = 0; p < 8; ++p) {
        const uint32_t r = 16u * p + g;
        u32x4* to = reinterpret_cast<u32x4*>(tile + r * QT_PITCH + (r / 32u) * SKEW + 8u * lane16);
        to[0] = u32x4{raw[p].r[0], raw[p].r[1], raw[p].r[2], raw[p].r[3]};
        if (TYPE == TYPE_F32) to[1] = u32x4{raw[p].r[4 % (sizeof(raw[p].r) / 4)], raw[p].r[5 % (sizeof(raw[p].r) / 4)], raw[p].r[6 % (sizeof(raw[p].r) / 4)], raw[p].r[7 % (sizeof(raw[p].r) / 4)]};
    }
    if (codes) {
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) {
            const uint32_t r = 16u * p + g;
            float v[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) v[k] = raw[p].at(k);
            uint32_t byte;
            const uint32_t c = mx4_encode8(v, byte);
            if (row0 + r < rows) codes[((row0 + r) * W + w) * 16u + lane16] = c;
            const uint32_t sw = mx4_scale_word(byte, lane16);
            if (lane16 == 0) s_scale[r] = sw;
        }
    }
    __syncthreads();
    if (codes && threadIdx.x < 128u && row0 + threadIdx.x < rows) scales[w * rows + row0 + threadIdx.x] = s_scale[threadIdx.x];
    const uint32_t b = threadIdx.x & 3u;         // block of 32 rows
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
        const uint32_t c = (threadIdx.x >> 2) + 64u * half;
        const E* from = tile + 32u * b * QT_PITCH + b * SKEW + c;
        uint32_t bits[32], a = 0;
#pragma unroll
        for (uint32_t k = 0; k < 32; ++k) {
            const uint32_t e = from[k * QT_PITCH];
            bits[k] = TYPE == TYPE_F32 ? e : TYPE == TYPE_BF16 ? e << 16 : __float_as_uint(half_to_float(e));
            const uint32_t m = bits[k] & 0x7FFFFFFFu;
            a = a > m ? a : m;
        }
        const uint32_t byte = mx4_scale_byte(a);
        const float s = mx4_scale(byte);
        u32x4 out;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            uint32_t o = 0;
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(bits[8 * k]), __uint_as_float(bits[8 * k + 1]), s, 0);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(bits[8 * k + 2]), __uint_as_float(bits[8 * k + 3]), s, 1);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(bits[8 * k + 4]), __uint_as_float(bits[8 * k + 5]), s, 2);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(bits[8 * k + 6]), __uint_as_float(bits[8 * k + 7]), s, 3);
            out[k] = byte == 255u ? 0u : o;
        }
        uint32_t sw = byte << (8u * b);
        sw |= dpp_u32<DPP_XOR1>(sw);
        sw |= dpp_u32<DPP_XOR2>(sw);
        if (col0 + c < cols) {
            *reinterpret_cast<u32x4*>(codes_t + ((col0 + c) * WT + wt) * 16u + 4u * b) = out;
            if (b == 0) scales_t[wt * cols + col0 + c] = sw;
        }
    }
}

// Reading back: the same shares as along rows.  Bound by memory: 50257 x 768 into bfloat16 16.7 us, 5.8 TB/s (30 us with one word of a lane under way).
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_dequantise(const uint32_t* __restrict__ codes, const uint32_t* __restrict__ scales, uint64_t rows,
                                                        uint64_t cols, uint64_t W, void* __restrict__ out, uint64_t ld) {
    __shared__ uint32_t s_scale[QWORDS * QROWS];
    const uint64_t row0 = (uint64_t)blockIdx.x * QROWS, word0 = (uint64_t)blockIdx.y * QWORDS;
    const uint32_t nr = (uint32_t)(rows - row0 < QROWS ? rows - row0 : QROWS), nw = (uint32_t)(W - word0 < QWORDS ? W - word0 : QWORDS);
    const uint32_t lane16 = threadIdx.x & 15u, units = nr * nw;
    for (uint32_t i = threadIdx.x; i < nw * QROWS; i += 256u) {
        const uint32_t w = i / QROWS, r = i % QROWS;
        if (r < nr) s_scale[i] = scales[(word0 + w) * rows + row0 + r];
    }
    uint32_t c[QU];
    auto fetch = [&](uint32_t u0) {
#pragma unroll
        for (uint32_t i = 0; i < QU; ++i) {
            const uint32_t u = u0 + 16u * i, r = u / nw, w = u - r * nw;
            c[i] = u < units ? codes[((row0 + r) * W + word0 + w) * 16u + lane16] : 0u;
        }
    };
    fetch(threadIdx.x >> 4);
    __syncthreads();
    for (uint32_t u0 = threadIdx.x >> 4; u0 < units; u0 += 16u * QU) {
        if (u0 >= 16u * QU) fetch(u0);
#pragma unroll
        for (uint32_t i = 0; i < QU; ++i) {
            const uint32_t u = u0 + 16u * i, r = u / nw, w = u - r * nw;
            if (u >= units) break;
            const uint64_t col = (word0 + w) * MX4_WORD + 8u * lane16;
            float v[8];
            mx4_decode8(c[i], (s_scale[w * QROWS + r] >> (8u * (lane16 >> 2))) & 255u, v);
            store8_first<TYPE>(out, (row0 + r) * ld + col, (int64_t)cols - (int64_t)col, v);
        }
    }
}

}  // namespace kimad
