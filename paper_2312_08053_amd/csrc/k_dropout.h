// Dropout from a counter-based generator, y = r + keep x / (1 - p): no mask is stored, the backward pass makes it again from the same numbers.
// Philox 4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of two 32-bit products whose halves
// are crossed.  A block's 128 bits serve eight elements: 16 bits decide one as well as 32 at p in steps of 2^-16, and with 32 the ten rounds, some 40 products
// at a quarter of the rate, would take longer than 16-bit elements do from memory.
#pragma once
#include "mx4.h"

namespace kimad {

struct DropoutArgs {
    const void *x, *residual;    // residual: or null
    void* out;
    uint64_t rows, cols, ld, ld_res, ld_out;
    uint32_t key[2], offset[2];  // the seed, and the counter's upper half
    uint32_t border;             // an element is dropped where its 16 bits are below
    float scale;
};

__device__ __forceinline__ u32x4 philox(uint64_t block, const DropoutArgs& a) {
    u32x4 c = {(uint32_t)block, (uint32_t)(block >> 32), a.offset[0], a.offset[1]};
    uint32_t k0 = a.key[0], k1 = a.key[1];
#pragma unroll
    for (uint32_t r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c[0] * 0xD2511F53u, q = (uint64_t)c[2] * 0xCD9E8D57u;
        c = u32x4{(uint32_t)(q >> 32) ^ c[1] ^ k0, (uint32_t)q, (uint32_t)(p >> 32) ^ c[3] ^ k1, (uint32_t)p};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// A thread takes eight elements, counted along the rows.  ROWS false: one row.
template <uint32_t TYPE, bool ROWS>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
    const uint64_t block = (uint64_t)blockIdx.x * 256 + threadIdx.x, n = a.rows * a.cols;
    if (8 * block >= n) return;
    uint64_t r = 0, c = 8 * block;
    if (ROWS) {
        if (n >> 32) { r = c / a.cols; c = c % a.cols; }
        else { r = (uint32_t)c / (uint32_t)a.cols; c = (uint32_t)c % (uint32_t)a.cols; }
    }
    auto one = [&](float x, uint32_t h, bool res, float y) {
        const float v = h < a.border ? 0.f : x * a.scale;
        return res ? v + y : v;
    };
    if (c + 8 <= a.cols) {
        const Raw8<TYPE> x = load8<TYPE>(a.x, r * a.ld + c);
        Raw8<TYPE> y;
        if (a.residual) y = load8<TYPE>(a.residual, r * a.ld_res + c);
        const u32x4 w = philox(block, a);
        float v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = one(x.at(k), w[k / 2] >> (16 * (k % 2)) & 0xFFFFu, a.residual, a.residual ? y.at(k) : 0.f);
        store8<TYPE>(a.out, r * a.ld_out + c, v);
        return;
    }
    const u32x4 w = philox(block, a);
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        if (8 * block + k >= n) return;
        const float y = a.residual ? load1<TYPE>(a.residual, r * a.ld_res + c) : 0.f;
        store1<TYPE>(a.out, r * a.ld_out + c, one(load1<TYPE>(a.x, r * a.ld + c), w[k / 2] >> (16 * (k % 2)) & 0xFFFFu, a.residual, y));
        if (++c == a.cols) { c = 0; ++r; }
    }
}

}  // namespace kimad
