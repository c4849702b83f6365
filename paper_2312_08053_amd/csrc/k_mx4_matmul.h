// Product of two matrices of microscaled 4-bit floats, C [M, N] = A [M, K] B [N, K]^T, sums in fp32.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of A by 16 of B over a word: lane l holds block l / 16 of row l % 16 (16 bytes of
// codes) and that block's scale byte, of A and of B; element i of the result's lane l is C[4 (l / 16) + i][l % 16].
#pragma once
#include "mx4.h"

namespace kimad {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mx4_mfma(u32x4 a, u32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
    const i32x8 va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, 0, sa, 0, sb);
}

// Four waves, a tile of 16 by 16 each.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_matmul(const u32x4* __restrict__ a, const uint32_t* __restrict__ sa, uint64_t M,
                                                    const u32x4* __restrict__ b, const uint32_t* __restrict__ sb, uint64_t N, uint64_t W,
                                                    void* __restrict__ out, uint64_t ld) {
    const uint32_t lane = threadIdx.x & 63u, r = lane & 15u, blk = lane >> 4;
    const uint64_t m0 = (uint64_t)blockIdx.y * 16, n0 = ((uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16;
    if (n0 >= N) return;
    const uint64_t m = m0 + r < M ? m0 + r : M - 1, n = n0 + r < N ? n0 + r : N - 1;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (uint64_t w = 0; w < W; ++w)
        acc = mx4_mfma(a[(m * W + w) * 4 + blk], b[(n * W + w) * 4 + blk], acc, (sa[w * M + m] >> (8 * blk)) & 255u, (sb[w * N + n] >> (8 * blk)) & 255u);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        if (m0 + 4 * blk + i < M && n0 + r < N) store1<TYPE>(out, (m0 + 4 * blk + i) * ld + n0 + r, acc[i]);
}

}  // namespace kimad
