// Softmax cross entropy of a linear head without its logits.  With z = x W^T, lse_r = ln sum_v exp(z_rv) and p = exp(z - lse),
//     loss_r = w_r (lse_r - z_{r, t_r}),   G = w (p - onehot(t)),   dx = G W,   dW = G^T x.
// The product z goes by tiles (k_gemm.h) whose end is END_SOFTMAX: of a strip of a row's columns (32 or 64; 16 where k_gemm_few makes them) only its largest sum m and
// s = sum exp(z - m) are kept, and for a gradient e = exp(z - m) in 16 bits (SmallFloat, whose rounding is below the type's), of a piece of the rows at a time.  With lse known, e
// becomes G in its place, e exp(m - lse) w, in the type of the products; lse stays in two parts, the largest logit and what is beside it, so that G is as near at any size of the
// logits.  At the target, where p - 1 may be much smaller than p, it is taken from the fp32 logit.  A second product for z in the place of e would cost 2 R V D operations more; e
// costs 4 bytes of traffic an element.  G is rounded to the type, for dw in fp32 too: the matrix cores take 16 bits, and a second product of what the rounding leaves would double
// two thirds of the operations (8192 x 50257 x 768 in bfloat16 against 64 bits: 0.0017 of the gradients' norm, which is their own rounding, with G in fp32 as with G in 16 bits).
#pragma once
#include "k_linear.h"

namespace kimad {

struct XentArgs {
    const f32x2* strips;
    const float* picked;
    const int32_t* target;
    const float* weight;         // or null: 1
    float *loss, *lse;           // or null
    f32x4* rows_out;             // [rows]: the largest logit, ln of the sum of exponentials of differences from it, the row's weight times `scale` (0: the row does not count)
    void* e;                     // [rows, pitch]: exp(z - m) as a SmallFloat, and then G
    const float* scale;          // two numbers on the device: what G is multiplied by, and its inverse (k_rows_copy)
    uint64_t rows, pitch;
    uint32_t vocab, strips_row, strip;
};

// A row's sums from its strips, by a workgroup: the loss and lse.
__global__ __launch_bounds__(256) void k_xent_rows(XentArgs a) {
    __shared__ Softmax room[4];
    const uint64_t row = blockIdx.x;
    const int32_t t = a.target[row];
    const float w = a.weight ? a.weight[row] : 1.f;
    bool live = (uint32_t)t < a.vocab && w != 0.f;
    Softmax q = {-INFINITY, 0.f};
    if (live) {
        for (uint32_t i = threadIdx.x; i < a.strips_row; i += 256) {
            const f32x2 v = a.strips[row * a.strips_row + i];
            q = join(q, Softmax{v[0], v[1]}, LOG2E);
        }
        q = join_block<256>(q, LOG2E, room);
        live = q.s != 0.f;                                                    // (every logit -Inf: the row leaves nothing)
    }
    if (threadIdx.x) return;
    const float log_s = logf(q.s);
    if (a.loss) a.loss[row] = live ? w * ((q.m - a.picked[row]) + log_s) : 0.f;
    if (a.lse) a.lse[row] = live ? q.m + log_s : 0.f;
    // (lse in its two parts: as one number it is off by |lse| 2^-24, and every probability by as much of itself)
    if (a.rows_out) a.rows_out[row] = f32x4{q.m, log_s, live ? w * a.scale[0] : 0.f, 0.f};
}

// e becomes G.  A thread takes eight columns.  Bound by memory.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_xent_gradient(XentArgs a, uint32_t chunks) {
    const uint64_t row = blockIdx.x / chunks;
    const uint64_t col = ((uint64_t)(blockIdx.x % chunks) * 256 + threadIdx.x) * 8;
    if (col >= a.pitch) return;
    const f32x4 of = a.rows_out[row];
    u32x4* at = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.e) + row * a.pitch + col);
    const bool live = of[2] != 0.f && col < a.vocab;
    u32x4 out = {0u, 0u, 0u, 0u};
    if (live) {
        const u32x4 w = *at;
        const float m = a.strips[row * a.strips_row + col / a.strip][0], f = __builtin_amdgcn_exp2f(((m - of[0]) - of[1]) * LOG2E) * of[2];
        const float fe = f * SmallFloat<TYPE>::TO_E;
        const uint32_t t = (uint32_t)a.target[row] - (uint32_t)col;
        float v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = col + k < a.vocab ? SmallFloat<TYPE>::at(w[k / 2], k % 2) * fe : 0.f;
        if (t < 8) {
            const float p = expm1f((a.picked[row] - of[0]) - of[1]) * of[2];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                if (t == k) v[k] = p;
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) out[k] = pack2<TYPE>(v[2 * k], v[2 * k + 1]);
    }
    *at = out;
}

}  // namespace kimad
