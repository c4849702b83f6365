// A round's update in microscaled 4-bit floats: the worker's side, q = round(g - h) and h <- h + q, and the server's, the same
// addition on its copies and the model's step.  The layers' words lie one after another: layer i begins at word
// floor(layer_start[i] / 128) + i, which leaves room for every layer's last, partly filled word (at most one word between two
// layers is empty, and holds zeros).
#pragma once
#include "mx4.h"

namespace kimad {

constexpr uint32_t UPDATE_LDS_L = 1023;      // layers whose starts are kept in LDS

// Where a group of sixteen lanes stands among the layers.
struct LayerWalk {
    const uint64_t* start;                   // in LDS, or in memory where there are too many layers
    uint32_t L, i;
    uint64_t first, next, lo, hi;            // words and elements of layer i
    __device__ __forceinline__ uint64_t word_of(uint32_t k) const { return start[k] / MX4_WORD + k; }
    __device__ __forceinline__ void take(uint32_t k) {
        i = k;
        lo = start[k]; hi = start[k + 1];
        first = lo / MX4_WORD + k; next = hi / MX4_WORD + k + 1;
    }
    __device__ __forceinline__ void find(uint64_t w) {   // the last layer that begins at or before word w
        uint32_t a = 0, b = L;
        while (b - a > 1) {
            const uint32_t mid = (a + b) >> 1;
            if (word_of(mid) <= w) a = mid; else b = mid;
        }
        take(a);
    }
    __device__ __forceinline__ void advance(uint64_t w) {
        while (w >= next && i + 1 < L) take(i + 1);
    }
};

// Starts that do not run from 0 to d without a step back would lead outside the buffers: every workgroup looks at all of them.
__device__ __forceinline__ bool starts_fit(const uint64_t* __restrict__ layer_start, uint32_t L, uint64_t d, uint64_t* s_start, int* s_bad) {
    if (threadIdx.x == 0) *s_bad = 0;
    __syncthreads();
    int mine = 0;
    for (uint32_t i = threadIdx.x; i <= L; i += 256u) {
        const uint64_t a = layer_start[i];
        if (L <= UPDATE_LDS_L) s_start[i] = a;
        if ((i == 0 && a != 0) || (i < L && layer_start[i + 1] < a) || (i == L && a != d)) mine = 1;
    }
    if (mine) *s_bad = 1;
    __syncthreads();
    return *s_bad == 0;
}

// Each workgroup walks a run of words, sixteen at a time.  Reads g and h once (8 bytes an element), writes h and 4.25 bits.
__global__ __launch_bounds__(256) void k_mx4_compress(const float* __restrict__ g, float* h, const uint64_t* __restrict__ layer_start, uint32_t L,
                                                      uint64_t d, uint64_t words, uint64_t share, uint32_t* __restrict__ codes,
                                                      uint32_t* __restrict__ scales, int32_t* status_out, int32_t err) {
    __shared__ uint64_t s_start[UPDATE_LDS_L + 1];
    __shared__ int s_bad;
    const bool fit = starts_fit(layer_start, L, d, s_start, &s_bad);
    if (status_out && blockIdx.x == 0 && threadIdx.x == 0) *status_out = fit ? 0 : err;
    if (!fit) return;
    const uint64_t begin = (uint64_t)blockIdx.x * share, end = begin + share < words ? begin + share : words;
    const uint32_t lane16 = threadIdx.x & 15u;
    uint64_t w = begin + (threadIdx.x >> 4);
    if (w >= end) return;
    LayerWalk at;
    at.start = L <= UPDATE_LDS_L ? s_start : layer_start;
    at.L = L;
    at.find(w);
    for (; w < end; w += 16u) {
        at.advance(w);
        const uint64_t e = at.lo + (w - at.first) * MX4_WORD + 8u * lane16;
        const int64_t n = (int64_t)(at.hi - e);
        const Raw8<TYPE_F32> gr = load8_first<TYPE_F32>(g, e, n, 0u), hr = load8_first<TYPE_F32>(h, e, n, 0u);
        float x[8], q[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) x[k] = gr.at(k) - hr.at(k);
        uint32_t byte;
        const uint32_t c = mx4_encode8(x, byte);
        codes[w * 16u + lane16] = c;
        const uint32_t sw = mx4_scale_word(byte, lane16);
        if (lane16 == 0) scales[w] = sw;
        mx4_decode8(c, byte, q);
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) q[k] = hr.at(k) + q[k];
        store8_first<TYPE_F32>(h, e, n, q);
    }
}

constexpr uint32_t UPDATE_MAX_WORKERS = 16;  // must equal KIMAD_MAX_WORKERS of the public header
struct Mx4ServerArgs {
    const uint32_t* codes[UPDATE_MAX_WORKERS];
    const uint32_t* scales[UPDATE_MAX_WORKERS];
    float* u_hat[UPDATE_MAX_WORKERS];
    double w[UPDATE_MAX_WORKERS];
    uint32_t M, L;
    uint64_t d, words, share;
    const uint64_t* layer_start;
    float* x;
    double gamma;
};
// One pass over everything: the workers' words, their estimators read and written, and the model's step from the values at hand.  The sum in
// fp64 in the workers' order, as in k_server_step.
__global__ __launch_bounds__(256) void k_mx4_server(Mx4ServerArgs a, int32_t* status_out, int32_t err) {
    __shared__ uint64_t s_start[UPDATE_LDS_L + 1];
    __shared__ int s_bad;
    const bool fit = starts_fit(a.layer_start, a.L, a.d, s_start, &s_bad);
    if (status_out && blockIdx.x == 0 && threadIdx.x == 0) *status_out = fit ? 0 : err;
    if (!fit) return;
    const uint64_t begin = (uint64_t)blockIdx.x * a.share, end = begin + a.share < a.words ? begin + a.share : a.words;
    const uint32_t lane16 = threadIdx.x & 15u;
    uint64_t w = begin + (threadIdx.x >> 4);
    if (w >= end) return;
    LayerWalk at;
    at.start = a.L <= UPDATE_LDS_L ? s_start : a.layer_start;
    at.L = a.L;
    at.find(w);
    for (; w < end; w += 16u) {
        at.advance(w);
        const uint64_t e = at.lo + (w - at.first) * MX4_WORD + 8u * lane16;
        const int64_t n = (int64_t)(at.hi - e);
        if (n <= 0) continue;
        Raw8<TYPE_F32> xr{};
        if (a.x) xr = load8_first<TYPE_F32>(a.x, e, n, 0u);
        double sum[8] = {};
#pragma unroll
        for (uint32_t m = 0; m < UPDATE_MAX_WORKERS; ++m) {
            if (m < a.M) {
                const Raw8<TYPE_F32> ur = load8_first<TYPE_F32>(a.u_hat[m], e, n, 0u);
                const uint32_t c = a.codes[m][w * 16u + lane16], byte = (a.scales[m][w] >> (8u * (lane16 >> 2))) & 255u;
                float q[8];
                mx4_decode8(c, byte, q);
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) {
                    q[k] = ur.at(k) + q[k];
                    sum[k] = sum[k] + a.w[m] * (double)q[k];
                }
                store8_first<TYPE_F32>(a.u_hat[m], e, n, q);
            }
        }
        if (a.x) {
            float r[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) r[k] = (float)((double)xr.at(k) - a.gamma * sum[k]);
            store8_first<TYPE_F32>(a.x, e, n, r);
        }
    }
}

}  // namespace kimad
