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

// Starts that do not run from 0 to d without a step back would lead outside the buffers: every workgroup looks at all of them.  `lined`: they are all
// multiples of 32, so that in buffers that begin on a cache line every layer does.
struct StartsRoom {
    uint64_t start[UPDATE_LDS_L + 1];
    uint32_t bad, lined;
};
__device__ __forceinline__ bool starts_fit(const uint64_t* __restrict__ layer_start, uint32_t L, uint64_t d, StartsRoom& room) {
    if (threadIdx.x == 0) { room.bad = 0; room.lined = 1; }
    __syncthreads();
    bool bad = false, lined = true;
    for (uint32_t i = threadIdx.x; i <= L; i += 256u) {
        const uint64_t a = layer_start[i];
        if (L <= UPDATE_LDS_L) room.start[i] = a;
        if ((i == 0 && a != 0) || (i < L && layer_start[i + 1] < a) || (i == L && a != d)) bad = true;
        if (i < L && a % 32 != 0) lined = false;
    }
    if (bad) room.bad = 1;
    if (!lined) room.lined = 0;
    __syncthreads();
    return room.bad == 0;
}

// Nontemporal accesses (NT below) where layers begin on cache lines and the buffers are too large for the device's cache to hold them until the next call (us with
// ordinary and with nontemporal accesses, entries of a model and workers):
//   compression   20 M 42, 47       120 M 304, 283
//   server   1    20 M 59, 72       120 M 443, 415
//            4     6 M 42, 48        20 M 155, 161     120 M 1047, 987
//            8     6 M 73, 87        20 M 313, 289      30 M  479, 432
//           16     1 M 35, 42         6 M 182, 163      30 M  909, 819
// Layers that begin elsewhere share lines between words, which are then fetched and written twice (120 M: 304, 353; 443, 550; 1047, 1411).
inline bool update_streams(uint64_t bytes) { return bytes > (384ull << 20); }

// A lane's part of a word: elements 4 l and on of its first half (blocks 0 and 1) and of its second (2 and 3), so that sixteen lanes read and write 256
// bytes side by side.  n: elements of the layer from the word's first one on.
template <bool NT>
struct Half4 {
    float v[2][4];
    __device__ __forceinline__ void load(const float* p, int64_t n, uint32_t lane16) {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const int64_t at = 64 * h + 4 * lane16;
            if (at + 4 <= n) {
                const f32x4_any* from = reinterpret_cast<const f32x4_any*>(p + at);
                const f32x4 q = NT ? __builtin_nontemporal_load(from) : *from;
                v[h][0] = q.x; v[h][1] = q.y; v[h][2] = q.z; v[h][3] = q.w;
            } else {
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) v[h][k] = at + k < n ? p[at + k] : 0.f;
            }
        }
    }
    __device__ __forceinline__ void store(float* p, int64_t n, uint32_t lane16) const {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const int64_t at = 64 * h + 4 * lane16;
            f32x4_any* to = reinterpret_cast<f32x4_any*>(p + at);
            const f32x4 q = {v[h][0], v[h][1], v[h][2], v[h][3]};
            if (at + 4 <= n) {
                if (NT) __builtin_nontemporal_store(q, to);
                else *to = q;
            } else
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    if (at + k < n) p[at + k] = v[h][k];
        }
    }
};

struct Mx4CompressArgs {
    const float* g;
    float* h;
    const uint64_t* layer_start;
    uint64_t d, words, share;
    uint16_t* codes;
    uint32_t* scales;
    uint32_t L, streams;         // streams: nontemporal accesses if the layers' starts allow
};
template <bool NT>
__device__ __forceinline__ void compress_words(const Mx4CompressArgs& a, LayerWalk at, uint64_t w, uint64_t end) {
    const uint32_t lane16 = threadIdx.x & 15u;
    for (; w < end; w += 16u) {
        at.advance(w);
        const uint64_t e = at.lo + (w - at.first) * MX4_WORD;
        const int64_t n = (int64_t)(at.hi - e);
        Half4<NT> gv, hv;
        gv.load(a.g + e, n, lane16);
        hv.load(a.h + e, n, lane16);
        uint32_t c[2], byte[2];
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) {
            float x[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) x[k] = gv.v[t][k] - hv.v[t][k];
            c[t] = mx4_encode4(x, byte[t]);
            mx4_decode4(c[t], byte[t], x);
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) hv.v[t][k] = hv.v[t][k] + x[k];
            a.codes[w * 32u + 16u * t + lane16] = (uint16_t)c[t];
        }
        uint32_t sw = (byte[0] | byte[1] << 16) << (lane16 & 8u);
        sw |= dpp_u32<DPP_ROR8>(sw);
        if (lane16 == 0) a.scales[w] = sw;
        hv.store(a.h + e, n, lane16);
    }
}
// Each workgroup walks a run of words, sixteen at a time.  Reads g and h once (8 bytes an element), writes h and 4.25 bits.  Bound by memory: 124 M entries
// 292 us, 5.3 TB/s.
__global__ __launch_bounds__(256) void k_mx4_compress(Mx4CompressArgs a, int32_t* status_out, int32_t err) {
    __shared__ StartsRoom room;
    const bool fit = starts_fit(a.layer_start, a.L, a.d, room);
    if (status_out && blockIdx.x == 0 && threadIdx.x == 0) *status_out = fit ? 0 : err;
    if (!fit) return;
    const uint64_t begin = (uint64_t)blockIdx.x * a.share, end = begin + a.share < a.words ? begin + a.share : a.words, w = begin + (threadIdx.x >> 4);
    if (w >= end) return;
    LayerWalk at;
    at.start = a.L <= UPDATE_LDS_L ? room.start : a.layer_start;
    at.L = a.L;
    at.find(w);
    if (a.streams && room.lined) compress_words<true>(a, at, w, end);
    else compress_words<false>(a, at, w, end);
}

constexpr uint32_t UPDATE_MAX_WORKERS = 16;  // must equal KIMAD_MAX_WORKERS of the public header
struct Mx4ServerArgs {
    const uint16_t* codes[UPDATE_MAX_WORKERS];
    const uint32_t* scales[UPDATE_MAX_WORKERS];
    float* u_hat[UPDATE_MAX_WORKERS];
    double w[UPDATE_MAX_WORKERS];
    uint32_t M, L, streams;
    uint64_t d, words, share;
    const uint64_t* layer_start;
    float* x;
    double gamma;
};
template <bool NT>
__device__ __forceinline__ void server_words(const Mx4ServerArgs& a, LayerWalk at, uint64_t w, uint64_t end) {
    constexpr uint32_t G = 2;    // workers whose reads are under way together (one: 431, 634 and 1055 us for 1, 2 and 4 workers of 120 M entries, two: 401, 610 and 1027, four: 433, 620 and 1039)
    const uint32_t lane16 = threadIdx.x & 15u;
    for (; w < end; w += 16u) {
        at.advance(w);
        const uint64_t e = at.lo + (w - at.first) * MX4_WORD;
        const int64_t n = (int64_t)(at.hi - e);
        if (n <= 0) continue;
        Half4<NT> xv;
        if (a.x) xv.load(a.x + e, n, lane16);
        double sum[2][4] = {};
#pragma unroll
        for (uint32_t m0 = 0; m0 < UPDATE_MAX_WORKERS; m0 += G) {
            if (m0 < a.M) {
                Half4<NT> u[G];
                uint32_t sw[G], c[G][2];
#pragma unroll
                for (uint32_t i = 0; i < G; ++i)
                    if (m0 + i < a.M) {
                        u[i].load(a.u_hat[m0 + i] + e, n, lane16);
                        sw[i] = a.scales[m0 + i][w];
#pragma unroll
                        for (uint32_t t = 0; t < 2; ++t) c[i][t] = a.codes[m0 + i][w * 32u + 16u * t + lane16];
                    }
#pragma unroll
                for (uint32_t i = 0; i < G; ++i)
                    if (m0 + i < a.M) {
#pragma unroll
                        for (uint32_t t = 0; t < 2; ++t) {
                            float q[4];
                            mx4_decode4(c[i][t], (sw[i] >> (16u * t + (lane16 & 8u))) & 255u, q);
#pragma unroll
                            for (uint32_t k = 0; k < 4; ++k) {
                                u[i].v[t][k] = u[i].v[t][k] + q[k];
                                sum[t][k] = sum[t][k] + a.w[m0 + i] * (double)u[i].v[t][k];
                            }
                        }
                        u[i].store(a.u_hat[m0 + i] + e, n, lane16);
                    }
            }
        }
        if (a.x) {
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) xv.v[t][k] = (float)((double)xv.v[t][k] - a.gamma * sum[t][k]);
            xv.store(a.x + e, n, lane16);
        }
    }
}

// One pass over everything: the workers' words, their estimators read and written, and the model's step from the values at hand.  The sum in
// fp64 in the workers' order, as in k_server_step.  Bound by memory: 124 M entries of one worker 422 us, of four 1094 (4.8 TB/s, off cache lines), on lines 987 for 120 M.
__global__ __launch_bounds__(256) void k_mx4_server(Mx4ServerArgs a, int32_t* status_out, int32_t err) {
    __shared__ StartsRoom room;
    const bool fit = starts_fit(a.layer_start, a.L, a.d, room);
    if (status_out && blockIdx.x == 0 && threadIdx.x == 0) *status_out = fit ? 0 : err;
    if (!fit) return;
    const uint64_t begin = (uint64_t)blockIdx.x * a.share, end = begin + a.share < a.words ? begin + a.share : a.words, w = begin + (threadIdx.x >> 4);
    if (w >= end) return;
    LayerWalk at;
    at.start = a.L <= UPDATE_LDS_L ? room.start : a.layer_start;
    at.L = a.L;
    at.find(w);
    if (a.streams && room.lined) server_words<true>(a, at, w, end);
    else server_words<false>(a, at, w, end);
}

}  // namespace kimad
