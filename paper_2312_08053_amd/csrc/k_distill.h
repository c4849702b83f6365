// Distillation from a teacher's top logits.  With q = softmax(z / T) over the vocabulary and p = softmax(t / T) over the
// teacher's k entries,
//     loss = w T^2 sum_j p_j (ln p_j - ln q_{idx_j}),      d loss / d z_v = w T (q_v - p_v).
// A row with weight 0, without an entry, or whose logits are all -Inf leaves nothing: loss, gradient and statistics are 0.
// The sums are fp32, the exponentials are taken of differences to the largest logit.
#pragma once
#include "mx4.h"

namespace kimad {

constexpr uint32_t DISTILL_MAX_K = 1024;

struct DistillArgs {
    const void* z;
    const uint32_t* idx;
    const float* val;
    const float* weight;         // or null: 1
    float* loss;                 // or null
    float* stats;                // [rows][2] or null: largest logit, sum of exp((z - largest) / T)
    void* grad;
    float* parts;                // split rows: [rows][chunks][2], the same two numbers of a chunk ...
    float* zj;                   // ... and [rows][k], the student's logits at the entries
    uint64_t rows, vocab, ld, ld_grad, chunk;
    uint32_t k, chunks, bloom;   // bloom: words of the table that finds indices given twice, a power of two
    float T, c;                  // c = log2(e) / T
};
// LDS that a workgroup asks for: index, p and student's logit of every entry, and the table.
__host__ __device__ inline uint32_t distill_bloom(uint32_t k) {
    uint32_t w = 32;
    while (w < k) w *= 2;
    return w;
}
inline uint32_t distill_lds(uint32_t k) { return 4u * (3u * k + distill_bloom(k)); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
template <uint32_t TYPE>
constexpr uint32_t minus_inf() { return TYPE == TYPE_F32 ? 0xFF800000u : TYPE == TYPE_F16 ? 0xFC00u : 0xFF80u; }

// The running pair of a softmax: m the largest, s the sum of exp((z - m) / T).  m is -Inf and s 0 while there is nothing but
// -Inf; a NaN stays in s.
struct Softmax {
    float m, s;
};
__device__ __forceinline__ Softmax join(Softmax a, Softmax b, float c) {
    const float m = fmaxf(a.m, b.m);
    // (the larger one's sum as it is: two of -Inf make no NaN)
    const float sa = a.m == m ? a.s : a.s * exp2_fast((a.m - m) * c), sb = b.m == m ? b.s : b.s * exp2_fast((b.m - m) * c);
    return {m, sa + sb};
}
// Over a workgroup's threads, the result in all of them.  `room` is free again behind the next barrier.
template <uint32_t NT>
__device__ __forceinline__ Softmax join_block(Softmax v, float c, Softmax* room) {
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) v = join(v, Softmax{__shfl_xor(v.m, o), __shfl_xor(v.s, o)}, c);
    if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (uint32_t i = 1; i < NT / 64; ++i) v = join(v, room[i], c);
    return v;
}
template <uint32_t NT>
__device__ __forceinline__ float sum_block(float v, float* room) {
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (uint32_t i = 1; i < NT / 64; ++i) v += room[i];
    return v;
}

template <uint32_t NT>
struct DistillRoom {
    Softmax teacher[NT / 64], row[NT / 64];
    float sum[NT / 64];
    uint32_t any, twice;
};

// A row's entries: indices (those beyond the vocabulary are none and become 0xFFFFFFFF), probabilities, and the student's logits
// unless they are given or those of other chunks' columns.  False where there is no entry.
// Entries of one index are one entry with the sum of their probabilities; it goes to the first of them, the others
// get 0xFFFFFFFF.  They are looked for only where two of the row's indices meet in the table.
template <uint32_t TYPE, uint32_t NT>
__device__ __forceinline__ bool read_teacher(const DistillArgs& a, uint64_t row, uint64_t from, uint64_t to, const float* zj, uint32_t* s_idx,
                                             float* s_p, float* s_z, uint32_t* s_table, DistillRoom<NT>& room) {
    const uint32_t k = a.k;
    if (threadIdx.x == 0) { room.any = 0; room.twice = 0; }
    for (uint32_t i = threadIdx.x; i < a.bloom; i += NT) s_table[i] = 0;
    __syncthreads();
    Softmax v = {-INFINITY, 0.f};
    bool any = false, meets = false;
    for (uint32_t j = threadIdx.x; j < k; j += NT) {
        const uint32_t i = a.idx[row * k + j];
        const bool in = i < a.vocab;
        const float t = in ? a.val[row * k + j] : -INFINITY;
        s_idx[j] = in ? i : 0xFFFFFFFFu;
        s_p[j] = t;
        s_z[j] = zj ? zj[row * k + j] : in && i >= from && i < to ? load1<TYPE>(a.z, row * a.ld + i) : 0.f;
        any = any || (in && t != -INFINITY);
        v = join(v, Softmax{t, t == -INFINITY ? 0.f : 1.f}, a.c);
        if (t != t) v.s = t;
        if (in) meets = meets || (atomicOr(&s_table[(i >> 5) & (a.bloom - 1u)], 1u << (i & 31u)) >> (i & 31u) & 1u);
    }
    if (any) room.any = 1;
    if (__syncthreads_or(meets)) {
        for (uint32_t j = threadIdx.x; j < k; j += NT)
            for (uint32_t l = 0; l < j; ++l)
                if (s_idx[l] == s_idx[j] && s_idx[j] != 0xFFFFFFFFu) room.twice = 1;
    }
    v = join_block<NT>(v, a.c, room.teacher);
    if (!room.any) return false;
    for (uint32_t j = threadIdx.x; j < k; j += NT) {
        const float t = s_p[j];
        s_p[j] = t == -INFINITY ? 0.f : exp2_fast((t - v.m) * a.c) / v.s;
    }
    __syncthreads();
    if (room.twice) {
        for (uint32_t j0 = 0; j0 < k; j0 += NT) {            // the sums, from untouched probabilities: s_z keeps its place, the table is free
            const uint32_t j = j0 + threadIdx.x;
            if (j < k && s_idx[j] != 0xFFFFFFFFu) {
                bool first = true;
                float p = 0.f;
                for (uint32_t l = 0; l < k; ++l)
                    if (s_idx[l] == s_idx[j]) { first = first && l >= j; p += s_p[l]; }
                s_table[j] = __float_as_uint(first ? p : -1.f);      // (no probability is negative)
            }
        }
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < k; j += NT)
            if (s_idx[j] != 0xFFFFFFFFu) {
                if (__uint_as_float(s_table[j]) == -1.f) { s_idx[j] = 0xFFFFFFFFu; s_p[j] = 0.f; }
                else s_p[j] = __uint_as_float(s_table[j]);
            }
        __syncthreads();
    }
    return true;
}

// T sum_j p_j (ln p_j - ln q_j) over the threads' entries; an entry with p = 0 adds nothing, whatever the student's logit.  (Times T, so
// that a logit of the type's lowest value overflows only where the loss does.)
template <uint32_t NT>
__device__ __forceinline__ float cross_terms(const DistillArgs& a, const uint32_t* s_idx, const float* s_p, const float* s_z, Softmax q) {
    const float log_s = logf(q.s);
    float sum = 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += NT) {
        const float p = s_p[j];
        if (s_idx[j] != 0xFFFFFFFFu && p != 0.f) sum += p * (a.T * (logf(p) + log_s) - (s_z[j] - q.m));
    }
    return sum;
}

// A row by one workgroup, held in registers between the softmax's sums and the gradient: read once, written once.
template <uint32_t TYPE, uint32_t NT, uint32_t NV, bool GRAD>
__global__ __launch_bounds__(NT) void k_distill_row(DistillArgs a) {
    extern __shared__ uint32_t s_dyn[];
    __shared__ DistillRoom<NT> room;
    uint32_t* s_idx = s_dyn;
    float *s_p = reinterpret_cast<float*>(s_dyn + a.k), *s_z = s_p + a.k;
    uint32_t* s_table = s_dyn + 3u * a.k;
    const uint64_t row = blockIdx.x;
    const float w = a.weight ? a.weight[row] : 1.f;
    Raw8<TYPE> raw[NV];
    bool live = w != 0.f;
    Softmax q = {-INFINITY, 0.f};
    if (live) {
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint64_t e = 8ull * (i * NT + threadIdx.x);
            raw[i] = load8_first<TYPE>(a.z, row * a.ld + e, (int64_t)a.vocab - (int64_t)e, minus_inf<TYPE>());
        }
        live = read_teacher<TYPE, NT>(a, row, 0, a.vocab, nullptr, s_idx, s_p, s_z, s_table, room);
    }
    if (live) {
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) q.m = fmaxf(q.m, raw[i].at(e));
        const float m = q.m == -INFINITY ? 0.f : q.m;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) q.s += exp2_fast((raw[i].at(e) - m) * a.c);
        q = join_block<NT>(q, a.c, room.row);
        live = q.s != 0.f;
    }
    if (a.loss) {
        const float sum = live ? sum_block<NT>(cross_terms<NT>(a, s_idx, s_p, s_z, q), room.sum) : 0.f;
        if (threadIdx.x == 0) a.loss[row] = live ? w * a.T * sum : 0.f;
    }
    if (a.stats && threadIdx.x == 0) {
        a.stats[2 * row] = live ? q.m : 0.f;
        a.stats[2 * row + 1] = live ? q.s : 0.f;
    }
    if (GRAD) {
        const float f = w * a.T, fs = f / q.s;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint64_t e = 8ull * (i * NT + threadIdx.x);
            float v[8];
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) v[x] = live ? exp2_fast((raw[i].at(x) - q.m) * a.c) * fs : 0.f;
            store8_first<TYPE>(a.grad, row * a.ld_grad + e, (int64_t)a.vocab - (int64_t)e, v);
        }
        if (live) {
            __syncthreads();                     // the entries' columns once more, behind the others' stores
            for (uint32_t j = threadIdx.x; j < a.k; j += NT)
                if (s_idx[j] != 0xFFFFFFFFu) store1<TYPE>(a.grad, row * a.ld_grad + s_idx[j], f * (exp2_fast((s_z[j] - q.m) * a.c) / q.s - s_p[j]));
        }
    }
}

constexpr uint32_t CHUNK_NT = 256, CHUNK_NV = 4, DISTILL_CHUNK = 8 * CHUNK_NT * CHUNK_NV;

// A chunk of a row: its part of the softmax's sums; the first chunk's workgroup also puts the student's logits at the entries aside.
template <uint32_t TYPE>
__global__ __launch_bounds__(CHUNK_NT) void k_distill_part(DistillArgs a) {
    __shared__ Softmax room[CHUNK_NT / 64];
    const uint64_t row = blockIdx.x / a.chunks;
    const uint32_t chunk = blockIdx.x % a.chunks;
    if (a.weight && a.weight[row] == 0.f) return;
    const uint64_t from = chunk * a.chunk, to = from + a.chunk < a.vocab ? from + a.chunk : a.vocab;
    Softmax q = {-INFINITY, 0.f};
    for (uint64_t e0 = from; e0 < to; e0 += DISTILL_CHUNK) {
        Raw8<TYPE> raw[CHUNK_NV];
#pragma unroll
        for (uint32_t i = 0; i < CHUNK_NV; ++i) {
            const uint64_t e = e0 + 8ull * (i * CHUNK_NT + threadIdx.x);
            raw[i] = load8_first<TYPE>(a.z, row * a.ld + e, (int64_t)to - (int64_t)e, minus_inf<TYPE>());
        }
        Softmax v = {-INFINITY, 0.f};
#pragma unroll
        for (uint32_t i = 0; i < CHUNK_NV; ++i)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) v.m = fmaxf(v.m, raw[i].at(e));
        const float m = v.m == -INFINITY ? 0.f : v.m;
#pragma unroll
        for (uint32_t i = 0; i < CHUNK_NV; ++i)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) v.s += exp2_fast((raw[i].at(e) - m) * a.c);
        q = join(q, v, a.c);
    }
    q = join_block<CHUNK_NT>(q, a.c, room);
    if (threadIdx.x == 0) {
        a.parts[2 * ((uint64_t)row * a.chunks + chunk)] = q.m;
        a.parts[2 * ((uint64_t)row * a.chunks + chunk) + 1] = q.s;
    }
    if (chunk == 0)
        for (uint32_t j = threadIdx.x; j < a.k; j += CHUNK_NT) {
            const uint32_t i = a.idx[row * a.k + j];
            a.zj[row * a.k + j] = i < a.vocab ? load1<TYPE>(a.z, row * a.ld + i) : 0.f;
        }
}

// A chunk of a row behind its sums, which come from the chunks' parts (PARTS) or from an earlier call's statistics: the
// gradient (GRAD), and in the first chunk the loss and the statistics.
template <uint32_t TYPE, bool PARTS, bool GRAD>
__global__ __launch_bounds__(CHUNK_NT) void k_distill_rest(DistillArgs a, uint32_t grid_chunks) {
    constexpr uint32_t NT = CHUNK_NT;
    extern __shared__ uint32_t s_dyn[];
    __shared__ DistillRoom<NT> room;
    uint32_t* s_idx = s_dyn;
    float *s_p = reinterpret_cast<float*>(s_dyn + a.k), *s_z = s_p + a.k;
    uint32_t* s_table = s_dyn + 3u * a.k;
    const uint64_t row = blockIdx.x / grid_chunks;
    const uint32_t chunk = blockIdx.x % grid_chunks;
    const uint64_t from = chunk * a.chunk, to = from + a.chunk < a.vocab ? from + a.chunk : a.vocab;
    const float w = a.weight ? a.weight[row] : 1.f;
    Softmax q = {-INFINITY, 0.f};
    bool live = w != 0.f;
    if (live) {
        if (PARTS) {
            for (uint32_t i = threadIdx.x; i < a.chunks; i += NT) {
                const float* p = a.parts + 2 * ((uint64_t)row * a.chunks + i);
                q = join(q, Softmax{p[0], p[1]}, a.c);
            }
            q = join_block<NT>(q, a.c, room.row);
        } else {
            q = Softmax{a.stats[2 * row], a.stats[2 * row + 1]};
        }
        live = q.s != 0.f;
    }
    if (live) live = read_teacher<TYPE, NT>(a, row, from, to, PARTS ? a.zj : nullptr, s_idx, s_p, s_z, s_table, room);
    if (PARTS && chunk == 0) {
        if (a.loss) {
            const float sum = live ? sum_block<NT>(cross_terms<NT>(a, s_idx, s_p, s_z, q), room.sum) : 0.f;
            if (threadIdx.x == 0) a.loss[row] = live ? w * a.T * sum : 0.f;
        }
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * row] = live ? q.m : 0.f;
            a.stats[2 * row + 1] = live ? q.s : 0.f;
        }
    }
    if (GRAD) {
        const float f = w * a.T, fs = f / q.s;
        for (uint64_t e0 = from; e0 < to; e0 += DISTILL_CHUNK) {
            Raw8<TYPE> raw[CHUNK_NV];
#pragma unroll
            for (uint32_t i = 0; i < CHUNK_NV; ++i) {
                const uint64_t e = e0 + 8ull * (i * NT + threadIdx.x);
                if (live) raw[i] = load8_first<TYPE>(a.z, row * a.ld + e, (int64_t)to - (int64_t)e, minus_inf<TYPE>());
            }
#pragma unroll
            for (uint32_t i = 0; i < CHUNK_NV; ++i) {
                const uint64_t e = e0 + 8ull * (i * NT + threadIdx.x);
                float v[8];
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x) v[x] = live ? exp2_fast((raw[i].at(x) - q.m) * a.c) * fs : 0.f;
                store8_first<TYPE>(a.grad, row * a.ld_grad + e, (int64_t)to - (int64_t)e, v);
            }
        }
        if (live) {
            __syncthreads();
            for (uint32_t j = threadIdx.x; j < a.k; j += NT)
                if (s_idx[j] >= from && s_idx[j] < to)
                    store1<TYPE>(a.grad, row * a.ld_grad + s_idx[j], f * (exp2_fast((s_z[j] - q.m) * a.c) / q.s - s_p[j]));
        }
    }
}

}  // namespace kimad
