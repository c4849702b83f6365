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
    uint64_t rows, ld, ld_grad;
    uint32_t vocab, k, chunks, bloom;   // bloom: words of the table that finds indices given twice, a power of two
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
// Over a wave's lanes, the result in all of them.
__device__ __forceinline__ Softmax join_wave(Softmax v, float c) {
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) v = join(v, Softmax{__shfl_xor(v.m, o), __shfl_xor(v.s, o)}, c);
    return v;
}
// Over a workgroup's threads.
template <uint32_t NT>
__device__ __forceinline__ Softmax join_block(Softmax v, float c, Softmax* room) {
    v = join_wave(v, c);
    if (NT == 64) return v;
    if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (uint32_t i = 1; i < NT / 64; ++i) v = join(v, room[i], c);
    return v;
}

// A row's elements in groups of eight that begin at 16-byte addresses: with mis elements in front of the row's first one back to such an address, group j
// holds elements 8 j - mis and on.  Reads take whole 16 bytes, of which the first and the last may hold neighbours of the row (never another page);
// what is not the row's is masked, and not written.
template <uint32_t TYPE>
constexpr uint32_t bytes_of() { return TYPE == TYPE_F32 ? 4 : 2; }
template <uint32_t TYPE>
__device__ __forceinline__ uint32_t misplaced(const void* p, uint64_t element) {
    return (uint32_t)((reinterpret_cast<uintptr_t>(p) / bytes_of<TYPE>() + element) % (16 / bytes_of<TYPE>()));
}
// NV * NT groups from group j0 on (the same for the workgroup), of which thread t holds every NT-th one from j0 + t on.
template <uint32_t TYPE, uint32_t NT, uint32_t NV>
struct Groups {
    Raw8<TYPE> raw[NV];
    static constexpr uint32_t B = bytes_of<TYPE>(), GROUP = 8 * B;
    // (a group of NT beyond the row is passed over by all threads)
    static __device__ __forceinline__ bool beyond(uint32_t i, uint32_t j0, uint32_t mis, uint32_t vocab) { return 8ull * (j0 + i * NT) >= (uint64_t)mis + vocab; }
    static __device__ __forceinline__ bool whole(uint32_t i, uint32_t j0, uint32_t mis, uint32_t vocab) {
        return (mis == 0 || j0 + i > 0) && 8ull * (j0 + (i + 1) * NT) <= (uint64_t)mis + vocab;
    }
    static __device__ __forceinline__ uint32_t element(uint32_t i, uint32_t j0, uint32_t mis) { return 8u * (j0 + i * NT + threadIdx.x) - mis; }   // (of group 0: below 0, a large number)

    __device__ __forceinline__ void load(const void* p, uint64_t row, uint32_t j0, uint32_t mis, uint32_t vocab) {
        const uint64_t end = ((uint64_t)mis + vocab) * B + 15 & ~15ull, begin = (uint64_t)j0 * GROUP, left = end > begin ? end - begin : 0;
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t*>(const_cast<void*>(p)) + (row - mis) * B + begin, 0,
                                                                               (int)(left < NV * NT * GROUP ? left : NV * NT * GROUP), 0x00020000);
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            if (!beyond(i, j0, mis, vocab)) {
#pragma unroll
                for (uint32_t h = 0; h < GROUP / 16; ++h) {
                    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from, threadIdx.x * GROUP + 16 * h, i * NT * GROUP, 0);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) raw[i].r[(4 * h + k) % (GROUP / 4)] = v[k];
                }
            }
        }
    }
    // What is not the row's becomes -Inf.
    __device__ __forceinline__ void mask(uint32_t j0, uint32_t mis, uint32_t vocab) {
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
            if (!whole(i, j0, mis, vocab) && !beyond(i, j0, mis, vocab)) {
                const uint32_t e = element(i, j0, mis);
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x)
                    if (e + x >= vocab) raw[i].set(x, minus_inf<TYPE>());
            }
    }
    // Largest element and sum, a group at a time: an element is taken apart once, and only as it lies in memory does it stay in a register.
    __device__ __forceinline__ Softmax softmax(uint32_t j0, uint32_t mis, uint32_t vocab, float c) const {
        Softmax q = {-INFINITY, 0.f};
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            if (!beyond(i, j0, mis, vocab)) {
                float v[8], m = q.m;
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x) {
                    v[x] = raw[i].at(x);
                    m = fmaxf(m, v[x]);
                }
                const float from = m == -INFINITY ? 0.f : m;
                float sum = 0.f;
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x) sum += exp2_fast((v[x] - from) * c);
                q.s = (q.m == m ? q.s : q.s * exp2_fast((q.m - m) * c)) + sum;
                q.m = m;
            }
        }
        return q;
    }
    // The gradient but for the entries' part, f q; zeros where `live` is false.
    __device__ __forceinline__ void store_gradient(void* p, uint64_t row, uint32_t j0, uint32_t mis, uint32_t vocab, Softmax q, float c, float f, bool live) {
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
            for (uint32_t k = 0; k < GROUP / 4; ++k) asm volatile("" : "+v"(raw[i].r[k]));   // (what was taken apart before is not kept: twice the registers)
        const float fs = f / q.s;
        uint8_t* base = static_cast<uint8_t*>(p) + (row - mis) * B + (uint64_t)j0 * GROUP;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            if (!beyond(i, j0, mis, vocab)) {
                float v[8] = {};
                if (live)
#pragma unroll
                    for (uint32_t x = 0; x < 8; ++x) v[x] = exp2_fast((raw[i].at(x) - q.m) * c) * fs;
                uint8_t* to = base + i * NT * GROUP + threadIdx.x * GROUP;
                const uint32_t e = element(i, j0, mis);
                if (whole(i, j0, mis, vocab) || (e < vocab && vocab - e >= 8)) store8<TYPE>(to, 0, v);
                else
#pragma unroll
                    for (uint32_t x = 0; x < 8; ++x)
                        if (e + x < vocab) store1<TYPE>(to, x, v[x]);
            }
        }
    }
};

// A row's entries, by one wave: indices (those beyond the vocabulary are none and become 0xFFFFFFFF), probabilities, and the student's logits unless
// they are given or stand outside [from, to).  False where there is no entry.  Entries of one index are one entry with the sum
// of their probabilities; it goes to the first of them, the others get 0xFFFFFFFF.  They are looked for, by some k^2 / 128 reads of LDS a lane, unless no two of the
// row's indices meet in the table, whose 32 k bits or more spare few rows that: with distinct random indices two meet by chance in 65 % of rows at k = 64, 97 % at 256.
template <uint32_t TYPE>
__device__ __forceinline__ bool read_teacher(const DistillArgs& a, uint64_t row, uint32_t from, uint32_t to, const float* zj, uint32_t* s_idx,
                                             float* s_p, float* s_z, uint32_t* s_table) {
    const uint32_t k = a.k, lane = threadIdx.x & 63u;
    for (uint32_t i = lane; i < a.bloom; i += 64) s_table[i] = 0;
    wave_sync_lds();
    Softmax v = {-INFINITY, 0.f};
    bool any = false, meets = false;
    constexpr uint32_t U = 4;                            // entries of a lane under way together
    for (uint32_t j0 = lane; j0 < k; j0 += 64 * U) {
        uint32_t i[U];
        float t[U], z[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t j = j0 + 64 * u;
            i[u] = j < k ? a.idx[row * k + j] : 0xFFFFFFFFu;
            t[u] = j < k ? a.val[row * k + j] : 0.f;
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t j = j0 + 64 * u;
            if (zj) z[u] = j < k ? zj[row * k + j] : 0.f;
            else z[u] = i[u] < a.vocab && i[u] >= from && i[u] < to ? load1<TYPE>(a.z, row * a.ld + i[u]) : 0.f;
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t j = j0 + 64 * u;
            if (j >= k) break;
            const bool in = i[u] < a.vocab;
            if (!in) t[u] = -INFINITY;
            s_idx[j] = in ? i[u] : 0xFFFFFFFFu;
            s_p[j] = t[u];
            s_z[j] = z[u];
            any = any || (in && t[u] != -INFINITY);
            const bool nan = t[u] != t[u];
            v = join(v, Softmax{t[u], t[u] == -INFINITY ? 0.f : 1.f}, a.c);
            if (nan) v.s = t[u];
            if (in) meets = meets || (atomicOr(&s_table[(i[u] >> 5) & (a.bloom - 1u)], 1u << (i[u] & 31u)) >> (i[u] & 31u) & 1u);
        }
    }
    if (!ballot(any)) return false;
    v = join_wave(v, a.c);
    wave_sync_lds();
    bool twice = false;
    if (ballot(meets))
        for (uint32_t j = lane; j < k; j += 64)
            for (uint32_t l = 0; l < j; ++l) twice = twice || (s_idx[l] == s_idx[j] && s_idx[j] != 0xFFFFFFFFu);
    for (uint32_t j = lane; j < k; j += 64) {
        const float t = s_p[j];
        s_p[j] = t == -INFINITY ? 0.f : exp2_fast((t - v.m) * a.c) / v.s;
    }
    wave_sync_lds();
    if (ballot(twice)) {
        for (uint32_t j = lane; j < k; j += 64) {
            bool first = true;
            float p = 0.f;
            for (uint32_t l = 0; l < k; ++l)
                if (s_idx[l] == s_idx[j]) { first = first && l >= j; p += s_p[l]; }
            s_table[j] = __float_as_uint(first ? p : -1.f);      // (no probability is negative)
        }
        wave_sync_lds();
        for (uint32_t j = lane; j < k; j += 64) {
            const float p = __uint_as_float(s_table[j]);
            if (p == -1.f) s_idx[j] = 0xFFFFFFFFu;
            s_p[j] = p == -1.f || s_idx[j] == 0xFFFFFFFFu ? 0.f : p;
        }
        wave_sync_lds();
    }
    return true;
}

// T sum_j p_j (ln p_j - ln q_j), by one wave; an entry with p = 0 adds nothing, whatever the student's logit.  (Times T, so that a logit of the type's
// lowest value overflows only where the loss does.)
__device__ __forceinline__ float cross_terms(const DistillArgs& a, const uint32_t* s_idx, const float* s_p, const float* s_z, Softmax q) {
    const float log_s = logf(q.s);
    float sum = 0.f;
    for (uint32_t j = threadIdx.x & 63u; j < a.k; j += 64) {
        const float p = s_p[j];
        if (s_idx[j] != 0xFFFFFFFFu && p != 0.f) sum += p * (a.T * (logf(p) + log_s) - (s_z[j] - q.m));
    }
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    return sum;
}

// Waves of a SIMD that the registers allow: the row's own and about 28 more.
template <uint32_t TYPE>
constexpr uint32_t distill_waves(uint32_t nv) {
    const uint32_t waves = 512 / ((TYPE == TYPE_F32 ? 8 : 4) * nv + 28);
    return waves > 8 ? 8 : waves;
}
// A row by one workgroup, held in registers between the softmax's sums and the gradient: read once, written once.  The first wave reads the entries while
// the row comes.  Bound by memory: 8192 x 50257 in bfloat16 305 to 328 us by machine, 5.0 to 5.4 TB/s, the loss alone 200 to 211; 4096 x 32000 in fp32 208 us, 5.0,
// the loss alone 118.
template <uint32_t TYPE, uint32_t NT, uint32_t NV, bool GRAD>
__global__ __launch_bounds__(NT, distill_waves<TYPE>(NV)) void k_distill_row(DistillArgs a) {
    extern __shared__ uint32_t s_dyn[];
    __shared__ Softmax s_wave[NT / 64];
    __shared__ uint32_t s_any;
    uint32_t* s_idx = s_dyn;
    float *s_p = reinterpret_cast<float*>(s_dyn + a.k), *s_z = s_p + a.k;
    uint32_t* s_table = s_dyn + 3u * a.k;
    const uint64_t row = blockIdx.x;
    const float w = a.weight ? a.weight[row] : 1.f;
    const uint32_t mis = misplaced<TYPE>(a.z, row * a.ld);
    const bool first_wave = threadIdx.x < 64u;
    Groups<TYPE, NT, NV> z;
    bool live = w != 0.f;
    Softmax q = {-INFINITY, 0.f};
    if (live) {
        z.load(a.z, row * a.ld, 0, mis, a.vocab);
        if (first_wave) {
            const bool any = read_teacher<TYPE>(a, row, 0, a.vocab, nullptr, s_idx, s_p, s_z, s_table);
            if (threadIdx.x == 0) s_any = any;
        }
        z.mask(0, mis, a.vocab);
        q = join_block<NT>(z.softmax(0, mis, a.vocab, a.c), a.c, s_wave);
        if (NT == 64) wave_sync_lds();
        live = s_any && q.s != 0.f;
    }
    if (first_wave) {
        const float sum = live && a.loss ? cross_terms(a, s_idx, s_p, s_z, q) : 0.f;
        if (threadIdx.x == 0) {
            if (a.loss) a.loss[row] = live ? w * a.T * sum : 0.f;
            if (a.stats) {
                a.stats[2 * row] = live ? q.m : 0.f;
                a.stats[2 * row + 1] = live ? q.s : 0.f;
            }
        }
    }
    if (GRAD) {
        const float f = w * a.T;
        z.store_gradient(a.grad, row * a.ld_grad, 0, mis, a.vocab, q, a.c, f, live);
        if (live) {
            __syncthreads();                     // the entries' columns once more, behind the others' stores
            for (uint32_t j = threadIdx.x; j < a.k; j += NT)
                if (s_idx[j] != 0xFFFFFFFFu) store1<TYPE>(a.grad, row * a.ld_grad + s_idx[j], f * (exp2_fast((s_z[j] - q.m) * a.c) / q.s - s_p[j]));
        }
    }
}

constexpr uint32_t CHUNK_NT = 256, CHUNK_NV = 4, DISTILL_CHUNK = CHUNK_NT * CHUNK_NV;   // groups of a chunk

// Rows of more than 65529 elements are read twice, by the two kernels below: 2048 x 131072 in bfloat16 308 us, 1.6e9 bytes at 5.2 TB/s (the loss alone, one read,
// 118; the gradient alone 185).  A chunk of a row: its part of the softmax's sums; the first chunk's workgroup also puts the student's logits at the entries aside.
template <uint32_t TYPE>
__global__ __launch_bounds__(CHUNK_NT) void k_distill_part(DistillArgs a) {
    __shared__ Softmax room[CHUNK_NT / 64];
    const uint64_t row = blockIdx.x / a.chunks;
    const uint32_t chunk = blockIdx.x % a.chunks;
    if (a.weight && a.weight[row] == 0.f) return;
    const uint32_t mis = misplaced<TYPE>(a.z, row * a.ld), j0 = chunk * DISTILL_CHUNK;
    Groups<TYPE, CHUNK_NT, CHUNK_NV> z;
    z.load(a.z, row * a.ld, j0, mis, a.vocab);
    z.mask(j0, mis, a.vocab);
    const Softmax q = join_block<CHUNK_NT>(z.softmax(j0, mis, a.vocab, a.c), a.c, room);
    if (threadIdx.x == 0) {
        a.parts[2 * (row * a.chunks + chunk)] = q.m;
        a.parts[2 * (row * a.chunks + chunk) + 1] = q.s;
    }
    if (chunk == 0)
        for (uint32_t j = threadIdx.x; j < a.k; j += CHUNK_NT) {
            const uint32_t i = a.idx[row * a.k + j];
            a.zj[row * a.k + j] = i < a.vocab ? load1<TYPE>(a.z, row * a.ld + i) : 0.f;
        }
}

// A chunk of a row behind its sums, which come from the chunks' parts (PARTS) or from an earlier call's statistics: the gradient (GRAD), and in the
// first chunk the loss and the statistics.
template <uint32_t TYPE, bool PARTS, bool GRAD>
__global__ __launch_bounds__(CHUNK_NT) void k_distill_rest(DistillArgs a, uint32_t grid_chunks) {
    constexpr uint32_t NT = CHUNK_NT;
    extern __shared__ uint32_t s_dyn[];
    __shared__ uint32_t s_any;
    uint32_t* s_idx = s_dyn;
    float *s_p = reinterpret_cast<float*>(s_dyn + a.k), *s_z = s_p + a.k;
    uint32_t* s_table = s_dyn + 3u * a.k;
    const uint64_t row = blockIdx.x / grid_chunks;
    const uint32_t chunk = blockIdx.x % grid_chunks;
    const uint32_t mis = misplaced<TYPE>(a.z, row * a.ld), j0 = chunk * DISTILL_CHUNK;
    const float w = a.weight ? a.weight[row] : 1.f;
    const bool first_wave = threadIdx.x < 64u;
    Softmax q = {-INFINITY, 0.f};
    Groups<TYPE, NT, CHUNK_NV> z;
    bool live = w != 0.f;
    if (live) {
        if (GRAD) z.load(a.z, row * a.ld, j0, mis, a.vocab);
        if (PARTS) {
            for (uint32_t i = threadIdx.x & 63u; i < a.chunks; i += 64) {
                const float* p = a.parts + 2 * (row * a.chunks + i);
                q = join(q, Softmax{p[0], p[1]}, a.c);
            }
            q = join_wave(q, a.c);
        } else {
            q = Softmax{a.stats[2 * row], a.stats[2 * row + 1]};
        }
        if (first_wave) {
            // (the columns of the chunk's groups: what an entry there was is read before it is written)
            const uint32_t begin = chunk * DISTILL_CHUNK * 8, from = begin < mis ? 0 : begin - mis;
            const bool any = read_teacher<TYPE>(a, row, from, from + DISTILL_CHUNK * 8, PARTS ? a.zj : nullptr, s_idx, s_p, s_z, s_table);
            if (threadIdx.x == 0) s_any = any;
        }
        __syncthreads();
        live = s_any && q.s != 0.f;
    }
    if (PARTS && chunk == 0 && first_wave) {
        const float sum = live && a.loss ? cross_terms(a, s_idx, s_p, s_z, q) : 0.f;
        if (threadIdx.x == 0) {
            if (a.loss) a.loss[row] = live ? w * a.T * sum : 0.f;
            if (a.stats) {
                a.stats[2 * row] = live ? q.m : 0.f;
                a.stats[2 * row + 1] = live ? q.s : 0.f;
            }
        }
    }
    if (GRAD) {
        const float f = w * a.T;
        z.store_gradient(a.grad, row * a.ld_grad, j0, mis, a.vocab, q, a.c, f, live);
        if (live) {
            __syncthreads();
            for (uint32_t j = threadIdx.x; j < a.k; j += NT) {
                const uint32_t i = s_idx[j];
                if (i != 0xFFFFFFFFu && (i + mis) / (8 * DISTILL_CHUNK) == chunk)
                    store1<TYPE>(a.grad, row * a.ld_grad + i, f * (exp2_fast((s_z[j] - q.m) * a.c) / q.s - s_p[j]));
            }
        }
    }
}

}  // namespace kimad
