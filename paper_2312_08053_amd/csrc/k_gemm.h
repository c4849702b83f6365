// Products of 16-bit matrices with fp32 sums, C [M, N] = A B, and what is done with a sum on its way out.
//
// An operand is stored along K (rows of K elements: A [M, K], B [N, K]) or across it (rows of M or N elements: A [K, M], B [K, N]), so that a layer's
// forward product and both of its gradients read activations, weights and gradients as they lie:
//   x W^T      A along K,  B along K
//   dz W       A along K,  B across K
//   dz^T x     A across K, B across K
// v_mfma_f32_32x32x16: lane l holds elements k = 8 (l / 32) .. + 7 of row l % 32, of A and of B; element i of the result's lane l is
// C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32].
#pragma once
#include "gemm_stage.h"
#include "k_mx4_matmul.h"

namespace kimad {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

template <uint32_t TYPE>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (TYPE == TYPE_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <uint32_t TYPE>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (TYPE == TYPE_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// ---- activations ---------------------------------------------------------------------------------------------------------------

enum : uint32_t { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };     // KIMAD_ACT_* of the public header

constexpr float LOG2E = 1.4426950408889634f;
// What the sigmoid of gelu (its tanh form, z sigmoid(2 sqrt(2 / pi) (z + 0.044715 z^3))) is taken of.
constexpr float GELU_A = 1.5957691216057308f, GELU_B = 0.044715f;
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-LOG2E * x)); }
template <uint32_t ACT>
__device__ __forceinline__ float act_inner(float z) { return ACT == ACT_GELU ? GELU_A * fmaf(GELU_B * z * z, z, z) : z; }
// (Comparisons, through which a NaN stays one, keep infinite z from meeting a sigmoid of 0, and their limits.)
template <uint32_t ACT>
__device__ __forceinline__ float act_as(float z) {
    if (ACT == ACT_NONE) return z;
    if (ACT == ACT_RELU) return z < 0.f ? 0.f : z;
    const float s = sigmoid(act_inner<ACT>(z));
    return (z < -1e30f ? -1e30f : z) * s;
}
template <uint32_t ACT>
__device__ __forceinline__ float slope_as(float z) {
    if (ACT == ACT_NONE) return 1.f;
    if (ACT == ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    z = z > 100.f ? 100.f : z < -100.f ? -100.f : z;                          // (the slope is 1 or 0 from there on)
    const float s = sigmoid(act_inner<ACT>(z)), zd = z * (s * (1.f - s));
    return s + (ACT == ACT_GELU ? zd * (GELU_A * fmaf(3.f * GELU_B * z, z, 1.f)) : zd);
}
// Calls f with the activation as a compile-time constant.
template <class F>
__device__ __forceinline__ void with_act(uint32_t act, F f) {
    if (act == ACT_NONE) f(std::integral_constant<uint32_t, ACT_NONE>{});
    else if (act == ACT_RELU) f(std::integral_constant<uint32_t, ACT_RELU>{});
    else if (act == ACT_GELU) f(std::integral_constant<uint32_t, ACT_GELU>{});
    else f(std::integral_constant<uint32_t, ACT_SILU>{});
}
__device__ __forceinline__ float act_of(float z, uint32_t act) {
    with_act(act, [&](auto a) { z = act_as<decltype(a)::value>(z); });
    return z;
}

// ---- tiles ---------------------------------------------------------------------------------------------------------------------

// Exponentials e = exp(s - m), 0 to 1, in 16 bits without a sign, whose rounding is below the type's and whose range is beyond what G in the type reaches:
//   of a product in bfloat16 six bits of exponent and ten of mantissa: exact to 2^-11 of e down to 2^-62, to 2^-73 below;
//   of one in fp16 five and eleven: 2^-12 down to 2^-30, 2^-42 below.
// The float e / 2^DOWN has such an exponent, and its bits, rounded, are the code.  (fp16 numbers 2^15 e, which the hardware rounds two at a time, lose what is below 2^-29 of the largest.)
template <uint32_t TYPE>
struct SmallFloat {
    static constexpr uint32_t EXPONENT = TYPE == TYPE_BF16 ? 6 : 5, DOWN = 128 - (1u << EXPONENT), LEFT = 9 - EXPONENT;   // LEFT: bits that are always 0 at the top
    static constexpr float TO_E = TYPE == TYPE_BF16 ? 0x1p64f : 0x1p96f, FROM_E = 1.f / TO_E;
    static_assert(DOWN == (TYPE == TYPE_BF16 ? 64 : 96), "the powers of two");
    static __device__ __forceinline__ uint32_t bits(float e) { return (__float_as_uint(e * FROM_E) << LEFT) + 0x8000u; }   // the code in the upper half
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_amdgcn_perm(bits(b), bits(a), 0x07060302u); }
    static __device__ __forceinline__ float at(uint32_t word, uint32_t half) { return __uint_as_float((half ? word & 0xFFFF0000u : word << 16) >> LEFT); }   // e / 2^DOWN
};

// What becomes of a sum s:  z = scale s + bias, z kept, act(z) + residual.
struct GemmEnd {
    void* out;                   // fp32 or of the operands' type
    const void* bias;            // [N], or null
    const void* residual;        // [M, N], or null
    void* z;                     // [M, N], or null
    const float* scale;          // one number on the device, or null: 1
    uint64_t ld, ld_res, ld_z;
    uint32_t act, res32;         // res32: the residual is fp32
};
// Or, for the cross entropy: exponentials and their sums (see k_xent.h).
struct SoftmaxEnd {
    f32x2* strips;               // [M][strips]: largest sum of a strip's columns, and the sum of exp(s - largest)
    void* e;                     // [M, pitch] exp(s - largest) as a SmallFloat, or null
    const int32_t* target;       // [M]
    float* picked;               // [M]: the sum at the target
    uint64_t pitch;
    uint32_t strips_row;
};
struct GemmArgs {
    const uint8_t *a, *b;
    uint64_t lda, ldb;           // elements from row to row as stored
    uint64_t M, N, K;            // K: a multiple of 8 where an operand is stored along it
    uint64_t k_rows_a, k_rows_b; // rows that an operand across K has (beyond them: zeros)
    uint32_t tiles_m, tiles_n, band;   // band: rows of tiles that are taken together, so that what an XCD reads at a time is shared
    uint32_t whole;              // the first so many tiles are summed by one workgroup each; the others' sums are shared out,
    uint32_t splits, share;      // in parts of `share` stages each (the last one fewer), part p of the t-th of them at parts + (p * (tiles - whole) + t) tiles
    float* parts;                // (as the waves' registers lie), which k_gemm_join adds
    GemmEnd end;
    SoftmaxEnd soft;
};

constexpr uint32_t GEMM_STAGE_K = 64;
// A tile of BM by BN, WM by WN waves.  64 of K are a stage, 128 bytes of a row that is stored along K, of which LDS holds two.
//   Along K, 16 bytes b of row r stand at b ^ (r / 2 % 8), so that sixteen lanes that read one b of sixteen rows meet different banks.
//   Across K, LDS has rows of one k, BM elements each, and a read that transposes: sixteen lanes bring 4 k of 16 elements, and each gets
//   one element's four.  Of a row the 64-byte pieces stand turned by its k, so that the four rows of such a read lie in different banks.
//
// What bounds it, by copies with parts left out (8192 x 2048 x 5632 along K, one tile of 256 a unit, 88 stages; microseconds): products and reads of LDS alone 101, loads
// alone 94 (64 KB a stage and unit, 16 TB/s in all), together on zeros 119 to 126, on random numbers 154 to 175 by machine: the matrix cores work in 61 % of the cycles, and with numbers in
// them the clock falls to 1.9 GHz.  That is not the card's limit: a library's product of these sizes takes 90 on zeros and 121 on random numbers where this one, measured beside it, takes 117
// and 153 (8192 x 5632 x 2048: 132 and 156, 140 and 173), so that a quarter of the time is this schedule's own.  Across K both (8192 x 8192 x 8192) 541, 661 and 870 on zeros as on random
// numbers: loads and transposing reads, which share LDS.  8192 x 8192 x 8192 along K 811 to 880, 1250 to 1360 TFLOP/s.
template <uint32_t BM_, uint32_t BN_, uint32_t WM_, uint32_t WN_>
struct GemmTile {
    static constexpr uint32_t BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr uint32_t WAVES = WM * WN, TI = BM / WM / 32, TJ = BN / WN / 32, STEPS = GEMM_STAGE_K / 16;
    static constexpr uint32_t LA = BM / 8 / WAVES, LB = BN / 8 / WAVES, LOADS = LA + LB;
    static constexpr uint32_t STAGE = (BM + BN) * GEMM_STAGE_K * 2;
    static constexpr uint32_t COLS = 32 * TJ, PITCH = COLS + 8;
    static constexpr uint32_t OUT = 8 * PITCH * 4, LDS = 2 * STAGE + WAVES * OUT;
    static constexpr uint32_t STRIP = COLS;                                   // columns of a strip of the softmax's end
};

// An operand's side of a tile's loads.  E: elements of the tile's edge, ACROSS: stored across K.
template <uint32_t E, uint32_t WAVES, bool ACROSS>
struct GemmSide {
    static constexpr uint32_t SK = GEMM_STAGE_K, LANES_ROW = ACROSS ? E / 8 : SK / 8, ROWS_LOAD = 64 / LANES_ROW;   // lanes of a stored row's part, rows of a load
    // What is brought next: a stage of K, of `rows` rows along K or elements across it.
    const uint8_t* base;
    uint64_t ld_bytes;
    uint32_t rows, k_left;       // k_left: of K (rows of it, across) from this stage on
    uint32_t bytes;
    uint32_t offset;             // of the lane, in its first load
    uint32_t block;              // along K: which 16 bytes of a row's part

    static __device__ __forceinline__ uint32_t turned(uint32_t k) { return E >= 128 ? k & 3u : (k >> 1) & 1u; }
    static __device__ __forceinline__ uint32_t turn(uint32_t row) { return (row >> 1) & 7u; }   // along K
    __device__ __forceinline__ void begin(uint32_t wave, uint32_t lane, uint64_t ld) {
        ld_bytes = 2 * ld;
        const uint32_t row = wave * ROWS_LOAD + lane / LANES_ROW, at = lane % LANES_ROW;
        // (the loads of a wave are WAVES * ROWS_LOAD rows apart, and turned alike)
        static_assert(ACROSS ? WAVES * ROWS_LOAD % 4 == 0 : WAVES * ROWS_LOAD % 16 == 0, "one order for all loads of a lane");
        block = ACROSS ? ((at >> 2) ^ turned(row)) << 2 | (at & 3u) : at ^ turn(row);
        offset = row * (uint32_t)ld_bytes + 16u * block;
    }
    // At row or element `first` of `all`, and at k0 of K.
    __device__ __forceinline__ void aim(const uint8_t* p, uint64_t first, uint64_t all, uint32_t k0, uint32_t K) {
        base = p + (ACROSS ? k0 * ld_bytes + 2 * first : first * ld_bytes + 2 * k0);
        rows = __builtin_amdgcn_readfirstlane(first >= all ? 0u : all - first < E ? (uint32_t)(all - first) : E);
        k_left = __builtin_amdgcn_readfirstlane(K > k0 ? K - k0 : 0u);
        measure();
    }
    __device__ __forceinline__ void next() {
        base += ACROSS ? SK * ld_bytes : 2 * SK;
        k_left = k_left > SK ? k_left - SK : 0u;
        measure();
    }
    __device__ __forceinline__ void measure() {
        const uint32_t k = k_left < SK ? k_left : SK;
        bytes = __builtin_amdgcn_readfirstlane(stage_bytes(ACROSS, ACROSS ? k : rows, ACROSS ? rows : k, (uint32_t)ld_bytes));   // (made once, not with every load)
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const { return buffer_of(base, bytes); }
    // The lane's offset in its first load; along K, a row's end would run into the next row: such lanes are beyond every buffer, in all of their loads.
    __device__ __forceinline__ uint32_t lane_offset() const { return !ACROSS && 8 * block >= k_left ? 0x80000000u : offset; }
    __device__ __forceinline__ uint32_t step() const { return WAVES * ROWS_LOAD * (uint32_t)ld_bytes; }
};

template <uint32_t E, bool ACROSS>
__device__ __forceinline__ u32x4 gemm_operand(const uint8_t* at, uint32_t k) {
    if constexpr (ACROSS) {
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        u32x4 v;
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) {
            const i16x4 h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + (k + 4 * t) * E * 2));
            const u32x2 w = __builtin_bit_cast(u32x2, h);
            v[2 * t] = w[0];
            v[2 * t + 1] = w[1];
        }
        return v;
    } else {
        return *reinterpret_cast<const u32x4*>(at);
    }
}

// The cache policy of a tile's stores: nontemporal, since operands that are read again and again should keep the L2 (4096 x 50304 x 768 into exponentials 410 us
// without, 362 with; into bfloat16 368 and 332).
constexpr int STREAM = 2;

enum : uint32_t { END_TYPE = 0, END_F32 = 1, END_SOFTMAX = 2 };

// Workgroups go to the eight XCDs in turn: the items are numbered so that an XCD takes a run of them.
__device__ __forceinline__ uint32_t in_runs(uint32_t id, uint32_t total) {
    const uint32_t xcd = id & 7u, each = total >> 3, more = total & 7u;
    return xcd * each + (xcd < more ? xcd : more) + (id >> 3);
}
// A tile by its number, in bands of `band` rows of tiles.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t tm, uint32_t tn, uint32_t band, uint32_t& m, uint32_t& n) {
    const uint32_t first = id / (band * tn) * band, high = tm - first < band ? tm - first : band, r = id % (band * tn);
    m = first + r % high;
    n = r / high;
}

// What is done with a wave's sums, TI times 32 rows from row0 of the tile on and its wn-th strip of columns.  `mine`: LDS of the wave's own, T::OUT bytes.  Whether the
// wave's last accesses are stores, 4 TI or more (fp32: 4 TI TJ).
template <uint32_t TYPE, class T, uint32_t TI, uint32_t END>
__device__ __forceinline__ bool gemm_end(const GemmArgs& g, const f32x16 (&acc)[TI][T::TJ], float* mine, uint64_t tile_m, uint64_t tile_n, uint32_t row0, uint32_t wn) {
    constexpr uint32_t BM = T::BM, BN = T::BN;
    // Eight rows at a time through LDS, so that stores run along the rows: 16 bytes a lane, whole cache lines.
    constexpr uint32_t BYTES = END == END_F32 ? 4 : 2, BEYOND = 0xFFFFFFF0u, EACH = 16 / BYTES, LANES = T::COLS / EACH;   // elements of a lane, lanes of a row
    constexpr uint32_t PASSES = 8 * LANES > 64 ? 8 * LANES / 64 : 1, PASS_ROWS = 8 / PASSES;
    uint32_t l;                                                           // the lane, found anew: kept through the loop, it would cost a register
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    const uint32_t rows = g.M - tile_m < BM ? (uint32_t)(g.M - tile_m) : BM, cols = g.N - tile_n < BN ? (uint32_t)(g.N - tile_n) : BN;
    const uint32_t row = l / LANES, wcol = wn * T::COLS + EACH * (l % LANES), col = EACH * (l % LANES);
    const bool row_in = PASSES > 1 || row < 8, whole = wcol + EACH <= cols, cut = wcol < cols && !whole;
    // eight rows of the wave's sums through LDS, pass by pass
    auto through = [&](uint32_t i, uint32_t e, f32x4 (&v)[PASSES][EACH / 4]) {
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) {
            const f32x16 x = acc[i][j];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) mine[(4 * (l >> 5) + k) * T::PITCH + 32 * j + (l & 31u)] = x[4 * e + k];
        }
        wave_sync_lds();
#pragma unroll
        for (uint32_t p = 0; p < PASSES; ++p)
#pragma unroll
            for (uint32_t q = 0; q < EACH / 4; ++q) v[p][q] = *reinterpret_cast<const f32x4*>(mine + ((p * PASS_ROWS + row) & 7u) * T::PITCH + col + 4 * q);
        wave_sync_lds();
    };
    if constexpr (END == END_SOFTMAX) {
        const SoftmaxEnd& o = g.soft;
        static_assert(PASSES == 1, "a lane's row of eight");
        const bool tile_cut = cols < BN;
        uint32_t target[4 * TI];                                       // as the lane's column, where it is one of the lane's
#pragma unroll
        for (uint32_t x = 0; x < 4 * TI; ++x) {
            const uint32_t r = row0 + 8 * x + row;
            target[x] = row_in && r < rows ? (uint32_t)o.target[tile_m + r] - (uint32_t)(tile_n + wcol) : EACH;
        }
        f32x4 next[1][2];
        through(0, 0, next);
#pragma unroll
        for (uint32_t x = 0; x < 4 * TI; ++x) {
            const uint32_t i = x / 4, e = x % 4, r = row0 + 8 * x + row;
            float v[EACH];
#pragma unroll
            for (uint32_t k = 0; k < EACH; ++k) v[k] = next[0][k / 4][k % 4];
            if (x + 1 < 4 * TI) through((x + 1) / 4, (x + 1) % 4, next);
            const bool in = row_in && r < rows;
            if (target[x] < EACH && target[x] + wcol < cols) {
                float at = v[0];
#pragma unroll
                for (uint32_t k = 1; k < EACH; ++k) at = target[x] == k ? v[k] : at;
                o.picked[tile_m + r] = at;
            }
            if (tile_cut)
#pragma unroll
                for (uint32_t k = 0; k < EACH; ++k) v[k] = wcol + k < cols ? v[k] : -INFINITY;
            float m = v[0], sum = 0.f;
#pragma unroll
            for (uint32_t k = 1; k < EACH; ++k) m = fmaxf(m, v[k]);
            m = fmaxf(m, __uint_as_float(dpp_u32<DPP_XOR1>(__float_as_uint(m))));
            m = fmaxf(m, __uint_as_float(dpp_u32<DPP_XOR2>(__float_as_uint(m))));
            if (LANES == 8) m = fmaxf(m, __uint_as_float(dpp_u32<DPP_HALF_MIRROR>(__float_as_uint(m))));
            const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (uint32_t k = 0; k < EACH; ++k) {
                // (the difference first: that from the largest is then 0, whatever its size, where m LOG2E would be off by |m| 2^-24)
                v[k] = __builtin_amdgcn_exp2f((v[k] - from) * LOG2E);
                sum += v[k];
            }
            sum += __uint_as_float(dpp_u32<DPP_XOR1>(__float_as_uint(sum)));
            sum += __uint_as_float(dpp_u32<DPP_XOR2>(__float_as_uint(sum)));
            if (LANES == 8) sum += __uint_as_float(dpp_u32<DPP_HALF_MIRROR>(__float_as_uint(sum)));
            if (o.e) {
                u32x4 out;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) out[k] = SmallFloat<TYPE>::pack(v[2 * k], v[2 * k + 1]);
                const uint32_t first = row0 + 32 * i;
                const __amdgpu_buffer_rsrc_t to = buffer_of(static_cast<uint8_t*>(o.e) + ((tile_m + first) * o.pitch + tile_n) * 2, 0xFFFFFF00u);
                __builtin_amdgcn_raw_buffer_store_b128(out, to, in && tile_n + wcol < o.pitch ? ((8 * e + row) * (uint32_t)o.pitch + wcol) * 2 : BEYOND, 0, STREAM);
            }
            if (in && l % LANES == 0 && wn * T::COLS < cols) o.strips[(tile_m + r) * o.strips_row + tile_n / T::STRIP + wn] = f32x2{m, sum};
        }
        return o.e != nullptr;
    } else {
        const GemmEnd& o = g.end;
        const float scale = o.scale ? *o.scale : 1.f;
        Raw8<TYPE> bias;                                                      // as it lies
#pragma unroll
        for (uint32_t k = 0; k < EACH / 2; ++k) bias.r[k] = 0;
        if (o.bias)
#pragma unroll
            for (uint32_t k = 0; k < EACH; ++k)
                if (wcol + k < cols) bias.set(k, static_cast<const uint16_t*>(o.bias)[tile_n + wcol + k]);
        const uint32_t at = (row * (uint32_t)o.ld + wcol) * BYTES;
        f32x4 next[PASSES][EACH / 4];                                     // the sums of the pass after this one, on their way
#pragma unroll
        for (uint32_t i = 0; i < TI; ++i) {
            const uint32_t first = row0 + 32 * i;               // the store's rows begin here: the lanes' offsets are those of 32 rows, below 2^32
            const __amdgpu_buffer_rsrc_t to = buffer_of(static_cast<uint8_t*>(o.out) + ((tile_m + first) * o.ld + tile_n) * BYTES, 0xFFFFFF00u);
            // A residual of 16 bits: that of the 32 rows is under way before the first is used.
            const uint8_t* res_base = static_cast<const uint8_t*>(o.residual) + ((tile_m + first + row) * o.ld_res + tile_n + wcol) * (o.res32 ? 4 : 2);
            uint32_t res[4][PASSES][EACH / 2];
            if (o.residual && !o.res32) {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
                    for (uint32_t p = 0; p < PASSES; ++p) {
                        const uint32_t r = 8 * e + p * PASS_ROWS;
                        const uint16_t* q = reinterpret_cast<const uint16_t*>(res_base) + r * o.ld_res;
                        if (row_in && first + r + row < rows) {
                            if (whole) {
#pragma unroll
                                for (uint32_t k = 0; k < EACH / 2; k += 2) {
                                    const u32x2_any w = *reinterpret_cast<const u32x2_any*>(q + 2 * k);
                                    res[e][p][k] = w[0];
                                    res[e][p][k + 1] = w[1];
                                }
                            } else {
#pragma unroll
                                for (uint32_t k = 0; k < EACH; k += 2)
                                    res[e][p][k / 2] = (wcol + k < cols ? (uint32_t)q[k] : 0u) | (wcol + k + 1 < cols ? (uint32_t)q[k + 1] << 16 : 0u);
                            }
                        }
                    }
            }
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                f32x4 v[PASSES][EACH / 4], res32[PASSES][EACH / 4];
                if (i + e == 0) through(0, 0, next);
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p)
#pragma unroll
                    for (uint32_t k = 0; k < EACH / 4; ++k) v[p][k] = next[p][k];
                if (o.residual && o.res32) {
#pragma unroll
                    for (uint32_t p = 0; p < PASSES; ++p) {
                        const uint32_t r = 8 * e + p * PASS_ROWS;
                        const float* q = reinterpret_cast<const float*>(res_base) + r * o.ld_res;
                        if (row_in && first + r + row < rows)
#pragma unroll
                            for (uint32_t k = 0; k < EACH; k += 4) {
                                if (whole) res32[p][k / 4] = *reinterpret_cast<const f32x4_any*>(q + k);
                                else
#pragma unroll
                                    for (uint32_t h = 0; h < 4; ++h) res32[p][k / 4][h] = wcol + k + h < cols ? q[k + h] : 0.f;
                            }
                    }
                }
                if (4 * i + e + 1 < 4 * TI) through((4 * i + e + 1) / 4, (e + 1) % 4, next);
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p) {
                    // (the whole offset in the lane's register: a 16-byte store with a scalar offset as well has stored values that the next instructions
                    // wrote into its data registers, in rows with such an offset and in no others)
                    const uint32_t r = 8 * e + p * PASS_ROWS, to_at = at + r * (uint32_t)o.ld * BYTES;
                    const bool in = row_in && first + r + row < rows;
                    float x[EACH];
#pragma unroll
                    for (uint32_t k = 0; k < EACH; ++k) x[k] = v[p][k / 4][k % 4];
                    if (o.bias || o.scale)
#pragma unroll
                        for (uint32_t k = 0; k < EACH; ++k) x[k] = fmaf(x[k], scale, bias.at(k));
                    if (o.z && in) {
                        uint16_t* q = static_cast<uint16_t*>(o.z) + (tile_m + first + r + row) * o.ld_z + tile_n + wcol;
                        if (whole) {
#pragma unroll
                            for (uint32_t k = 0; k < EACH; k += 4) __builtin_nontemporal_store((u32x2_any{pack2<TYPE>(x[k], x[k + 1]), pack2<TYPE>(x[k + 2], x[k + 3])}), reinterpret_cast<u32x2_any*>(q + k));
                        } else if (cut) {
#pragma unroll
                            for (uint32_t k = 0; k < EACH; ++k)
                                if (wcol + k < cols) store1<TYPE>(q, k, x[k]);
                        }
                    }
                    with_act(o.act, [&](auto kind) {
#pragma unroll
                        for (uint32_t k = 0; k < EACH; ++k) x[k] = act_as<decltype(kind)::value>(x[k]);
                    });
                    if (o.residual)
#pragma unroll
                        for (uint32_t k = 0; k < EACH; ++k) {
                            const uint32_t w = res[e][p][k / 2] >> (16 * (k % 2)) & 0xFFFFu;
                            x[k] += o.res32 ? res32[p][k / 4][k % 4] : TYPE == TYPE_BF16 ? __uint_as_float(w << 16) : half_to_float(w);
                        }
                    u32x4 out;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) out[k] = BYTES == 4 ? __float_as_uint(x[k]) : pack2<TYPE>(x[2 * k % EACH], x[(2 * k + 1) % EACH]);
                    __builtin_amdgcn_raw_buffer_store_b128(out, to, in && whole ? to_at : BEYOND, 0, STREAM);
                    if (in && cut) {
#pragma unroll
                        for (uint32_t k = 0; k < EACH; ++k) {
                            const uint32_t ok = wcol + k < cols ? to_at + k * BYTES : BEYOND;
                            if (BYTES == 4) __builtin_amdgcn_raw_buffer_store_b32(out[k % 4], to, ok, 0, 0);
                            else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(out[k / 2 % 4] >> (16 * (k % 2))), to, ok, 0, 0);
                        }
                    }
                }
            }
        }
        if (cols % EACH == 0) return true;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // (so many more stores that the counter would not tell)
        return false;
    }
}

template <uint32_t TYPE, class T, bool ACROSS_A, bool ACROSS_B, uint32_t END>
__global__ __launch_bounds__(64 * T::WAVES, 2) void k_gemm_tile(GemmArgs g) {
    constexpr uint32_t BM = T::BM, BN = T::BN, WM = T::WM, WN = T::WN;
    __shared__ __attribute__((aligned(1024))) uint8_t s_mem[T::LDS];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = lds_address(s_mem), tiles = g.tiles_m * g.tiles_n, shared = tiles - g.whole, items = g.whole + shared * g.splits;
    const uint32_t stages = (uint32_t)((g.K + GEMM_STAGE_K - 1) / GEMM_STAGE_K);

    GemmSide<BM, T::WAVES, ACROSS_A> sa;
    GemmSide<BN, T::WAVES, ACROSS_B> sb;
    sa.begin(wave, lane, g.lda);
    sb.begin(wave, lane, g.ldb);
    // An item's tile, and the part of its sum that it is: the whole tiles come first, then the shared ones' first parts and so on.
    struct Item {
        uint32_t tile, part, first, count;                                    // first, count: stages
    };
    auto item_at = [&](uint32_t id) {
        if (id < g.whole) return Item{in_runs(id, g.whole), 0u, 0u, stages};
        const uint32_t i = in_runs(id - g.whole, shared * g.splits), part = i / shared, first = part * g.share;
        return Item{g.whole + i % shared, part, first, stages - first < g.share ? stages - first : g.share};
    };
    uint32_t stages_in;                                                       // of the item, this one counted
    auto aim = [&](uint32_t item) {
        uint32_t tm = 0, tn = 0;
        const bool none = item >= items;                                      // (behind the last one the loads go on, of nothing)
        const Item it = none ? Item{0u, 0u, 0u, stages} : item_at(item);
        if (!none) tile_at(it.tile, g.tiles_m, g.tiles_n, g.band, tm, tn);
        const uint32_t k0 = it.first * GEMM_STAGE_K;
        stages_in = it.count;
        sa.aim(g.a, (uint64_t)tm * BM, none ? 0 : g.M, k0, ACROSS_A ? (uint32_t)g.k_rows_a : (uint32_t)g.K);
        sb.aim(g.b, (uint64_t)tn * BN, none ? 0 : g.N, k0, ACROSS_B ? (uint32_t)g.k_rows_b : (uint32_t)g.K);
    };
    uint32_t item_in = blockIdx.x, buffer_in = 0;
    aim(item_in);
    // part `k` of `n` of a stage's loads
    auto bring = [&](uint32_t k, uint32_t n) {
        const uint32_t stage = lds0 + buffer_in * T::STAGE + wave * 1024u;
        const __amdgpu_buffer_rsrc_t from_a = sa.buffer(), from_b = sb.buffer();
        const uint32_t off_a = sa.lane_offset(), off_b = sb.lane_offset();
#pragma unroll
        for (uint32_t i = k * T::LOADS / n; i < (k + 1) * T::LOADS / n; ++i) {
            if (i < T::LA) load_lds16(from_a, off_a + i * sa.step(), 0, stage + i * T::WAVES * 1024u);
            else load_lds16(from_b, off_b + (i - T::LA) * sb.step(), 0, stage + BM * GEMM_STAGE_K * 2 + (i - T::LA) * T::WAVES * 1024u);
        }
    };
    auto brought = [&]() {
        buffer_in ^= 1u;
        sa.next();
        sb.next();
        if (--stages_in == 0) {
            item_in += gridDim.x;
            aim(item_in);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    const uint32_t wm = wave / WN, wn = wave % WN, r32 = lane & 31u, kb = lane >> 5;
    f32x16 acc[T::TI][T::TJ];
    struct Half {                                                             // the operands of 16 of K
        u32x4 a[T::TI], b[T::TJ];
    } half0, half1;
    // Where a lane reads: along K its row's 16 bytes, across K its four elements of a row of one k.
    const uint32_t turn = sa.turn(r32), k_lane = 8 * kb + ((lane & 15u) >> 2), in_piece = 32 * ((lane >> 4) & 1u) + 8 * (lane & 3u);
    auto lane_at = [&](uint32_t edge, uint32_t first, bool across) {          // of 32 rows of the tile from `first` on
        return across ? k_lane * edge * 2 + (((first >> 5) ^ (edge >= 128 ? k_lane & 3u : (k_lane >> 1) & 1u)) << 6) + in_piece : (first + r32) * GEMM_STAGE_K * 2;
    };
    // The k-th of the operands of 16 of K, in the order in which the products want them.
    constexpr uint32_t READS = T::TI + T::TJ;
    auto read = [&](uint32_t buffer, uint32_t step, uint32_t k, Half& h) {
        const uint8_t *at_a = s_mem + buffer * T::STAGE, *at_b = at_a + BM * GEMM_STAGE_K * 2;
        const uint32_t along = 16u * ((2 * step + kb) ^ turn), i = k == 0 ? 0 : k - T::TJ, j = k - 1;
        if (k == 0 || k > T::TJ) h.a[i] = gemm_operand<BM, ACROSS_A>(at_a + lane_at(BM, wm * (BM / WM) + 32 * i, ACROSS_A) + (ACROSS_A ? 0 : along), 16 * step);
        else h.b[j] = gemm_operand<BN, ACROSS_B>(at_b + lane_at(BN, wn * (BN / WN) + 32 * j, ACROSS_B) + (ACROSS_B ? 0 : along), 16 * step);
    };
    auto read_all = [&](uint32_t buffer, uint32_t step, Half& h) {
#pragma unroll
        for (uint32_t k = 0; k < READS; ++k) read(buffer, step, k, h);
    };
    auto multiply = [&](const Half& h, auto between) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
            for (uint32_t j = 0; j < T::TJ; ++j) {
                acc[i][j] = mfma32<TYPE>(h.a[i], h.b[j], acc[i][j]);
                // (used here: the compiler would otherwise move the products behind the branches and waits that follow, where no reads are left to hide)
                asm volatile("" : "+v"(acc[i][j]));
                between(i * T::TJ + j);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr uint32_t PRODUCTS = T::TI * T::TJ;
    // Reads along K go between the products that they run beside, those across K before them (8192 x 2048 x 5632: along 174 us before, 170 between; both across
    // 8192 x 8192 x 8192 870 and 1278: a read that transposes is two).
    constexpr bool BETWEEN = !ACROSS_A && !ACROSS_B;
    auto read_beside = [&](uint32_t buffer, uint32_t step, uint32_t k, Half& h) {
        if (!BETWEEN) return;
#pragma unroll
        for (uint32_t r = k * READS / PRODUCTS; r < (k + 1) * READS / PRODUCTS; ++r) read(buffer, step, r, h);
    };
    // The reads of one half are under way while the other is multiplied, across stages and items too; the barrier in front of a stage's last 16 of K waits
    // for the next stage, and behind it this stage's buffer takes the one after the next.  A tile is stored while the next item's first stage
    // comes; the next barrier lets these stores be.
    constexpr uint32_t STORES = END == END_F32 ? 4 * T::TI * T::TJ : 4 * T::TI;
    bring(0, 1);
    brought();
    bring(0, 1);
    brought();
    vm_wait_barrier<T::LOADS, 0>(0);
    uint32_t buffer = 0;
    read_all(0, 0, half0);
    uint32_t stores_behind = 0;                                               // 1: a tile's stores, STORES or more, are behind the loads that the next barrier waits for
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t here = item_at(item).count;
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
            for (uint32_t j = 0; j < T::TJ; ++j) acc[i][j] = f32x16{};
#pragma nounroll
        for (uint32_t s = 0; s < here; ++s) {
#pragma unroll
            for (uint32_t step = 1; step < T::STEPS; ++step) {
                if (!BETWEEN) read_all(buffer, step, step % 2 ? half1 : half0);
                multiply(step % 2 ? half0 : half1, [&](uint32_t k) { read_beside(buffer, step, k, step % 2 ? half1 : half0); });
            }
            vm_wait_barrier<0, STORES>(stores_behind);
            stores_behind = 0;
            buffer ^= 1u;
            if (!BETWEEN) read_all(buffer, 0, half0);                         // (behind the last item reads and loads go on, of a buffer and of nothing)
            multiply(half1, [&](uint32_t k) {
                read_beside(buffer, 0, k, half0);
                bring(k, PRODUCTS);                                           // (between the products, what sets up the loads costs no time)
            });
            brought();
        }

        const Item it = item_at(item);
        if (END != END_SOFTMAX && item >= g.whole) {
            uint32_t l;                                                       // the lane, found anew: kept through the loop, it would cost a register
            asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
            f32x4* to = reinterpret_cast<f32x4*>(g.parts + ((uint64_t)it.part * shared + it.tile - g.whole) * (BM * BN)) + wave * (T::TI * T::TJ * 256) + l;
#pragma unroll
            for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
                for (uint32_t j = 0; j < T::TJ; ++j) {
                    const f32x16 x = acc[i][j];
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) to[(4 * (i * T::TJ + j) + e) * 64] = f32x4{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]};
                }
            stores_behind = 1;
        } else {
            uint32_t tm, tn;
            tile_at(it.tile, g.tiles_m, g.tiles_n, g.band, tm, tn);
            float* mine = reinterpret_cast<float*>(s_mem + 2 * T::STAGE + wave * T::OUT);
            const bool counted = gemm_end<TYPE, T, T::TI, END>(g, acc, mine, (uint64_t)tm * BM, (uint64_t)tn * BN, wm * (BM / WM), wn);
            stores_behind = counted ? 1u : 0u;
        }
        read_all(buffer, 0, half0);                                           // (once more: kept through the end, it would cost 24 registers)
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                          // no load may reach LDS that is another workgroup's by then
}

// The parts of the shared tiles' sums, in their order, and their end: a wave takes 32 rows of one wave's part of a tile.  Bound by memory.
template <uint32_t TYPE, class T, uint32_t END>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g) {
    __shared__ __attribute__((aligned(16))) uint8_t s_mem[4 * T::OUT];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t shared = g.tiles_m * g.tiles_n - g.whole, unit = blockIdx.x * 4 + wave, t = unit / (T::WAVES * T::TI);
    if (t >= shared) return;
    const uint32_t w = unit / T::TI % T::WAVES, i = unit % T::TI;
    uint32_t tm, tn;
    tile_at(g.whole + t, g.tiles_m, g.tiles_n, g.band, tm, tn);
    const uint64_t tile_m = (uint64_t)tm * T::BM, tile_n = (uint64_t)tn * T::BN;
    const uint32_t row0 = w / T::WN * (T::BM / T::WM) + 32 * i, wn = w % T::WN;
    if (tile_m + row0 >= g.M || tile_n + wn * T::COLS >= g.N) return;
    const f32x4* from = reinterpret_cast<const f32x4*>(g.parts + (uint64_t)t * (T::BM * T::BN)) + (w * T::TI + i) * (T::TJ * 256) + lane;
    const uint64_t step = (uint64_t)shared * (T::BM * T::BN / 4);
    f32x16 acc[1][T::TJ];
#pragma unroll
    for (uint32_t j = 0; j < T::TJ; ++j) acc[0][j] = f32x16{};
    constexpr uint32_t U = 4;                                                 // parts under way together
    for (uint32_t p = 0; p < g.splits; p += U) {
        f32x4 v[U][T::TJ * 4];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t k = 0; k < T::TJ * 4; ++k)
                if (p + u < g.splits) v[u][k] = from[(p + u) * step + k * 64];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
            if (p + u < g.splits)
#pragma unroll
                for (uint32_t k = 0; k < T::TJ * 16; ++k) acc[0][k / 16][k % 16] += v[u][k / 4][k % 4];
    }
    gemm_end<TYPE, T, 1, END>(g, acc, reinterpret_cast<float*>(s_mem + wave * T::OUT), tile_m, tile_n, row0, wn);
}

}  // namespace kimad
