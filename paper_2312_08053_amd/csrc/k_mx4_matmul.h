// Product of two matrices of microscaled 4-bit floats, C [M, N] = A [M, K] B [N, K]^T, sums in fp32.
//
// The matrix instructions take 4-bit operands with a scale byte a block, so nothing is decoded:
//   v_mfma_scale_f32_32x32x64:   lane l holds block l / 32 of row l % 32 (16 bytes of codes) and its scale byte, of A and of B; element i of
//                                the result's lane l is C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32]
//   v_mfma_scale_f32_16x16x128:  block l / 16 of row l % 16; element i is C[4 (l / 16) + i][l % 16]
#pragma once
#include "mx4.h"

namespace kimad {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
    const uint8_t *a, *b;        // codes
    const uint32_t *sa, *sb;     // scale words
    void* out;
    uint64_t M, N, W, ld;        // W words a row
    uint64_t scale_rows;         // rows of the matrix that A's M rows are of: from word to word of A's scales
    uint32_t tiles_m, tiles_n;
    uint32_t splits, share;      // parts of the sum, `share` stages each (the last one fewer); more than one: part p goes to out + p M ld
};

__device__ __forceinline__ i32x8 mx4_operand(u32x4 v) { return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0}; }

// 16 bytes of every lane from `offset` of a buffer to LDS, at `lds` + 16 * lane, without a register in between; a lane beyond the buffer brings zeros.  The
// LDS address is a number here: the compiler then leaves it to the kernel's own waits (vm_wait_barrier) which of these loads a read of LDS needs.
typedef __attribute__((address_space(3))) uint32_t lds_u32;
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint32_t scalar_offset, uint32_t lds) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_u32*)(uintptr_t)lds, 16, (int)offset, (int)scalar_offset, 0, 0);
}
// 4 bytes of every lane, at `lds` + 4 * lane.
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint32_t lds) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_u32*)(uintptr_t)lds, 4, (int)offset, 0, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// Until the wave's loads and stores are done but for the last N of them, or the last N + MORE where `more` is not 0; then the workgroup's barrier.  (One
// piece of assembly, so that the loop around it stays one loop.)
template <uint32_t N, uint32_t MORE>
__device__ __forceinline__ void vm_wait_barrier(uint32_t more) {
    static_assert(N + MORE < 64, "what the counter holds");
    asm volatile("s_cmp_lg_u32 %2, 0\n\ts_cbranch_scc1 .Lmore%=\n\ts_waitcnt vmcnt(%0)\n.Lmore%=:\n\ts_waitcnt vmcnt(%1) lgkmcnt(0)\n\ts_barrier" ::"n"(N), "n"(N + MORE),
                 "s"(__builtin_amdgcn_readfirstlane(more)) : "memory", "scc");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p);
}

// Tile number -> tile.  Workgroups go to the eight XCDs in turn; an XCD takes a run of tiles, in bands of eight rows of tiles, so that what its
// compute units read at a time stays in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t& m, uint32_t& n) {
    const uint32_t total = tm * tn, xcd = id & 7u, each = total >> 3, more = total & 7u;
    id = xcd * each + (xcd < more ? xcd : more) + (id >> 3);
    const uint32_t band = 8u * tn, first = id / band * 8u, high = tm - first < 8u ? tm - first : 8u, r = id % band;
    m = first + r % high;
    n = r / high;
}

// A tile of BM by BN, WM by WN waves.  Two words of K are a stage, of which LDS holds two: codes (128 bytes a row, whole cache lines: a word at a time, four
// stages, took 8 % longer) and scale words.  The blocks of a row are stored in an order that turns with the row (block b of row r at b ^ (r / 2 % 8)), so
// that sixteen lanes that read one block of sixteen rows meet sixteen different groups of banks.
// What bounds it: K = 16384, a tile of 256 a unit, 64 stages take a unit 220 thousand cycles by the counters, of which its matrix cores work in 131 thousand.  The loads
// alone (a copy of the kernel without products) took some 187 thousand, 25 bytes a clock however they are made, reads of LDS alone 100: the loads, and
// what of the products is not hidden beside them.  On codes of zero these cycles run at 2.5 GHz, 98 us, on random ones at 1.95, 130 us: that much is
// the power limit's.  8192 x 5632 x 2048 into bfloat16 60 to 65 us by machine, 2.9 to 3.1 PFLOP/s; 50257 x 768 x 8192 into fp32 187 to 205 us, 3.1 to 3.4.
template <uint32_t BM_, uint32_t BN_, uint32_t WM_, uint32_t WN_>
struct MatmulTile {
    static constexpr uint32_t BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr uint32_t WAVES = WM * WN, TI = BM / WM / 32, TJ = BN / WN / 32;
    static constexpr uint32_t LOADS = (BM + BN) / 8 / WAVES, GROUPS = (BM + BN) / 32, SLOADS = (GROUPS + WAVES - 1) / WAVES;
    static constexpr uint32_t CODES = (BM + BN) * 128, STAGE = CODES + (BM + BN) * 8;
    static constexpr uint32_t COLS = 32 * TJ, PITCH = COLS + 8;               // of a wave's rows on their way out: 4 rows further, 32 banks further
    static constexpr uint32_t OUT = 8 * PITCH * 4, LDS = 2 * STAGE + WAVES * OUT;
};

template <uint32_t TYPE, class T>
__global__ __launch_bounds__(64 * T::WAVES, 2) void k_mx4_matmul_tile(MatmulArgs g) {
    constexpr uint32_t BM = T::BM, BN = T::BN, WM = T::WM, WN = T::WN;
    __shared__ __attribute__((aligned(1024))) uint8_t s_mem[T::LDS];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t row_bytes = g.W * 64, stages = (g.W + 1) / 2;
    const uint32_t lds0 = lds_address(s_mem), tiles = g.tiles_m * g.tiles_n, items = tiles * g.splits;

    // what the lane brings: of 8 rows a load, block (lane % 8) ^ (row / 2 % 8) of row lane / 8; zeros beyond the matrix
    static_assert(T::WAVES % 2 == 0, "a wave's groups of 8 rows have the same order of blocks");
    const uint32_t block = (lane & 7u) ^ ((4u * wave + (lane >> 4)) & 7u), offset = (lane >> 3) * (uint32_t)row_bytes + 16u * block;
    __amdgpu_buffer_rsrc_t from[T::LOADS];
    const uint32_t* sbase[T::SLOADS];
    uint32_t sbytes[T::SLOADS];
    uint64_t stage_in, stage_end;
    auto aim = [&](uint32_t item) {
        uint32_t tm = 0, tn = 0;
        const bool none = item >= items;                                      // (behind the last one the loads go on, of nothing)
        if (!none) tile_of(item % tiles, g.tiles_m, g.tiles_n, tm, tn);
        stage_in = none ? 0 : (uint64_t)(item / tiles) * g.share;
        stage_end = stage_in + g.share < stages ? stage_in + g.share : stages;
        const uint64_t m0 = (uint64_t)tm * BM, n0 = (uint64_t)tn * BN;
#pragma unroll
        for (uint32_t i = 0; i < T::LOADS; ++i) {
            const uint32_t group = i * T::WAVES + wave;                       // of 8 rows: A's first, then B's
            const bool of_a = group < BM / 8;
            const uint64_t first = (of_a ? m0 : n0) + 8 * (of_a ? group : group - BM / 8), rows = none ? 0 : of_a ? g.M : g.N;
            from[i] = buffer_of((of_a ? g.a : g.b) + first * row_bytes, first < rows ? (uint32_t)(rows - first < 8 ? rows - first : 8) * (uint32_t)row_bytes : 0u);
        }
#pragma unroll
        for (uint32_t i = 0; i < T::SLOADS; ++i) {
            const uint32_t half = (i * T::WAVES + wave) % T::GROUPS % (T::GROUPS / 2);   // of 64 rows' scale words: A's, B's, then those of a second word
            const bool of_a = half < BM / 64;
            const uint64_t first = (of_a ? m0 : n0) + 64 * (of_a ? half : half - BM / 64), rows = none ? 0 : of_a ? g.M : g.N;
            sbase[i] = (of_a ? g.sa : g.sb) + first + (2 * stage_in + (i * T::WAVES + wave) % T::GROUPS / (T::GROUPS / 2)) * (of_a ? g.scale_rows : g.N);
            sbytes[i] = first < rows ? (uint32_t)(rows - first < 64 ? rows - first : 64) * 4u : 0u;
        }
    };
    // The stages of all the workgroup's items, one after another, into the two buffers in turn.
    uint32_t item_in = blockIdx.x, buffer_in = 0;
    aim(item_in);
    // part `k` of `n` of a stage's loads
    auto bring = [&](uint32_t k, uint32_t n) {
        const uint32_t stage = lds0 + buffer_in * T::STAGE;
        const bool one = 2 * stage_in + 1 == g.W;                             // (then the second word's codes are zeros, with the first one's scales)
        const uint32_t lane_offset = one && block >= 4 ? 0xFFFFFFF0u : offset;
#pragma unroll
        for (uint32_t i = k * T::LOADS / n; i < (k + 1) * T::LOADS / n; ++i)
            load_lds16(from[i], lane_offset, (uint32_t)stage_in * 128u, stage + (i * T::WAVES + wave) * 1024u);
        if (k + 1 < n) return;
#pragma unroll
        for (uint32_t i = 0; i < T::SLOADS; ++i) {
            const uint32_t group = (i * T::WAVES + wave) % T::GROUPS;
            const uint64_t rows = group % (T::GROUPS / 2) < BM / 64 ? g.scale_rows : g.N;
            load_lds4(buffer_of(one && group >= T::GROUPS / 2 ? sbase[i] - rows : sbase[i], sbytes[i]), 4 * lane, stage + T::CODES + group * 256u);
            sbase[i] += 2 * rows;
        }
    };
    auto brought = [&]() {
        buffer_in ^= 1u;
        if (++stage_in == stage_end) {
            item_in += gridDim.x;
            aim(item_in);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    const uint32_t wm = wave / WN, wn = wave % WN, r32 = lane & 31u, kb = lane >> 5;
    const uint32_t a_row = wm * (BM / WM) + r32, b_row = BM + wn * (BN / WN) + r32;
    f32x16 acc[T::TI][T::TJ];
    // The operands of half a word: its codes, and the scale words turned so that the lane's own bytes are the lowest and the third.
    struct Half {
        u32x4 a[T::TI], b[T::TJ];
    } half0, half1;
    uint32_t sa[T::TI], sb[T::TJ], sa_raw[T::TI], sb_raw[T::TJ];
    const uint32_t turn = (r32 >> 1) & 7u;                      // (rows 32 apart have the same order of blocks)
    auto read = [&](uint32_t buffer, uint32_t word, uint32_t step, Half& h) {
        const uint8_t* at = s_mem + buffer * T::STAGE + 16u * ((4 * word + 2 * step + kb) ^ turn);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) h.a[i] = *reinterpret_cast<const u32x4*>(at + (a_row + 32 * i) * 128);
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) h.b[j] = *reinterpret_cast<const u32x4*>(at + (b_row + 32 * j) * 128);
    };
    auto read_scales = [&](uint32_t buffer, uint32_t word) {
        const uint32_t* words = reinterpret_cast<const uint32_t*>(s_mem + buffer * T::STAGE + T::CODES) + word * (BM + BN);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) sa_raw[i] = words[a_row + 32 * i];
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) sb_raw[j] = words[b_row + 32 * j];
    };
    auto turn_scales = [&]() {
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) sa[i] = sa_raw[i] >> (8 * kb);
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) sb[j] = sb_raw[j] >> (8 * kb);
    };
    auto multiply = [&](const Half& h, auto opsel, auto between) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
            for (uint32_t j = 0; j < T::TJ; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(h.a[i]), mx4_operand(h.b[j]), acc[i][j], 4, 4, decltype(opsel)::value, sa[i],
                                                                             decltype(opsel)::value, sb[j]);
                // (used here: the compiler would otherwise move the products behind the branches and waits that follow, where no reads are left to hide)
                asm volatile("" : "+v"(acc[i][j]));
                between(i * T::TJ + j);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto nothing = [](uint32_t) {};
    constexpr std::integral_constant<int, 0> first_half{};
    constexpr std::integral_constant<int, 2> second_half{};
    // The reads of one half are under way while the other is multiplied, across stages and items too: the barrier in front of a stage's last half waits for
    // the next stage, whose first half is then read, and behind it this stage is no longer read and its buffer takes the one after the next.  A
    // tile is stored while the next item's first stage comes; the next barrier lets these stores be.
    constexpr uint32_t STORES = 4 * T::TI * (TYPE == TYPE_F32 ? T::TJ : 1);
    bring(0, 1);
    brought();
    bring(0, 1);
    brought();
    vm_wait_barrier<T::LOADS + T::SLOADS, 0>(0);
    uint32_t buffer = 0;
    read_scales(0, 0);
    read(0, 0, 0, half0);
    uint32_t stores_behind = 0;                                               // 1: the wave's last STORES accesses are a tile's stores
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint64_t first = (uint64_t)(item / tiles) * g.share, here = stages - first < g.share ? stages - first : g.share;
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
            for (uint32_t j = 0; j < T::TJ; ++j) acc[i][j] = f32x16{};
#pragma nounroll
        for (uint64_t s = 0; s < here; ++s) {
            turn_scales();
            read(buffer, 0, 1, half1);
            multiply(half0, first_half, nothing);
            read_scales(buffer, 1);
            read(buffer, 1, 0, half0);
            multiply(half1, second_half, nothing);
            turn_scales();
            read(buffer, 1, 1, half1);
            multiply(half0, first_half, nothing);
            vm_wait_barrier<0, STORES>(stores_behind);
            stores_behind = 0;
            buffer ^= 1u;
            read_scales(buffer, 0);                                           // (behind the last item: of a buffer, and for nothing)
            read(buffer, 0, 0, half0);
            multiply(half1, second_half, [&](uint32_t k) { bring(k, T::TI * T::TJ); });   // the loads between the products: what sets them up costs no time
            brought();
        }

        uint32_t tm, tn;
        tile_of(item % tiles, g.tiles_m, g.tiles_n, tm, tn);
        const uint64_t tile_m = (uint64_t)tm * BM, tile_n = (uint64_t)tn * BN;
        // Eight rows at a time through LDS, so that stores run along the rows: 16 bytes a lane, whole cache lines.  (Four columns a lane by lane exchanges, whose
        // neighbours stored to four rows, took 75 us for 8192 x 5632 x 2048 in 16 bits, and this 61; 85 and 44 for 1000 x 50257 x 768.)
        constexpr uint32_t BYTES = TYPE == TYPE_F32 ? 4 : 2, BEYOND = 0xFFFFFFF0u, EACH = 16 / BYTES, LANES = T::COLS / EACH;   // elements of a lane, lanes of a row
        constexpr uint32_t PASSES = 8 * LANES > 64 ? 8 * LANES / 64 : 1, PASS_ROWS = 8 / PASSES;
        uint32_t l;                                                           // the lane, found anew: kept through the loop, it would cost a register
        asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
        float* mine = reinterpret_cast<float*>(s_mem + 2 * T::STAGE + wave * T::OUT);
        const uint32_t rows = g.M - tile_m < BM ? (uint32_t)(g.M - tile_m) : BM, cols = g.N - tile_n < BN ? (uint32_t)(g.N - tile_n) : BN;
        const bool cut = cols % EACH != 0;                                    // some lanes have elements on both sides of the last column
        const uint32_t row = l / LANES, col = EACH * (l % LANES), wcol = wn * T::COLS + col, at = (row * (uint32_t)g.ld + wcol) * BYTES;
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) {
            const uint32_t first = wm * (BM / WM) + 32 * i;                   // the store's rows begin here: the lanes' offsets are those of 32 rows, below 2^32
            const __amdgpu_buffer_rsrc_t to = buffer_of(static_cast<uint8_t*>(g.out) + (((item / tiles) * g.M + tile_m + first) * g.ld + tile_n) * BYTES, 0xFFFFFF00u);
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
#pragma unroll
                for (uint32_t j = 0; j < T::TJ; ++j) {
                    const f32x16 v = acc[i][j];
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) mine[(4 * (l >> 5) + k) * T::PITCH + 32 * j + (l & 31u)] = v[4 * e + k];
                }
                wave_sync_lds();
                f32x4 v[PASSES][EACH / 4];
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p)
#pragma unroll
                    for (uint32_t q = 0; q < EACH / 4; ++q) v[p][q] = *reinterpret_cast<const f32x4*>(mine + ((p * PASS_ROWS + row) & 7u) * T::PITCH + col + 4 * q);
                wave_sync_lds();
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p) {
                    // (the whole offset in the lane's register: a 16-byte store with a scalar offset as well has stored values that the next instructions
                    // wrote into its data registers, in rows with such an offset and in no others)
                    const uint32_t r = 8 * e + p * PASS_ROWS, o = at + r * (uint32_t)g.ld * BYTES;
                    u32x4 out;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if (TYPE == TYPE_F32) out[k] = __float_as_uint(v[p][0][k]);
                        else out[k] = pack2<TYPE>(v[p][(k / 2) % (EACH / 4)][2 * k % 4], v[p][(k / 2) % (EACH / 4)][2 * k % 4 + 1]);
                    }
                    const bool in = (PASSES > 1 || row < 8) && first + r + row < rows;
                    __builtin_amdgcn_raw_buffer_store_b128(out, to, in && wcol + EACH <= cols ? o : BEYOND, 0, 0);
                    if (cut && in && wcol < cols && wcol + EACH > cols) {
#pragma unroll
                        for (uint32_t k = 0; k < EACH; ++k) {
                            const uint32_t ok = wcol + k < cols ? o + k * BYTES : BEYOND;
                            if (TYPE == TYPE_F32) __builtin_amdgcn_raw_buffer_store_b32(out[k % 4], to, ok, 0, 0);
                            else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(out[k / 2] >> (16 * (k % 2))), to, ok, 0, 0);
                        }
                    }
                }
            }
        }
        stores_behind = cut ? 0u : 1u;
        if (cut) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // (so many more stores that the counter would not tell)
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                          // no load may reach LDS that is another workgroup's by then
}

// The parts of a sum, in their order.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_matmul_join(const float* __restrict__ parts, uint32_t splits, uint64_t M, uint64_t N, void* __restrict__ out, uint64_t ld) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= M * N) return;
    float v = parts[i];
    for (uint32_t p = 1; p < splits; ++p) v += parts[p * M * N + i];
    store1<TYPE>(out, i / N * ld + i % N, v);
}

// Few rows of A: sixteen rows of B by a wave, or by a workgroup's four (SPLIT: each takes a quarter of the words), which go straight to registers, U words under way
// at a time.  Bound by the reads of B: one row by 32000 x 2048 7.9 us, 4.4 TB/s.  MT: sixteens of A's rows.
template <uint32_t TYPE, uint32_t MT, bool SPLIT>
__global__ __launch_bounds__(256) void k_mx4_matmul_few(MatmulArgs g) {
    __shared__ f32x4 s_part[SPLIT ? 3 : 1][MT][64];
    constexpr uint32_t U = MT == 1 ? 8 : 4;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, blk = lane >> 4;
    const uint64_t n0 = ((uint64_t)blockIdx.x * (SPLIT ? 1 : 4) + (SPLIT ? 0 : wave)) * 16, n = n0 + r < g.N ? n0 + r : g.N - 1;
    if (!SPLIT && n0 >= g.N) return;
    // (a multiple of two words: whole cache lines)
    const uint64_t quarter = (g.W + 7) / 8 * 2, begin = SPLIT ? wave * quarter : 0, end = !SPLIT || begin + quarter > g.W ? g.W : begin + quarter;
    const u32x4* b = reinterpret_cast<const u32x4*>(g.b) + n * g.W * 4 + blk;
    const u32x4* a[MT];
    uint64_t m[MT];
    f32x4 acc[MT];
#pragma unroll
    for (uint32_t t = 0; t < MT; ++t) {
        m[t] = 16 * t + r < g.M ? 16 * t + r : g.M - 1;
        a[t] = reinterpret_cast<const u32x4*>(g.a) + m[t] * g.W * 4 + blk;
        acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto words = [&](uint64_t w, auto count) {
        constexpr uint32_t C = decltype(count)::value;
        u32x4 vb[C], va[C][MT];
        uint32_t sb[C], sa[C][MT];
#pragma unroll
        for (uint32_t u = 0; u < C; ++u) {
            vb[u] = b[(w + u) * 4];
            sb[u] = g.sb[(w + u) * g.N + n];
#pragma unroll
            for (uint32_t t = 0; t < MT; ++t) {
                va[u][t] = a[t][(w + u) * 4];
                sa[u][t] = g.sa[(w + u) * g.scale_rows + m[t]];
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < C; ++u)
#pragma unroll
            for (uint32_t t = 0; t < MT; ++t)
                acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(va[u][t]), mx4_operand(vb[u]), acc[t], 4, 4, 0, sa[u][t] >> (8 * blk), 0, sb[u] >> (8 * blk));
    };
    uint64_t w = begin;
    for (; w + U <= end; w += U) words(w, std::integral_constant<uint32_t, U>{});
    for (; w < end; ++w) words(w, std::integral_constant<uint32_t, 1>{});
    if (SPLIT) {
        if (wave)
#pragma unroll
            for (uint32_t t = 0; t < MT; ++t) s_part[wave - 1][t][lane] = acc[t];
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (uint32_t t = 0; t < MT; ++t) acc[t] = acc[t] + s_part[0][t][lane] + s_part[SPLIT ? 1 : 0][t][lane] + s_part[SPLIT ? 2 : 0][t][lane];
    }
#pragma unroll
    for (uint32_t t = 0; t < MT; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint64_t row = 16 * t + 4 * blk + i;
            if (row < g.M && n0 + r < g.N) store1<TYPE>(g.out, row * g.ld + n0 + r, acc[t][i]);
        }
}

// A product over no words.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_mx4_matmul_none(void* out, uint64_t M, uint64_t N, uint64_t ld) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < M * N) store1<TYPE>(out, i / N * ld + i % N, 0.f);
}

}  // namespace kimad
