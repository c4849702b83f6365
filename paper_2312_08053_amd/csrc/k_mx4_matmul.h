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
    uint32_t tiles_m, tiles_n;
};

__device__ __forceinline__ i32x8 mx4_operand(u32x4 v) { return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0}; }

// 16 bytes of every lane from `offset` of a buffer to LDS, at `lds` + 16 * lane, without a register in between; a lane beyond the buffer brings zeros.  The
// LDS address is a number here: the compiler then leaves it to the kernel's own waits (vm_wait_barrier) which of these loads a read of LDS needs.
typedef __attribute__((address_space(3))) uint32_t lds_u32;
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint32_t scalar_offset, uint32_t lds) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_u32*)(uintptr_t)lds, 16, (int)offset, (int)scalar_offset, 0, 0);
}
// 4 bytes of every lane, at `lds` + 4 * lane.
__device__ __forceinline__ void load_lds4(const void* base, uint32_t offset, uint32_t lds) {
    __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) uint32_t*)((uintptr_t)base + offset), (lds_u32*)(uintptr_t)lds, 4, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// Until at most N of the wave's loads are under way; then the workgroup's barrier.
template <uint32_t N>
__device__ __forceinline__ void vm_wait_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
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

// A tile of BM by BN, WM by WN waves.  Two words of K at a time, a stage, of which LDS holds two: codes (128 bytes a row, whole cache lines) and scale
// words.  The blocks of a row are stored in an order that turns with the row (block b of row r at b ^ (r / 2 % 8)), so that sixteen lanes that
// read one block of sixteen rows meet sixteen different groups of banks.
template <uint32_t BM, uint32_t BN, uint32_t WM, uint32_t WN>
struct MatmulTile {
    static constexpr uint32_t WAVES = WM * WN, TI = BM / WM / 32, TJ = BN / WN / 32;
    static constexpr uint32_t LOADS = (BM + BN) / 8 / WAVES, GROUPS = (BM + BN) / 64 * 2, SLOADS = (GROUPS + WAVES - 1) / WAVES;
    static constexpr uint32_t CODES = (BM + BN) * 128, STAGE = CODES + (BM + BN) * 8;
    static constexpr uint32_t PITCH = 32 * TJ + 8;                            // of a row in the epilogue: 4 rows further, 32 banks further
    static constexpr uint32_t LDS = 2 * STAGE > WAVES * 32 * PITCH * 4 ? 2 * STAGE : WAVES * 32 * PITCH * 4;
};

template <uint32_t TYPE, uint32_t BM, uint32_t BN, uint32_t WM, uint32_t WN>
__global__ __launch_bounds__(64 * WM * WN) void k_mx4_matmul_tile(MatmulArgs g) {
    using T = MatmulTile<BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) uint8_t s_mem[T::LDS];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const uint64_t m0 = (uint64_t)tm * BM, n0 = (uint64_t)tn * BN, row_bytes = g.W * 64;

    // what the lane brings: of 8 rows a load, block (lane % 8) ^ (row / 2 % 8) of row lane / 8; zeros beyond the matrix.  Of a last stage of one
    // word the lanes that would bring the second one bring the first.
    static_assert(T::WAVES % 2 == 0, "a wave's groups of 8 rows have the same order of blocks");
    const uint32_t block = (lane & 7u) ^ ((4u * wave + (lane >> 4)) & 7u), offset = (lane >> 3) * (uint32_t)row_bytes + 16u * block;
    __amdgpu_buffer_rsrc_t from[T::LOADS];
#pragma unroll
    for (uint32_t i = 0; i < T::LOADS; ++i) {
        const uint32_t group = i * T::WAVES + wave;                           // of 8 rows: A's first, then B's
        const bool of_a = group < BM / 8;
        const uint64_t first = (of_a ? m0 : n0) + 8 * (of_a ? group : group - BM / 8), rows = of_a ? g.M : g.N;
        from[i] = buffer_of((of_a ? g.a : g.b) + first * row_bytes, first < rows ? (uint32_t)(rows - first < 8 ? rows - first : 8) * (uint32_t)row_bytes : 0u);
    }
    uint32_t soffset[T::SLOADS], sto[T::SLOADS], sword[T::SLOADS];
    const uint32_t* sbase[T::SLOADS];
    uint64_t srows[T::SLOADS];
#pragma unroll
    for (uint32_t i = 0; i < T::SLOADS; ++i) {
        const uint32_t group = (i * T::WAVES + wave) % T::GROUPS;             // of 64 rows' scale words: A's, B's, then those of the second word
        const uint32_t half = group % (T::GROUPS / 2);
        const bool of_a = half < BM / 64;
        const uint64_t first = of_a ? m0 : n0;
        srows[i] = of_a ? g.M : g.N;
        const uint32_t r = (of_a ? half : half - BM / 64) * 64 + lane, most = (uint32_t)(srows[i] - first < 256 ? srows[i] - first : 256) - 1;
        sbase[i] = (of_a ? g.sa : g.sb) + first;
        soffset[i] = 4u * (r < most ? r : most);
        sword[i] = group / (T::GROUPS / 2);
        sto[i] = T::CODES + group * 256u;
    }
    const uint32_t lds0 = lds_address(s_mem);
    const uint64_t stages = (g.W + 1) / 2;

    auto bring = [&](uint64_t s) {
        const uint32_t stage = lds0 + (uint32_t)(s & 1) * T::STAGE;
        const bool one = 2 * s + 1 == g.W;
#pragma unroll
        for (uint32_t i = 0; i < T::LOADS; ++i) load_lds16(from[i], one && block >= 4 ? offset - 64u : offset, (uint32_t)s * 128u, stage + (i * T::WAVES + wave) * 1024u);
#pragma unroll
        for (uint32_t i = 0; i < T::SLOADS; ++i) load_lds4(sbase[i] + (2 * s + (one ? 0 : sword[i])) * srows[i], soffset[i], stage + sto[i]);
    };

    const uint32_t wm = wave / WN, wn = wave % WN, r32 = lane & 31u, kb = lane >> 5;
    const uint32_t a_row = wm * (BM / WM) + r32, b_row = BM + wn * (BN / WN) + r32;
    f32x16 acc[T::TI][T::TJ];
#pragma unroll
    for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) acc[i][j] = f32x16{};

    // The operands of half a word: its codes, and the scale words turned so that the lane's own bytes are the lowest and the third.
    struct Half {
        u32x4 a[T::TI], b[T::TJ];
    } half0, half1;
    uint32_t sa[2][T::TI], sb[2][T::TJ];
    const uint32_t turn = (r32 >> 1) & 7u;                                    // (rows 32 apart have the same order of blocks)
    auto read = [&](uint64_t s, uint32_t word, uint32_t step, Half& h) {
        const uint8_t* at = s_mem + (uint32_t)(s & 1) * T::STAGE + 16u * ((4 * word + 2 * step + kb) ^ turn);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) h.a[i] = *reinterpret_cast<const u32x4*>(at + (a_row + 32 * i) * 128);
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) h.b[j] = *reinterpret_cast<const u32x4*>(at + (b_row + 32 * j) * 128);
    };
    auto read_scales = [&](uint64_t s, uint32_t word) {
        const uint32_t* words = reinterpret_cast<const uint32_t*>(s_mem + (uint32_t)(s & 1) * T::STAGE + T::CODES) + word * (BM + BN);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) sa[word][i] = words[a_row + 32 * i];
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) sb[word][j] = words[b_row + 32 * j];
    };
    auto turn_scales = [&](uint32_t word) {
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i) sa[word][i] >>= 8 * kb;
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j) sb[word][j] >>= 8 * kb;
    };
    auto multiply = [&](const Half& h, uint32_t word, auto opsel) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < T::TI; ++i)
#pragma unroll
            for (uint32_t j = 0; j < T::TJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(h.a[i]), mx4_operand(h.b[j]), acc[i][j], 4, 4, decltype(opsel)::value, sa[word][i],
                                                                             decltype(opsel)::value, sb[word][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> first_half{};
    constexpr std::integral_constant<int, 2> second_half{};
    // The reads of one half are under way while the other is multiplied, across stages too: the barrier in front of a stage's last half waits for the
    // next stage, whose first half is then read, and behind it this stage is no longer read and its buffer takes the one after the next.
    if (g.W) {
        bring(0);
        if (stages > 1) {
            bring(1);
            vm_wait_barrier<T::LOADS + T::SLOADS>();
        } else {
            vm_wait_barrier<0>();
        }
        read_scales(0, 0);
        read(0, 0, 0, half0);
    }
    for (uint64_t s = 0; s < g.W / 2; ++s) {
        turn_scales(0);
        read(s, 0, 1, half1);
        multiply(half0, 0, first_half);
        read_scales(s, 1);
        read(s, 1, 0, half0);
        multiply(half1, 0, second_half);
        turn_scales(1);
        read(s, 1, 1, half1);
        multiply(half0, 1, first_half);
        vm_wait_barrier<0>();
        if (s + 2 < stages) bring(s + 2);
        read_scales(s + 1, 0);                                                // (behind the last stage: of a buffer, and for nothing)
        read(s + 1, 0, 0, half0);
        multiply(half1, 1, second_half);
    }
    if (g.W & 1) {
        turn_scales(0);
        read(g.W / 2, 0, 1, half1);
        multiply(half0, 0, first_half);
        multiply(half1, 0, second_half);
    }

    // the wave's tile leaves 32 rows at a time through LDS, so that stores run along the rows
    __syncthreads();
    float* mine = reinterpret_cast<float*>(s_mem) + wave * 32 * T::PITCH;
    constexpr uint32_t COLS = 32 * T::TJ, LANES = COLS / 8;
#pragma unroll
    for (uint32_t i = 0; i < T::TI; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < T::TJ; ++j)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) mine[(8 * (e / 4) + 4 * kb + e % 4) * T::PITCH + 32 * j + r32] = acc[i][j][e];
        wave_sync_lds();
#pragma unroll
        for (uint32_t p = 0; p < 32 * LANES / 64; ++p) {
            const uint32_t r = p * (64 / LANES) + lane / LANES, c = 8 * (lane % LANES);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(mine + r * T::PITCH + c), hi = *reinterpret_cast<const f32x4*>(mine + r * T::PITCH + c + 4);
            const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const uint64_t m = m0 + wm * (BM / WM) + 32 * i + r, n = n0 + wn * COLS + c;
            if (m < g.M) store8_first<TYPE>(g.out, m * g.ld + n, (int64_t)g.N - (int64_t)n, v);
        }
        wave_sync_lds();
    }
}

}  // namespace kimad
