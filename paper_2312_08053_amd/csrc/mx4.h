// Microscaled 4-bit floats: an element is an E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign), 32 neighbours share a
// scale 2^(byte - 127).  Four such blocks are a word: 64 bytes of codes, two to a byte with the first one low, and one
// 32-bit word of scale bytes, the first block's lowest.  In these kernels sixteen lanes hold a word, eight elements each,
// so that a block is four neighbouring lanes.
#pragma once
#include "common.h"

namespace kimad {

constexpr uint32_t MX4_WORD = 128;           // elements of a word
enum : uint32_t { TYPE_F32 = 0, TYPE_F16 = 1, TYPE_BF16 = 2 };   // KIMAD_VALUES_* of the public header

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Rows may begin anywhere: vectors that are aligned like their elements only (the hardware takes such addresses).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float half_to_float(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
// Two values rounded to nearest even, the first one low; a NaN stays one.
template <uint32_t TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 v = {a, b};
    if (TYPE == TYPE_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// One element of a typed array, and eight that stand side by side.
template <uint32_t TYPE>
__device__ __forceinline__ float load1(const void* p, uint64_t i) {
    if (TYPE == TYPE_F32) return static_cast<const float*>(p)[i];
    const uint32_t b = static_cast<const uint16_t*>(p)[i];
    return TYPE == TYPE_F16 ? half_to_float(b) : __uint_as_float(b << 16);
}
template <uint32_t TYPE>
__device__ __forceinline__ void store1(void* p, uint64_t i, float v) {
    if (TYPE == TYPE_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = (uint16_t)pack2<TYPE>(v, v);
}

// Eight elements as they lie in memory (four or eight registers), loaded now and turned into floats later.
template <uint32_t TYPE>
struct Raw8 {
    uint32_t r[TYPE == TYPE_F32 ? 8 : 4];
    __device__ __forceinline__ float at(uint32_t i) const {
        if (TYPE == TYPE_F32) return __uint_as_float(r[i]);
        const uint32_t b = r[i / 2];
        if (TYPE == TYPE_BF16) return __uint_as_float(i % 2 ? b & 0xFFFF0000u : b << 16);
        return half_to_float(i % 2 ? b >> 16 : b & 0xFFFFu);
    }
    __device__ __forceinline__ void set(uint32_t i, uint32_t bits) {
        if (TYPE == TYPE_F32) r[i] = bits;
        else r[i / 2] = i % 2 ? (r[i / 2] & 0xFFFFu) | bits << 16 : (r[i / 2] & 0xFFFF0000u) | bits;
    }
};
template <uint32_t TYPE>
__device__ __forceinline__ Raw8<TYPE> load8(const void* p, uint64_t i) {
    Raw8<TYPE> v;
    if (TYPE == TYPE_F32) {
        const f32x4_any* q = reinterpret_cast<const f32x4_any*>(static_cast<const float*>(p) + i);
        const f32x4 a = q[0], b = q[1];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) { v.r[k] = __float_as_uint(a[k]); v.r[(k + 4) % (TYPE == TYPE_F32 ? 8 : 4)] = __float_as_uint(b[k]); }
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) v.r[k] = a[k];
    }
    return v;
}
// The first `n` of eight elements (n may be below 0 or more than 8); the others become zeros.
template <uint32_t TYPE>
__device__ __forceinline__ Raw8<TYPE> load8_first(const void* p, uint64_t i, int64_t n) {
    if (n >= 8) return load8<TYPE>(p, i);
    Raw8<TYPE> v;
#pragma unroll
    for (uint32_t k = 0; k < sizeof(v.r) / 4; ++k) v.r[k] = 0;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        uint32_t b = 0;
        if ((int64_t)k < n) b = TYPE == TYPE_F32 ? static_cast<const uint32_t*>(p)[i + k] : (uint32_t)static_cast<const uint16_t*>(p)[i + k];
        v.set(k, b);
    }
    return v;
}
template <uint32_t TYPE>
__device__ __forceinline__ void store8(void* p, uint64_t i, const float v[8]) {
    if (TYPE == TYPE_F32) {
        f32x4_any* q = reinterpret_cast<f32x4_any*>(static_cast<float*>(p) + i);
        q[0] = f32x4{v[0], v[1], v[2], v[3]};
        q[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        u32x4 a;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) a[k] = pack2<TYPE>(v[2 * k], v[2 * k + 1]);
        *reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(p) + i) = a;
    }
}
template <uint32_t TYPE>
__device__ __forceinline__ void store8_first(void* p, uint64_t i, int64_t n, const float v[8]) {
    if (n >= 8) { store8<TYPE>(p, i, v); return; }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
        if ((int64_t)k < n) store1<TYPE>(p, i + k, v[k]);
}

// Lane exchanges inside four and sixteen neighbouring lanes, as operands of vector instructions (no LDS).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_ROR4 = 0x124, DPP_ROR8 = 0x128, DPP_HALF_MIRROR = 0x141;

// The scale byte of a block whose largest magnitude has these bits: two below the exponent, so that the largest element lies in
// [4, 8) and rounds to 4 or 6.  The smallest scale is 2^-127; a block with Inf or NaN gets 255 and stands for NaN as a whole.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? 255u : (e < 2u ? 2u : e) - 2u;
}
// 2^(byte - 127) as a float; 255 gives +Inf, which the conversions below take for NaN.
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// A lane's eight elements of a block that it shares with its three neighbours: codes and scale byte.  The conversion divides by the
// scale (exactly, it is a power of two) and rounds to nearest even, values beyond 6 to 6.
__device__ __forceinline__ uint32_t mx4_encode8(const float v[8], uint32_t& byte) {
    uint32_t a = 0;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) { const uint32_t b = key_of(v[k]); a = a > b ? a : b; }
    uint32_t o = dpp_u32<DPP_XOR1>(a);
    a = a > o ? a : o;
    o = dpp_u32<DPP_XOR2>(a);
    a = a > o ? a : o;
    byte = mx4_scale_byte(a);
    const float s = mx4_scale(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return byte == 255u ? 0u : c;
}
// The same with four elements a lane, of a block that eight neighbours share: 16 bits of codes.
__device__ __forceinline__ uint32_t mx4_encode4(const float v[4], uint32_t& byte) {
    uint32_t a = 0;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) { const uint32_t b = key_of(v[k]); a = a > b ? a : b; }
    uint32_t o = dpp_u32<DPP_XOR1>(a);
    a = a > o ? a : o;
    o = dpp_u32<DPP_XOR2>(a);
    a = a > o ? a : o;
    o = dpp_u32<DPP_HALF_MIRROR>(a);
    a = a > o ? a : o;
    byte = mx4_scale_byte(a);
    const float s = mx4_scale(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    return byte == 255u ? 0u : c;
}
__device__ __forceinline__ void mx4_decode4(uint32_t codes, uint32_t byte, float v[4]) {
    const float s = mx4_scale(byte);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
// What eight codes stand for.
__device__ __forceinline__ void mx4_decode8(uint32_t codes, uint32_t byte, float v[8]) {
    const float s = mx4_scale(byte);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}
// The word of scale bytes from the bytes of a word's sixteen lanes (the same in the four lanes of a block), in all of them.
__device__ __forceinline__ uint32_t mx4_scale_word(uint32_t byte, uint32_t lane16) {
    uint32_t w = byte << (8u * (lane16 >> 2));
    w |= dpp_u32<DPP_ROR4>(w);
    return w | dpp_u32<DPP_ROR8>(w);
}

}  // namespace kimad
