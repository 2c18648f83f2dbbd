// Element types of the paged caches on the device: 16-bit values, the 4-bit codes that stand for them, and the matrix
// instructions that take them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_pages.h"

namespace tent {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Loads and stores of device memory: without the address space the compiler may take them for LDS or scratch.
template <class V>
__device__ __forceinline__ V dev_load(const void* p) { return *(const __attribute__((address_space(1))) V*)(uintptr_t)p; }
template <class V>
__device__ __forceinline__ void dev_store(void* p, V v) { *(__attribute__((address_space(1))) V*)(uintptr_t)p = v; }
// Rows that are written once and not read again by the call: past the caches' order of use.
template <class V>
__device__ __forceinline__ void dev_stream(void* p, V v) { __builtin_nontemporal_store(v, (__attribute__((address_space(1))) V*)(uintptr_t)p); }

// A launch takes fewer than 2^32 lanes, so more than this many workgroups of up to 256 go in several launches, each told its first.
// A multiple of eight: workgroups keep their XCDs.
constexpr uint32_t kMostBlocks = 1u << 23;
template <class Launch>
int launch_blocks(uint64_t blocks, Launch launch, uint32_t most = kMostBlocks)
{
    if (blocks > 0x7FFFFFFFull) return TENT_ERR_RANGE;
    for (uint64_t first = 0; first < blocks; first += most) {
        launch((uint32_t)first, (uint32_t)(blocks - first < most ? blocks - first : most));
        if (hipGetLastError() != hipSuccess) return TENT_ERR_HIP;
    }
    return TENT_OK;
}

__device__ __forceinline__ void kv_note(int32_t* errors, int32_t what)
{
    if (errors) atomicOr(errors, what);
}

// The power of two that a scale byte stands for, as the conversion instructions take it: only the exponent field counts,
// 0 is 2^-127 and 255 makes every value NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

struct Bf16 {
    using Pair = bf16x2;
    using Oct = bf16x8;
    static constexpr int kLow = -127, kHigh = 125;                      // powers of two a block may have
    static constexpr uint32_t kInf = 0x7F80u;                           // magnitudes from here on are infinite or NaN
    // Softmax weights are held times 2^this, so that those which decide a result near the type's least values (2^-133) are not
    // below what 32 bits and the matrix instructions hold as normal numbers.
    static constexpr float kWeightShift = 16.f;
    static constexpr bool kLarge = true;                                 // sums of weights times values may pass 32 bits (see kv_attend.h)
    static __device__ __forceinline__ float to_float(uint32_t half) { return __uint_as_float(half << 16); }
    static __device__ __forceinline__ uint32_t pack2(float a, float b)
    {
        const bf16x2 v = {(__bf16)a, (__bf16)b};                        // to nearest, ties to even
        return __builtin_bit_cast(uint32_t, v);
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t encode2(uint32_t old, uint32_t pair, float scale)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, pair), scale, kByte);
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Oct, a), __builtin_bit_cast(Oct, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Oct, a), __builtin_bit_cast(Oct, b), c, 0, 0, 0);
    }
};

struct Fp16 {
    using Pair = f16x2;
    using Oct = f16x8;
    static constexpr int kLow = -23, kHigh = 13;
    static constexpr uint32_t kInf = 0x7C00u;
    // A weight is at most 1 (2^8 while the maximum lags, see kv_attend.h): times 2^7 it stays below 65504, and weights
    // down to 2^-21 keep all 11 bits.
    static constexpr float kWeightShift = 7.f;
    static constexpr bool kLarge = false;                                // 2^30 times 2^15 times 65504 is far below
    static __device__ __forceinline__ float to_float(uint32_t half)
    {
        return (float)__builtin_bit_cast(_Float16, (unsigned short)half);
    }
    static __device__ __forceinline__ uint32_t pack2(float a, float b)
    {
        const f16x2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kByte));
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t encode2(uint32_t old, uint32_t pair, float scale)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, pair), scale, kByte);
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Oct, a), __builtin_bit_cast(Oct, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Oct, a), __builtin_bit_cast(Oct, b), c, 0, 0, 0);
    }
};

// Eight codes as eight 16-bit values.
template <class E>
__device__ __forceinline__ u32x4 decode8(uint32_t codes, float scale)
{
    return u32x4{E::template decode2<0>(codes, scale), E::template decode2<1>(codes, scale), E::template decode2<2>(codes, scale),
                 E::template decode2<3>(codes, scale)};
}

// The scale byte of a block of 32 whose largest magnitude is `top` (16-bit pattern without the sign): the least power of two
// that 7 times reaches it.  The bits above the mantissa give floor(log2); 1.75 is where 4 times the power stops being enough.
template <class E>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    if (top >= E::kInf) return 255u;
    const uint32_t bits = __float_as_uint(E::to_float(top));             // a 16-bit value below 2^-126 is far below the least power
    int power = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    power = power < E::kLow ? E::kLow : power > E::kHigh ? E::kHigh : power;
    return (uint32_t)(power + 127);
}

// Packs eight 16-bit values of this lane, one quarter of a block that four lanes in a row hold: the codes of the eight, and
// the block's scale byte (the same in the four lanes).
template <class E>
__device__ __forceinline__ uint32_t encode8(u32x4 v, uint32_t& byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = v[i] & 0x7FFFu, hi = (v[i] >> 16) & 0x7FFFu;
        top = lo > top ? lo : top;
        top = hi > top ? hi : top;
    }
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true);   // lane ^ 1
    top = o > top ? o : top;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true);            // lane ^ 2
    top = o > top ? o : top;
    byte = scale_byte<E>(top);
    const float scale = scale_of(byte);
    uint32_t codes = E::template encode2<0>(0u, v[0], scale);
    codes = E::template encode2<1>(codes, v[1], scale);
    codes = E::template encode2<2>(codes, v[2], scale);
    codes = E::template encode2<3>(codes, v[3], scale);
    return byte == 255u ? 0u : codes;
}

}  // namespace tent
