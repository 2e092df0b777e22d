// Activations in 8 bits: e4m3 (4 bits of exponent, 3 of fraction, largest 448, no infinity) with one power of two per 32
// neighbouring values of a row, kept as its exponent plus 127 in a byte.
#pragma once

#include "ubp_device.h"

namespace ubp {

constexpr int kGroup = 32;

// The byte for a group whose largest finite magnitude has the bits `top` (fp32): the smallest exponent s >= -127 with
// top <= 448 2^s = 1.75 2^(s + 8).
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top) {
    const int b = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(b, 0);
}
__device__ __forceinline__ float exponent_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// E (4 or a multiple of 4) codes -> their values times a power of two, in T, to nearest.  The conversion takes the power from
// the exponent bits of `scale` alone, the exponent byte itself, 0 for 2^-127 included.  (For every code and every byte but
// 255 its results are those of a product in fp32 and a rounding to T.)
template <typename T, int E> __device__ __forceinline__ void e4m3_to(const uint32_t *codes, float scale, T *out) {
#pragma unroll
    for (int w = 0; w < E / 4; ++w) {
        if constexpr (__is_same(T, __bf16)) {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], scale, false);
            const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], scale, true);
            __builtin_memcpy(out + 4 * w, &lo, 4);
            __builtin_memcpy(out + 4 * w + 2, &hi, 4);
        } else if constexpr (__is_same(T, _Float16)) {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[w], scale, false);
            const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[w], scale, true);
            __builtin_memcpy(out + 4 * w, &lo, 4);
            __builtin_memcpy(out + 4 * w + 2, &hi, 4);
        } else {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[w], scale, false);
            const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[w], scale, true);
            __builtin_memcpy(out + 4 * w, &lo, 8);
            __builtin_memcpy(out + 4 * w + 2, &hi, 8);
        }
    }
}

} // namespace ubp
