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
__device__ __forceinline__ float exponent_value(uint32_t byte) { // 2^(byte - 127)
    return __builtin_bit_cast(float, byte == 0u ? 0x00400000u : byte << 23);
}
__device__ __forceinline__ float exponent_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// E (4 or a multiple of 4) codes -> their values times scale
template <int E> __device__ __forceinline__ void e4m3_values(const uint32_t *codes, float scale, float (&v)[E]) {
    typedef float float2v __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int w = 0; w < E / 4; ++w) {
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w], true);
        v[4 * w] = lo[0] * scale;
        v[4 * w + 1] = lo[1] * scale;
        v[4 * w + 2] = hi[0] * scale;
        v[4 * w + 3] = hi[1] * scale;
    }
}

} // namespace ubp
