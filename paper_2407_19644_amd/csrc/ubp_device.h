// Device-side helpers shared by the HIP kernels of the UBP library (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "ubp_internal.h"

namespace ubp {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; } // round to nearest even

template <typename T, int VEC> struct VecOf { typedef T type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct VecOf<T, 1> { typedef T type; };

template <typename T, int VEC>
__device__ __forceinline__ void load_row(const T *p, float (&out)[VEC]) {
    if constexpr (VEC == 1) {
        out[0] = to_f32(*p);
    } else {
        typedef typename VecOf<T, VEC>::type V;
        V v = *reinterpret_cast<const V *>(p);
#pragma unroll
        for (int t = 0; t < VEC; ++t) out[t] = to_f32((T)v[t]);
    }
}

template <typename T, int VEC>
__device__ __forceinline__ void store_row(T *p, const float (&in)[VEC]) {
    if constexpr (VEC == 1) {
        *p = from_f32<T>(in[0]);
    } else {
        typedef typename VecOf<T, VEC>::type V;
        V v;
#pragma unroll
        for (int t = 0; t < VEC; ++t) v[t] = from_f32<T>(in[t]);
        *reinterpret_cast<V *>(p) = v;
    }
}

// Epilogue on an accumulator tile of the MFMA kernels: lane 16 g + n holds 4 pixels of row
// (first row of the stripe) + n.  A uniform test keeps the plain product free of it.
__device__ __forceinline__ float epilogue_value(const Epilogue &e, float v, float b) {
    return fminf(fmaxf(v + b, e.lo), e.hi);
}
__device__ __forceinline__ float epilogue_bias(const Epilogue &e, int row, int M) {
    return (e.bias != nullptr && row < M) ? e.bias[row] : 0.f;
}
__device__ __forceinline__ void epilogue_tile(const Epilogue &e, float4v &acc, float b) {
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[v] = epilogue_value(e, acc[v], b);
}

// ---- activations beyond a clamp.  Both are v times a distribution function of v, so that one quotient or one polynomial
// gives the function and, in the backward pass, its slope.
// sigma(u) by the hardware's exp2 and reciprocal (1 ulp each); u so large that exp2 overflows gives 0.
__device__ __forceinline__ float sigmoid(float u) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * -1.44269504089f));
}
// Phi(v) = 1/2 erfc(-v / sqrt 2).  The tail Q(z) = 1 - Phi(z), z >= 0, is exp(-z^2 / 2) times a smooth function, here a
// polynomial in t = 1 / (1 + 0.3 z): fitted for a small largest relative error on 0 <= z <= 14.5, where Q leaves fp32; with the
// constants in fp32 it is 1e-7.  In fp32, with an exp2 and a reciprocal rounded to nearest, Phi is within 2.1e-7 of the truth, and
// its tail within 1.5e-6 of itself up to z = 5 and 5.3e-6 up to z = 10 (the rounding of z^2).
// density: exp(-v^2 / 2), which the slope needs too.
__device__ __forceinline__ float normal_cdf(float v, float &density) {
    const float z = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.3f, z, 1.f));
    density = __builtin_amdgcn_exp2f(z * z * -0.72134752044f);
    float q = 0.03831019252538681f;
    q = fmaf(q, t, -0.168900728225708f);
    q = fmaf(q, t, 0.22824111580848694f);
    q = fmaf(q, t, -0.07616594433784485f);
    q = fmaf(q, t, 0.14238862693309784f);
    q = fmaf(q, t, 0.09471195936203003f);
    q = fmaf(q, t, 0.12192083895206451f);
    q = fmaf(q, t, 0.11948668211698532f);
    q = fmaf(q, t, 7.272966286109295e-06f) * density;
    return v > 0.f ? 1.f - q : q;
}
// The argument of the odd polynomial c1 v + c3 v^3, kept where its powers are finite: sigma is 0 or 1 long before.
__device__ __forceinline__ float cubic(float v, float c1, float c3) {
    const float w = fminf(fmaxf(v, -1e9f), 1e9f);
    return w * fmaf(c3 * w, w, c1);
}

// The kernels' sources are compiled twice: as they are, and with UBP_WIDE for the epilogue with on == 2, whose activations
// and residual take registers that the plain kernels have better use for (in one kernel behind a branch, the block kernel
// spilled 120 registers and 50 others lost a wavefront per SIMD).  The launchers of the second kind have names of their own.
#ifdef UBP_WIDE
constexpr bool kWide = true;
#define UBP_LAUNCHER(name) name##_wide
#else
constexpr bool kWide = false;
#define UBP_LAUNCHER(name) name
#endif

// Epilogue with on == 2, without the residual.
__device__ __forceinline__ void epilogue_act(const Epilogue &e, float *v, int n, float b) {
    if (e.act == kActSigmoid && e.c3 == 0.f) {
        // (SiLU: no powers that could overflow.  5 instructions fewer: kernel 6 on 4096 x 4096 with 8192 pixels took 103 us, not 109)
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float x = v[i] + b;
            v[i] = x * sigmoid(x * e.c1);
        }
    } else if (e.act == kActSigmoid) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float x = v[i] + b;
            v[i] = x * sigmoid(cubic(x, e.c1, e.c3));
        }
    } else if (e.act == kActNormal) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float x = v[i] + b;
            float d;
            v[i] = x * normal_cdf(x, d);
        }
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = epilogue_value(e, v[i], b);
    }
}
// n neighbouring values of the residual (pixels px .. of a row; nothing outside the M x N matrix is read; zeros without one).
template <typename TY, int VEC> struct Residual {
    typedef typename std::conditional<sizeof(TY) == 4, uint32_t, uint16_t>::type Bits;
    static constexpr int kWords = (VEC * (int)sizeof(TY) + 3) / 4;
    uint32_t r[kWords]; // (packed: the wavefronts that hold these have few registers left)
    __device__ __forceinline__ void load(const Epilogue &e, int row, int px, int M, int N) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) r[w] = 0u;
        if (e.res == nullptr || row >= M) return;
        const Bits *src = static_cast<const Bits *>(e.res) + (int64_t)row * e.ldr + px;
        if (VEC > 1 && e.res_vec && px + VEC <= N) {
            typedef typename VecOf<Bits, VEC>::type V;
            const V x = *reinterpret_cast<const V *>(src);
            __builtin_memcpy(r, &x, sizeof x);
        } else {
#pragma unroll
            for (int v = 0; v < VEC; ++v)
                if (px + v < N) {
                    if constexpr (sizeof(TY) == 4) r[v] = src[v];
                    else r[v / 2] |= (uint32_t)src[v] << (16 * (v & 1));
                }
        }
    }
    __device__ __forceinline__ float value(int v) const {
        if constexpr (sizeof(TY) == 4) return __builtin_bit_cast(float, r[v]);
        else return to_f32(__builtin_bit_cast(TY, (uint16_t)(r[v / 2] >> (16 * (v & 1)))));
    }
    // act(v + b) + residual
    __device__ __forceinline__ void apply(const Epilogue &e, float (&v)[VEC], float b) const {
        epilogue_act(e, v, VEC, b);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] += value(i);
    }
    __device__ __forceinline__ void apply(const Epilogue &e, float4v &acc, float b) const {
        float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        apply(e, v, b);
        acc = float4v{v[0], v[1], v[2], v[3]};
    }
};

template <bool BF16>
__device__ __forceinline__ float4v mfma16(short8v a, short8v b, float4v c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// transposed 8-byte read at an absolute LDS byte address
__device__ __forceinline__ short4v lds_read_tr(uint32_t lds_addr) {
    typedef __attribute__((address_space(3))) short4v *lds_ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)lds_addr);
}

// the same, a constant number of bytes further on
__device__ __forceinline__ short4v lds_read_tr(uint32_t lds_addr, int offset) {
    typedef __attribute__((address_space(3))) short4v *lds_ptr;
    typedef __attribute__((address_space(3))) char *lds_char_ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)((lds_char_ptr)(uintptr_t)lds_addr + offset));
}

// 16 bytes per lane from global memory straight into LDS at lds_base + 16 * lane (lds_base
// wave-uniform).  Written as inline assembly on purpose: the compiler then does not treat
// the load as a pending LDS write, which would make it wait for ALL outstanding vector
// memory operations before every LDS read.  Ordering against the LDS reads of the staged
// data is done by hand (wait_vmcnt, then the producer's counter of resident chunks).
__device__ __forceinline__ void load16_to_lds(const void *gbase, uint32_t lane_off, uint32_t lds_base) {
    // address = gbase (wave-uniform, in SGPRs) + lane_off (32-bit per-lane byte offset)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_off), "s"(gbase), "s"(lds_base));
}

__device__ __forceinline__ uint32_t lds_address(const char *p) {
    typedef __attribute__((address_space(3))) const char *lds_ptr;
    return (uint32_t)(uintptr_t)(lds_ptr)p;
}

template <int N> __device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt immediate out of range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// waits until at most n vector memory operations of this wavefront are outstanding (n is
// wave-uniform; it is rounded down to the nearest available immediate, which only waits longer)
__device__ __forceinline__ void wait_vmcnt_at_most(int n) {
    if (n >= 48) wait_vmcnt<48>();
    else if (n >= 32) wait_vmcnt<32>();
    else if (n >= 24) wait_vmcnt<24>();
    else if (n >= 16) wait_vmcnt<16>();
    else if (n >= 12) wait_vmcnt<12>();
    else if (n >= 8) wait_vmcnt<8>();
    else if (n >= 6) wait_vmcnt<6>();
    else if (n >= 4) wait_vmcnt<4>();
    else if (n >= 3) wait_vmcnt<3>();
    else if (n >= 2) wait_vmcnt<2>();
    else if (n >= 1) wait_vmcnt<1>();
    else wait_vmcnt<0>();
}

__device__ __forceinline__ uint32_t flag_load(uint32_t *p) {
    return __hip_atomic_load(p, __ATOMIC_ACQUIRE, __HIP_MEMORY_SCOPE_WORKGROUP);
}

constexpr int kSpinLimit = 1 << 22; // polls before a wait gives up (each poll is >= 100 cycles)

// s_barrier with only the LDS counter drained: __syncthreads() would also wait for every
// outstanding vector memory operation, i.e. for loads that are meant to stay in flight
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Raises a kernel's dynamic LDS limit to all of a CU's LDS, once per device ordinal (the limit
// belongs to the function on a device).  One instance per kernel instantiation.  at_zero: the kernel counts on its dynamic
// LDS beginning at LDS address 0, which it does as long as there is no static LDS; otherwise the kernel is refused.
struct LdsLimit {
    std::atomic<uint64_t> done{0};
    ubp_status raise(const void *fn, bool at_zero = false) {
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) {
            (void)hipGetLastError();
            return UBP_ERR_DEVICE;
        }
        const uint64_t bit = (dev >= 0 && dev < 64) ? (uint64_t(1) << dev) : 0;
        if (bit && (done.load(std::memory_order_acquire) & bit)) return UBP_OK;
        if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) {
            (void)hipGetLastError();
            return UBP_ERR_DEVICE;
        }
        hipFuncAttributes f;
        if (at_zero && (hipFuncGetAttributes(&f, fn) != hipSuccess || f.sharedSizeBytes != 0)) {
            (void)hipGetLastError();
            return UBP_ERR_DEVICE;
        }
        done.fetch_or(bit, std::memory_order_release);
        return UBP_OK;
    }
};

// One launch.  By hipLaunchKernel and not by <<< >>>, whose way through the runtime's stack of launch configurations is
// two more calls into it: small calls are bound by the host.
template <class T> struct SameType { using type = T; };
template <class... P>
ubp_status launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, typename SameType<P>::type... a) {
    void *args[] = {static_cast<void *>(&a)...};
    (void)hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, args, lds, st);
    return hipGetLastError() == hipSuccess ? UBP_OK : UBP_ERR_DEVICE;
}

} // namespace ubp
