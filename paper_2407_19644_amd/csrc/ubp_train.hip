// Backward pass of a layer's epilogue, and its inputs kept in 8 bits: kernels that pass over their data once.
#include "ubp_device.h"
#include "ubp_fp8.h"

#include <cstdint>

namespace ubp {

namespace {

// ------------------------------------------------------------------ gradient of the epilogue
// act'(z).  With F the distribution function of the forward pass: F + z F'.
__device__ __forceinline__ float slope(const ActGradArgs &a, float z) {
    // (beyond 1e4 both slopes are 0 or 1 in fp32, and nothing below overflows)
    const float w = fminf(fmaxf(z, -1e4f), 1e4f);
    float r;
    if (a.act == kActSigmoid) {
        // (1 - s as e s where s is next to 1: the difference would lose what the tail is worth)
        const float e = __builtin_amdgcn_exp2f(cubic(w, a.c1, a.c3) * -1.44269504089f);
        const float s = __builtin_amdgcn_rcpf(1.f + e);
        r = fmaf(w * fmaf(3.f * a.c3 * w, w, a.c1), (e > 1.f ? 1.f - s : e * s) * s, s);
    } else if (a.act == kActNormal) {
        float d;
        const float p = normal_cdf(w, d);
        r = fmaf(w * 0.39894228040f, d, p);
    } else {
        return a.pass == kPassAll || (z <= a.hi && (a.pass == kPassAbove ? z > a.lo : z >= a.lo)) ? 1.f : 0.f;
    }
    return z == z ? r : z;
}

// A sum of any length, to about 2^-24 of the sum of magnitudes: what an addition drops is kept beside it (one addition after the
// other would be off by up to n 2^-25 of itself where terms are of one size; a row may have millions).
struct LongSum {
    float sum = 0.f, low = 0.f;
    __device__ __forceinline__ void add(float v) {
        const float s = sum + v, t = s - sum;
        low += (sum - (s - t)) + (v - t);
        sum = s;
    }
    // (beside an Inf or NaN stands nothing that counts)
    __device__ __forceinline__ float value() const {
        const float s = sum + low;
        return fabsf(s) < INFINITY ? s : sum;
    }
};

// A lane takes 16 bytes of neighbouring tokens of a row at once, a wavefront a part of 1 KB: G = dY act'(Z), and the sum of
// G's fp32 values, before they are rounded.  Four wavefronts of a workgroup take a row each, or, where rows are longer than a
// part, every fourth part of one row (of kActGroup tokens of it, where rows are few), whose sums meet in LDS in order.  A lane's
// sums of its 16 bytes are added up by LongSum, however many they are.
// What bounds it: memory.  4096 rows of 8192 bf16 tokens, SiLU: 43 us, 4.70 TB/s (a large copy: 4.92).  One load of each matrix
// in flight per lane leaves room for 8 wavefronts per SIMD; four, with 5 wavefronts, took 54 us.  960 rows of 1568 fp16 tokens:
// 7.4 us, the launch.
template <typename T>
__global__ __launch_bounds__(256) void act_grad_kernel(ActGradArgs a) {
    constexpr int E = 16 / (int)sizeof(T), PART = 64 * E;
    static_assert(kActGroup % (4 * PART) == 0, "a group is whole rounds of parts");
    __shared__ float sums[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const bool shared = a.N > PART;
    const int64_t unit = (int64_t)blockIdx.x;
    const int64_t row = shared ? unit / a.row_groups : 4 * unit + wave;
    const int group = shared ? (int)(unit % a.row_groups) : 0;
    if (row >= a.M) return;                     // (whole workgroups where rows are shared)
    const T *dy = static_cast<const T *>(a.dY) + row * a.lddy, *z = static_cast<const T *>(a.Z) + row * a.ldz;
    T *gout = static_cast<T *>(a.G) + row * a.ldg;
    LongSum total;
    const int first = group * kActGroup, last = a.row_groups > 1 ? min(first + kActGroup, a.N) : a.N;
    for (int n0 = first + (shared ? wave * PART : 0); n0 < last; n0 += 4 * PART) {
        const int col = n0 + lane * E;
        T y[E], zz[E], o[E];
        if (col + E <= a.N) {
            __builtin_memcpy(y, dy + col, 16);
            if (a.pass != kPassAll) __builtin_memcpy(zz, z + col, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                y[e] = zz[e] = (T)0.f;
                if (col + e < a.N) {
                    y[e] = dy[col + e];
                    if (a.pass != kPassAll) zz[e] = z[col + e];
                }
            }
        }
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            // (a slope of 0 of ReLU and clamp stops what comes, whatever it is)
            const float s = slope(a, to_f32(zz[e])), d = to_f32(y[e]);
            const float v = a.act == kActClamp ? (s != 0.f ? d : 0.f) : d * s;
            part += v;
            o[e] = from_f32<T>(v);
        }
        total.add(part);
        if (col + E <= a.N) {
            __builtin_memcpy(gout + col, o, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col + e < a.N) gout[col + e] = o[e];
        }
    }
    if (a.dbias == nullptr) return;
    float sum = total.value();
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (!shared) {
        if (lane == 0) a.dbias[row] = sum;
        return;
    }
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        if (a.row_groups == 1) a.dbias[row] = s;
        else a.part[row * a.row_groups + group] = s;
    }
}

// The sums of a row's parts, in order.
__global__ __launch_bounds__(256) void row_sum_kernel(ActGradArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.M) return;
    LongSum total;
    for (int p = 0; p < a.row_groups; ++p) total.add(a.part[row * a.row_groups + p]);
    a.dbias[row] = total.value();
}

template <typename T> ubp_status act_grad(ActGradArgs a, hipStream_t st) {
    const bool shared = a.N > 64 * 16 / (int)sizeof(T);
    const int64_t grid = shared ? (int64_t)a.M * a.row_groups : ((int64_t)a.M + 3) / 4;
    if (grid * 256 >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED; // (a launch's threads are counted in 32 bits)
    const ubp_status rc = launch_kernel(&act_grad_kernel<T>, dim3((unsigned)grid), dim3(256), 0, st, a);
    if (rc != UBP_OK || a.dbias == nullptr || a.row_groups == 1) return rc;
    return launch_kernel(&row_sum_kernel, dim3((unsigned)((a.M + 255) / 256)), dim3(256), 0, st, a);
}

// ------------------------------------------------------------------ inputs in 8 bits
// A lane takes 16 neighbouring values, half a group; a wavefront 1024.  What bounds both ways: memory.  4096 rows of 8192 bf16
// values: 42 us there and back, 4.83 TB/s; 2304 rows of 12543, at any alignment: 40 us, 4.35 TB/s.
constexpr int kLaneValues = 16;
constexpr int kWaveValues = 64 * kLaneValues;

template <typename T> __device__ __forceinline__ void load16(const T *src, int valid, T (&x)[kLaneValues]) {
    if (valid >= kLaneValues) {
        __builtin_memcpy(x, src, sizeof x);
    } else {
#pragma unroll
        for (int e = 0; e < kLaneValues; ++e) {
            x[e] = (T)0.f;
            if (e < valid) x[e] = src[e];
        }
    }
}

// x / 2^s to the nearest e4m3, s the group's exponent; what is not finite becomes NaN.  Where s is as large as the type
// allows, 2^(s + 8) is beyond the type: values next to it go down to 240 2^s, which is no further than half a step.
template <typename T>
__global__ __launch_bounds__(256) void save_kernel(CheckpointArgs a) {
    constexpr uint32_t kTop = sizeof(T) == 2 && __is_same(T, _Float16) ? 135u : 247u;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = unit / a.units;
    const int col = (int)(unit % a.units) * kWaveValues + lane * kLaneValues;
    if (row >= a.K) return;
    T x[kLaneValues];
    load16(static_cast<const T *>(a.X) + row * a.ldx + col, a.N - col, x);
    uint32_t top = 0u;
#pragma unroll
    for (int e = 0; e < kLaneValues; ++e) {
        const uint32_t u = __builtin_bit_cast(uint32_t, to_f32(x[e])) & 0x7fffffffu;
        top = max(top, u < 0x7f800000u ? u : 0u);
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    const uint32_t byte = exponent_byte(top);
    const float inverse = exponent_inverse(byte), limit = byte >= kTop ? 240.f : 448.f;
    uint32_t q[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float y[4];
        uint32_t bad = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = to_f32(x[4 * w + e]);
            y[e] = fminf(fmaxf(v * inverse, -limit), limit);
            if ((__builtin_bit_cast(uint32_t, v) & 0x7fffffffu) >= 0x7f800000u) bad |= 0x7fu << (8 * e);
        }
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
        q[w] = (uint32_t)c | bad;
    }
    uint8_t *dst = a.Q + row * a.ldq + col;
    if (col + kLaneValues <= a.N) {
        __builtin_memcpy(dst, q, 16);
    } else {
#pragma unroll
        for (int e = 0; e < kLaneValues; ++e)
            if (col + e < a.N) dst[e] = (uint8_t)(q[e / 4] >> (8 * (e & 3)));
    }
    if ((lane & 1) == 0 && col < a.N) a.S[row * a.lds + col / kGroup] = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(256) void load_kernel(CheckpointArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = unit / a.units;
    const int col = (int)(unit % a.units) * kWaveValues + lane * kLaneValues;
    if (row >= a.K || col >= a.N) return;
    const uint8_t *src = a.Q + row * a.ldq + col;
    uint32_t q[4] = {0u, 0u, 0u, 0u};
    if (col + kLaneValues <= a.N) {
        __builtin_memcpy(q, src, 16);
    } else {
#pragma unroll
        for (int e = 0; e < kLaneValues; ++e)
            if (col + e < a.N) q[e / 4] |= (uint32_t)src[e] << (8 * (e & 3));
    }
    T o[kLaneValues];
    e4m3_to<T, kLaneValues>(q, __builtin_bit_cast(float, (uint32_t)a.S[row * a.lds + col / kGroup] << 23), o);
    T *dst = static_cast<T *>(a.out) + row * a.ldx + col;
    if (col + kLaneValues <= a.N) {
        __builtin_memcpy(dst, o, sizeof o);
    } else {
#pragma unroll
        for (int e = 0; e < kLaneValues; ++e)
            if (col + e < a.N) dst[e] = o[e];
    }
}

ubp_status launch_rows(void (*kernel)(CheckpointArgs), CheckpointArgs a, hipStream_t st) {
    a.units = (a.N + kWaveValues - 1) / kWaveValues;
    const int64_t grid = ((int64_t)a.K * a.units + 3) / 4;
    if (grid * 256 >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED;
    return launch_kernel(kernel, dim3((unsigned)grid), dim3(256), 0, st, a);
}

} // namespace

ubp_status launch_act_grad(const ActGradArgs &a, ubp_dtype dtype, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == UBP_F32 ? act_grad<float>(a, st) : dtype == UBP_F16 ? act_grad<_Float16>(a, st) : act_grad<__bf16>(a, st);
}
ubp_status launch_save(const CheckpointArgs &a, ubp_dtype dtype, void *stream) {
    return launch_rows(dtype == UBP_F32 ? &save_kernel<float> : dtype == UBP_F16 ? &save_kernel<_Float16> : &save_kernel<__bf16>, a,
                       static_cast<hipStream_t>(stream));
}
ubp_status launch_load(const CheckpointArgs &a, ubp_dtype dtype, void *stream) {
    return launch_rows(dtype == UBP_F32 ? &load_kernel<float> : dtype == UBP_F16 ? &load_kernel<_Float16> : &load_kernel<__bf16>, a,
                       static_cast<hipStream_t>(stream));
}

} // namespace ubp
