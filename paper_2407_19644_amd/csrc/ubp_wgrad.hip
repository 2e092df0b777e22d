// Weight gradient of a pruned layer: dW[i][k] = sum over the tokens of G[i][n] X[k][n], for the kept weights alone.
#include "ubp_device.h"
#include "ubp_fp8.h"

#include <cstdint>

namespace ubp {

namespace {

constexpr int kRowBytes = 128; // of a row of G or X that a stage takes: 64 16-bit or 32 fp32 tokens, a cache line
constexpr int kThreads = 64 * kGradWaves;

// Place of 16-byte piece q of LDS row r: 16 neighbouring rows of one piece lie in all 16 units of 256 bytes, i.e. in all 64
// banks, for rows of 128, 64 (a checkpoint's 64 codes) and 32 bytes (32 codes).
template <int BYTES> __device__ __forceinline__ uint32_t place(uint32_t r, uint32_t q) {
    static_assert(BYTES == 128 || BYTES == 64 || BYTES == 32, "a row of a stage");
    constexpr int shift = BYTES == 128 ? 1 : BYTES == 64 ? 2 : 3;
    return r * BYTES + 16u * (q ^ ((r >> shift) & (BYTES / 16 - 1)));
}

template <typename T> __device__ __forceinline__ float4v product(uint4v a, uint4v b, float4v c);
template <> __device__ __forceinline__ float4v product<__bf16>(uint4v a, uint4v b, float4v c) {
    return mfma16<true>(__builtin_bit_cast(short8v, a), __builtin_bit_cast(short8v, b), c);
}
template <> __device__ __forceinline__ float4v product<_Float16>(uint4v a, uint4v b, float4v c) {
    return mfma16<false>(__builtin_bit_cast(short8v, a), __builtin_bit_cast(short8v, b), c);
}
// (lane group g holds tokens 4 g .. 4 g + 3 of both: product m takes the m-th of each group)
template <> __device__ __forceinline__ float4v product<float>(uint4v a, uint4v b, float4v c) {
    const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
#pragma unroll
    for (int m = 0; m < 4; ++m) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[m], y[m], c, 0, 0, 0);
    return c;
}

// A tile's sums: of one range of several, or, where there is only one, at their places.
__device__ __forceinline__ void store_tile(const GradArgs &a, float4v sum, int split, int64_t tile, int lane) {
    if (a.part) {
        *reinterpret_cast<float4v *>(a.part + ((int64_t)split * a.n_tiles + tile) * 256 + lane * 4) = sum;
        return;
    }
    const uint4v to = *reinterpret_cast<const uint4v *>(a.inv + tile * 256 + lane * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if ((int32_t)to[e] >= 0) a.out[to[e]] = a.accumulate ? a.out[to[e]] + sum[e] : sum[e];
}

// One workgroup = one region (at most 16 TILES tiles of 16 rows of G x 16 rows of X) and one range of tokens.  Both operands
// of the matrix instruction have the tokens along their inner dimension, as G and X have them in memory, so that a tile may
// pair any rows: nothing is transposed, and only tiles that keep weights are formed.
//  * A stage = 128 bytes (a cache line, where rows begin at one) of every row that the region needs, 64 of a checkpoint's,
//    through registers into LDS, which holds one stage: a row's register is loaded again as soon as it has been written
//    there, so that loads are in flight all the time.  Rows of any alignment and pitch.
//  * A tile reads 1 KB of each operand from LDS per half a stage, a tile ahead, and its sums stay in a wavefront's
//    registers for the whole range.
//  * CKPT: X is a checkpoint.  Its codes stay as they are in LDS, and a lane widens its 8 codes of a tile by 4 conversions that
//    take the exponent along: exact but for fp16 values below its normal range.  Exponents come 16 at a time.
//  * The last stage of a row may be short; it is staged token by token, zeros behind the last one.
//  * Ranges of tokens are summed by a second kernel, in order; with one range the sums go straight to their places.
template <typename T, bool CKPT, int TILES, int GS, int XS>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(GradArgs a) {
    constexpr int E = 16 / (int)sizeof(T);       // tokens of a 16-byte piece
    constexpr int STAGE = 8 * E;                 // tokens of a stage
    constexpr int XB = CKPT ? STAGE : kRowBytes; // bytes of a row of X
    constexpr int XL = XB / 16;                  // lanes that load it
    constexpr int GR = kThreads / 8, XR = kThreads / XL; // rows at once
    constexpr int PG = (GS + GR - 1) / GR, PX = (XS + XR - 1) / XR; // loads per lane
    static_assert(XS <= kThreads, "a lane per row for the exponents");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const uint32_t g = (uint32_t)(lane >> 4), n = (uint32_t)(lane & 15);
    // Workgroup ids go round-robin over the 8 XCDs: the pairs, regions of a range next to each other, are cut into 8 equal
    // runs, so that a range's rows come from memory to about one L2.
    const int64_t pairs = (int64_t)a.n_regions * a.splits;
    const int xcd = blockIdx.x & 7;
    const int64_t pair = (pairs * xcd >> 3) + (blockIdx.x >> 3);
    if (pair >= (pairs * (xcd + 1) >> 3)) return;
    const int split = (int)(pair / a.n_regions);
    const int32_t *reg = a.regions + 8 * (pair % a.n_regions);
    const int first = reg[0], tiles = reg[1], g_slots = reg[3], x_slots = reg[4] - reg[3];
    const int32_t *rows = a.rows + reg[2];
    const uint32_t x_area = (uint32_t)a.slots_g * kRowBytes, s_area = x_area + (uint32_t)a.slots_x * XB;

    const int all = (int)(((int64_t)a.N + STAGE - 1) / STAGE), full = a.N / STAGE;
    const int s0 = split * a.per_split, s1 = split == a.splits - 1 ? all : s0 + a.per_split, f1 = min(s1, full);

    // this lane's rows: pass i takes row list entries i GR + thread / 8 (of X: i XR + thread / XL), at a place a constant further on
    int64_t go[PG], xo[PX];
    const uint32_t gq = threadIdx.x % 8, xq = threadIdx.x % XL;
    const int gr = (int)threadIdx.x / 8, xr = (int)threadIdx.x / XL;
    const char *gbase = static_cast<const char *>(a.G) + (int64_t)s0 * kRowBytes, *xbase = static_cast<const char *>(a.X) + (int64_t)s0 * XB;
    const uint32_t gu = place<kRowBytes>((uint32_t)gr, gq), xu = x_area + place<XB>((uint32_t)xr, xq);
    static_assert(GR % 16 == 0 && XR % 16 == 0, "the rows of two passes differ by a multiple of 16: their places by a constant");
#pragma unroll
    for (int i = 0; i < PG; ++i)
        go[i] = (int64_t)rows[min(i * GR + gr, g_slots - 1)] * a.ldg * (int)sizeof(T) + 16 * gq;
#pragma unroll
    for (int i = 0; i < PX; ++i)
        xo[i] = (int64_t)rows[g_slots + min(i * XR + xr, x_slots - 1)] * a.ldx * (CKPT ? 1 : (int)sizeof(T)) + 16 * xq;
    // exponents: lane r has 16 neighbouring ones of row r, from group `window` on
    const int groups = (int)(((int64_t)a.N + 31) / 32);
    const uint8_t *sp = nullptr;
    int window = 0;
    uint4v exps = {0u, 0u, 0u, 0u};
    auto fetch_exps = [&](int group) {
        window = max(0, min(group, groups - 16));
        if (groups >= 16) {
            __builtin_memcpy(&exps, sp + window, 16);
        } else {
            exps = uint4v{0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < 15; ++k)
                if (k < groups) exps[k / 4] |= (uint32_t)sp[k] << (8 * (k & 3));
        }
    };
    auto put_exps = [&](int s) {
        // (the two groups of 64 tokens, or the one of 32)
        const int first_group = (int)((int64_t)s * STAGE / 32), k = first_group - window;
        const uint32_t lo = k < 8 ? (k < 4 ? exps[0] : exps[1]) : (k < 12 ? exps[2] : exps[3]);
        const uint32_t hi = k + 1 < 8 ? (k + 1 < 4 ? exps[0] : exps[1]) : (k + 1 < 12 ? exps[2] : exps[3]);
        const uint32_t b0 = (lo >> (8 * (k & 3))) & 0xffu, b1 = STAGE == 64 && first_group + 1 < groups ? (hi >> (8 * ((k + 1) & 3))) & 0xffu : b0;
        if ((int)threadIdx.x < x_slots) *reinterpret_cast<uint16_t *>(smem + s_area + 2 * threadIdx.x) = (uint16_t)(b0 | b1 << 8);
    };
    if constexpr (CKPT) {
        sp = a.S + (int64_t)rows[g_slots + min((int)threadIdx.x, x_slots - 1)] * a.lds;
        fetch_exps((int)((int64_t)s0 * STAGE / 32));
    }

    uint4v hg[PG], hx[PX];
    if (s0 < f1) {
#pragma unroll
        for (int i = 0; i < PG; ++i)
            if (i * GR < g_slots) __builtin_memcpy(&hg[i], gbase + go[i], 16);
#pragma unroll
        for (int i = 0; i < PX; ++i)
            if (i * XR < x_slots) __builtin_memcpy(&hx[i], xbase + xo[i], 16);
    }

    // ---- this wavefront's tiles
    const int per = (tiles + kGradWaves - 1) / kGradWaves;
    const int my0 = wave * per, mine = min(per, tiles - my0);
    uint32_t ops[TILES];                         // of this lane's piece: 16-byte unit in the rows of G | place in those of X << 16
    float4v acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const uint32_t o = t < mine ? a.ops[(int64_t)(first + my0 + t) * 16 + n] : (uint32_t)g_slots << 16;
        const uint32_t x = (o >> 16) - (uint32_t)g_slots;
        const uint32_t to = CKPT ? place<XB>(x, g * E / 16) + g * E % 16 : place<XB>(x, g) / 16;
        ops[t] = place<kRowBytes>(o & 0xffffu, g) / 16 | to << 16;
        acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    auto multiply = [&]() {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            struct Operands {
                uint4v x;
                uint32_t y[CKPT ? E / 4 : 4], e;
            };
            Operands o[2];
            auto load = [&](int t) {
                Operands &p = o[t & 1];
                asm volatile("" : "+v"(ops[t])); // (addresses are worked out here: kept for all tiles they are spilled)
                p.x = *reinterpret_cast<const uint4v *>(smem + (((ops[t] & 0xffffu) ^ (4u * u)) << 4));
                const uint32_t to = CKPT ? (ops[t] >> 16) ^ (XB / 2u * u) : ((ops[t] >> 16) ^ (4u * u)) << 4;
                __builtin_memcpy(p.y, __builtin_assume_aligned(smem + x_area + to, CKPT ? E : 16), sizeof p.y);
                if constexpr (CKPT) p.e = *reinterpret_cast<const uint8_t *>(smem + s_area + (to / XB) * 2u + u);
            };
            load(0);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                if (t >= mine) break;
                if (t + 1 < TILES) load(t + 1);
                const Operands &p = o[t & 1];
                uint4v y;
                if constexpr (CKPT) {
                    T w[E];
                    e4m3_to<T, E>(p.y, p.e, w);
                    __builtin_memcpy(&y, w, 16);
                } else {
                    __builtin_memcpy(&y, p.y, 16);
                }
                acc[t] = product<T>(p.x, y, acc[t]);
            }
        }
    };

    for (int s = s0; s < f1; ++s) {
        if (s > s0) lds_barrier();               // (all of the stage before has been read; loads stay in flight)
        if constexpr (CKPT) {
            put_exps(s);
            const int next = (int)((int64_t)(s + 1) * STAGE / 32);
            if (s + 1 < all && next + STAGE / 32 > window + 16) fetch_exps(next);
        }
        const bool more = s + 1 < f1;
        gbase += kRowBytes;
        xbase += XB;
#pragma unroll
        for (int i = 0; i < PG; ++i) {
            if (i * GR >= g_slots) continue;
            if (i * GR + gr < g_slots) *reinterpret_cast<uint4v *>(smem + gu + i * (GR * kRowBytes)) = hg[i];
            if (more) __builtin_memcpy(&hg[i], gbase + go[i], 16);
        }
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            if (i * XR >= x_slots) continue;
            if (i * XR + xr < x_slots) *reinterpret_cast<uint4v *>(smem + xu + i * (XR * XB)) = hx[i];
            if (more) __builtin_memcpy(&hx[i], xbase + xo[i], 16);
        }
        lds_barrier();
        multiply();
    }
    if (f1 < s1) {
        // the stage behind the last full one, in the last range
        const int n0 = full * STAGE;
        __syncthreads();
        if constexpr (CKPT) put_exps(full);
        for (int p = threadIdx.x; p < (g_slots + (CKPT ? 0 : x_slots)) * 8; p += kThreads) {
            const int slot = p / 8, q = p % 8;
            const bool in_g = slot < g_slots;
            const T *src = in_g ? static_cast<const T *>(a.G) + (int64_t)rows[slot] * a.ldg : static_cast<const T *>(a.X) + (int64_t)rows[slot] * a.ldx;
            T w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] = (T)0.f;
                if (n0 + q * E + e < a.N) w[e] = src[n0 + q * E + e];
            }
            uint4v o;
            __builtin_memcpy(&o, w, 16);
            *reinterpret_cast<uint4v *>(smem + (in_g ? place<kRowBytes>((uint32_t)slot, (uint32_t)q)
                                                     : x_area + place<kRowBytes>((uint32_t)(slot - g_slots), (uint32_t)q))) = o;
        }
        if constexpr (CKPT)
            for (int p = threadIdx.x; p < x_slots * XL; p += kThreads) {
                const int slot = p / XL, q = p % XL, col = n0 + q * 16;
                const uint8_t *src = static_cast<const uint8_t *>(a.X) + (int64_t)rows[g_slots + slot] * a.ldx;
                uint4v codes = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (col + e < a.N) codes[e / 4] |= (uint32_t)src[col + e] << (8 * (e & 3));
                *reinterpret_cast<uint4v *>(smem + x_area + place<XB>((uint32_t)slot, (uint32_t)q)) = codes;
            }
        __syncthreads();
        multiply();
    }

#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        if (t >= mine) continue;
        store_tile(a, acc[t], split, first + my0 + t, lane);
    }
}

// The ranges' sums, in order, to the values' places (no ranges: zeros).
__global__ __launch_bounds__(256) void weight_sum_kernel(GradArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n_tiles * 64) return;
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) sum += *reinterpret_cast<const float4v *>(a.part + ((int64_t)s * a.n_tiles * 64 + i) * 4);
    const uint4v to = *reinterpret_cast<const uint4v *>(a.inv + i * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if ((int32_t)to[e] >= 0) a.out[to[e]] = a.accumulate ? a.out[to[e]] + sum[e] : sum[e];
}

template <typename T, bool CKPT, int SHAPE> ubp_status launch_one(GradArgs a, hipStream_t st, bool dry) {
    constexpr GradShape S = kGradShapes[SHAPE];
    constexpr auto kernel = &weight_grad_kernel<T, CKPT, S.tiles, S.g_slots, S.x_slots>;
    constexpr int STAGE = kRowBytes / (int)sizeof(T);
    static LdsLimit limit;
    const ubp_status rc = limit.raise(reinterpret_cast<const void *>(kernel));
    if (rc != UBP_OK || dry) return rc;
    const int64_t grid = 8 * (((int64_t)a.n_regions * a.splits + 7) / 8);
    if (grid * kThreads >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED; // (a launch's threads are counted in 32 bits)
    static_assert(kGradUnit % STAGE == 0, "a range is whole stages");
    a.per_split /= STAGE;
    const size_t lds = (size_t)a.slots_g * kRowBytes + (size_t)a.slots_x * (CKPT ? STAGE + 2 : kRowBytes);
    return launch_kernel(kernel, dim3((unsigned)grid), dim3(kThreads), lds, st, a);
}

template <typename T, bool CKPT> ubp_status launch_t(const GradArgs &a, int shape, hipStream_t st, bool dry) {
    static_assert(kNumGradShapes == 3, "their instantiations");
    switch (shape) {
    case 0: return launch_one<T, CKPT, 0>(a, st, dry);
    case 1: return launch_one<T, CKPT, 1>(a, st, dry);
    case 2: return launch_one<T, CKPT, 2>(a, st, dry);
    }
    return UBP_ERR_UNSUPPORTED;
}

} // namespace

ubp_status launch_weight_grad(const GradArgs &a, ubp_dtype dtype, bool checkpoint, int shape, void *stream, bool dry) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (dtype) {
    case UBP_F32: return checkpoint ? launch_t<float, true>(a, shape, st, dry) : launch_t<float, false>(a, shape, st, dry);
    case UBP_F16: return checkpoint ? launch_t<_Float16, true>(a, shape, st, dry) : launch_t<_Float16, false>(a, shape, st, dry);
    case UBP_BF16: return checkpoint ? launch_t<__bf16, true>(a, shape, st, dry) : launch_t<__bf16, false>(a, shape, st, dry);
    }
    return UBP_ERR_INVALID_ARG;
}

ubp_status launch_weight_sum(const GradArgs &a, void *stream) {
    const int64_t grid = (a.n_tiles * 64 + 255) / 256;
    if (grid * 256 >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED;
    return launch_kernel(&weight_sum_kernel, dim3((unsigned)grid), dim3(256), 0, static_cast<hipStream_t>(stream), a);
}

} // namespace ubp
