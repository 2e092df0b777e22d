// Weight gradient of a pruned layer: dW[i][k] = sum over the tokens of G[i][n] X[k][n], for the kept weights alone.
#include "ubp_device.h"
#include "ubp_fp8.h"

#include <cstdint>

namespace ubp {

namespace {

constexpr int kRowBytes = 64; // of a row of G or X that a step takes: 32 16-bit or 16 fp32 tokens
constexpr int kThreads = 64 * kGradWaves;

// The 16-byte unit of piece q of LDS row r: 16 neighbouring rows of one piece lie in all 16 units of 256 bytes, i.e. in
// all 64 banks.
__device__ __forceinline__ uint32_t unit_of(uint32_t r, uint32_t q) { return 4u * r + (q ^ ((r >> 2) & 3u)); }

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

// One workgroup = one region (at most 8 T tiles of 16 rows of G x 16 rows of X) and one range of tokens.  Both operands of
// the matrix instruction have the tokens along their inner dimension, as G and X have them in memory, so that a tile may
// pair any rows: nothing is transposed, and only tiles that keep weights are formed.
//  * A step = 64 bytes of every row that the region needs, through registers into one of two LDS buffers (the next step's
//    loads are in flight while this one is multiplied), 16 bytes per lane.
//  * A tile reads 1 KB of each operand from LDS per step, and its sums stay in a wavefront's registers for the whole range.
//  * Ranges of tokens are summed by a second kernel, in order; with one range the sums go straight to their places.
// CKPT: X is a checkpoint (8 bits and an exponent per 32 tokens), widened to T's type on its way into LDS, which is exact
// but for fp16 values below its normal range.
template <typename T, bool CKPT, int TILES>
__global__ __launch_bounds__(kThreads, 2) void weight_grad_kernel(GradArgs a) {
    constexpr int E = 16 / (int)sizeof(T);       // tokens of a 16-byte piece
    constexpr int STEP = 4 * E;                  // tokens of a step
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, n = lane & 15;
    // Workgroup ids go round-robin over the 8 XCDs: the pairs, regions of a range next to each other, are cut into 8 equal
    // runs, so that a range's rows come from memory to about one L2.
    const int64_t pairs = (int64_t)a.n_regions * a.splits;
    const int xcd = blockIdx.x & 7;
    const int64_t pair = (pairs * xcd >> 3) + (blockIdx.x >> 3);
    if (pair >= (pairs * (xcd + 1) >> 3)) return;
    const int split = (int)(pair / a.n_regions);
    const int32_t *reg = a.regions + 8 * (pair % a.n_regions);
    const int first = reg[0], tiles = reg[1], g_slots = reg[3], slots = reg[4];
    const int32_t *rows = a.rows + reg[2];

    const int per = (tiles + kGradWaves - 1) / kGradWaves;
    const int my0 = wave * per, mine = min(per, tiles - my0);
    // LDS units of this lane's pieces: row n of the tile's rows of G | of X << 16
    uint32_t ops[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const uint32_t o = t < mine ? a.ops[(int64_t)(first + my0 + t) * 16 + n] : 0u;
        ops[t] = unit_of(o & 0xffffu, (uint32_t)g) | unit_of(o >> 16, (uint32_t)g) << 16;
    }
    float4v acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = float4v{0.f, 0.f, 0.f, 0.f};

    const int all_steps = (a.N + STEP - 1) / STEP;
    const int s0 = split * a.per_split, s1 = min(s0 + a.per_split, all_steps);
    const int q = threadIdx.x & 3;               // this thread's piece of its rows
    constexpr int kRowsAtOnce = kThreads / 4;
    constexpr int MAXP = (kGradMaxSlots + kRowsAtOnce - 1) / kRowsAtOnce;
    const uint32_t buffer = (uint32_t)a.slots * kRowBytes;

    uint4v held[MAXP];
    auto fetch = [&](int s) {
        const int n0 = s * STEP + q * E;         // first token of the piece
#pragma unroll
        for (int i = 0; i < MAXP; ++i) {
            const int slot = i * kRowsAtOnce + (int)(threadIdx.x >> 2);
            if (i * kRowsAtOnce >= slots) break;
            held[i] = uint4v{0u, 0u, 0u, 0u};
            if (slot >= slots) continue;
            const int row = rows[slot];
            if (row < 0 || n0 >= a.N) continue;
            if (CKPT && slot >= g_slots) {
                const uint8_t *src = static_cast<const uint8_t *>(a.X) + (int64_t)row * a.ldx + n0;
                uint32_t b[2] = {0u, 0u};
                if (n0 + E <= a.N) {
                    __builtin_memcpy(b, src, E);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (n0 + e < a.N) b[e / 4] |= (uint32_t)src[e] << (8 * (e & 3));
                }
                const float scale = exponent_value(a.S[(int64_t)row * a.lds + (n0 >> 5)]);
                float v[E];
                e4m3_values<E>(b, scale, v);
                T w[E];
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = from_f32<T>(v[e]);
                __builtin_memcpy(&held[i], w, 16);
            } else {
                const T *src = slot < g_slots ? static_cast<const T *>(a.G) + (int64_t)row * a.ldg + n0
                                              : static_cast<const T *>(a.X) + (int64_t)row * a.ldx + n0;
                if (n0 + E <= a.N) {
                    __builtin_memcpy(&held[i], src, 16);
                } else {
                    T w[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        w[e] = (T)0.f;
                        if (n0 + e < a.N) w[e] = src[e];
                    }
                    __builtin_memcpy(&held[i], w, 16);
                }
            }
        }
    };
    auto put = [&](uint32_t at) {
#pragma unroll
        for (int i = 0; i < MAXP; ++i) {
            const int slot = i * kRowsAtOnce + (int)(threadIdx.x >> 2);
            if (i * kRowsAtOnce >= slots) break;
            if (slot < slots) *reinterpret_cast<uint4v *>(smem + at + 16u * unit_of((uint32_t)slot, (uint32_t)q)) = held[i];
        }
    };

    if (s0 < s1) {
        fetch(s0);
        put(0u);
    }
    __syncthreads();
    uint32_t at = 0u;
    for (int s = s0; s < s1; ++s) {
        if (s + 1 < s1) fetch(s + 1);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const uint4v x = *reinterpret_cast<const uint4v *>(smem + at + 16u * (ops[t] & 0xffffu));
            const uint4v y = *reinterpret_cast<const uint4v *>(smem + at + 16u * (ops[t] >> 16));
            acc[t] = product<T>(x, y, acc[t]);
        }
        at = buffer - at;
        if (s + 1 < s1) put(at);
        __syncthreads();
    }

#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        if (t >= mine) continue;
        const int64_t tile = first + my0 + t;
        if (a.part) {
            *reinterpret_cast<float4v *>(a.part + ((int64_t)split * a.n_tiles + tile) * 256 + lane * 4) = acc[t];
        } else {
            const uint4v to = *reinterpret_cast<const uint4v *>(a.inv + tile * 256 + lane * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((int32_t)to[e] >= 0) a.out[to[e]] = a.accumulate ? a.out[to[e]] + acc[t][e] : acc[t][e];
        }
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

template <typename T, bool CKPT, int TILES> ubp_status launch_one(const GradArgs &a, hipStream_t st, bool dry) {
    static LdsLimit limit;
    const ubp_status rc = limit.raise(reinterpret_cast<const void *>(&weight_grad_kernel<T, CKPT, TILES>));
    if (rc != UBP_OK || dry) return rc;
    const int64_t grid = 8 * (((int64_t)a.n_regions * a.splits + 7) / 8);
    if (grid * kThreads >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED; // (a launch's threads are counted in 32 bits)
    return launch_kernel(&weight_grad_kernel<T, CKPT, TILES>, dim3((unsigned)grid), dim3(kThreads), (size_t)2 * a.slots * kRowBytes, st, a);
}

template <typename T, bool CKPT> ubp_status launch_t(const GradArgs &a, int tiles, hipStream_t st, bool dry) {
    if (tiles <= 2) return launch_one<T, CKPT, 2>(a, st, dry);
    if (tiles <= 4) return launch_one<T, CKPT, 4>(a, st, dry);
    if (tiles <= 8) return launch_one<T, CKPT, 8>(a, st, dry);
    if (tiles <= 16) return launch_one<T, CKPT, 16>(a, st, dry);
    static_assert(kGradMaxTiles == 28, "the largest instantiation");
    return launch_one<T, CKPT, kGradMaxTiles>(a, st, dry);
}

} // namespace

ubp_status launch_weight_grad(const GradArgs &a, ubp_dtype dtype, bool checkpoint, int max_tiles, void *stream, bool dry) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (dtype) {
    case UBP_F32: return checkpoint ? launch_t<float, true>(a, max_tiles, st, dry) : launch_t<float, false>(a, max_tiles, st, dry);
    case UBP_F16: return checkpoint ? launch_t<_Float16, true>(a, max_tiles, st, dry) : launch_t<_Float16, false>(a, max_tiles, st, dry);
    case UBP_BF16: return checkpoint ? launch_t<__bf16, true>(a, max_tiles, st, dry) : launch_t<__bf16, false>(a, max_tiles, st, dry);
    }
    return UBP_ERR_INVALID_ARG;
}

ubp_status launch_weight_sum(const GradArgs &a, void *stream) {
    const int64_t grid = (a.n_tiles * 64 + 255) / 256;
    if (grid * 256 >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED;
    return launch_kernel(&weight_sum_kernel, dim3((unsigned)grid), dim3(256), 0, static_cast<hipStream_t>(stream), a);
}

} // namespace ubp
