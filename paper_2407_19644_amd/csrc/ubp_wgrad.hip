// Weight gradient of a pruned layer: dW[i][k] = sum over the tokens of G[i][n] X[k][n], for the kept weights alone.
#include "ubp_device.h"
#include "ubp_fp8.h"

#include <cstdint>

namespace ubp {

namespace {

constexpr int kRowBytes = kGradRowBytes; // of a row of G or X that a stage takes: 64 16-bit or 32 fp32 tokens, a cache line
constexpr int kThreads = 64 * kGradWaves;

// A stage lies in LDS in two halves, each with rows of BYTES bytes: 64 of G and X, 32 or 16 of a checkpoint's codes.  Place of
// 16-byte piece q of row r of a half: 16 neighbouring rows of one piece lie in all 16 units of 256 bytes, i.e. in all 64 banks.
template <int BYTES> __device__ __forceinline__ uint32_t place(uint32_t r, uint32_t q) {
    static_assert(BYTES == 64 || BYTES == 32 || BYTES == 16, "a row of half a stage");
    return r * BYTES + 16u * (BYTES == 64 ? q ^ ((r >> 2) & 3u) : BYTES == 32 ? q ^ ((r >> 3) & 1u) : q);
}

// LDS by its byte addresses, of which a constant part costs nothing.
template <typename V> __device__ __forceinline__ V lds_get(uint32_t at, int offset = 0) {
    typedef __attribute__((address_space(3))) const char *bytes;
    typedef __attribute__((address_space(3))) const V *values;
    return *(values)((bytes)(uintptr_t)at + offset);
}
template <typename V> __device__ __forceinline__ void lds_put(uint32_t at, V v, int offset = 0) {
    typedef __attribute__((address_space(3))) char *bytes;
    typedef __attribute__((address_space(3))) V *values;
    *(values)((bytes)(uintptr_t)at + offset) = v;
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

// The first `count` of the elements that 16 bytes hold, zeros behind them; nothing behind them is read.  (Fewer bytes than 16
// are 8, 4, 2 and 1 of them, side by side, as many loads at most and all in flight together: one element after the other, each
// would wait for memory, which for 7 tokens took as long as 6 stages.)
template <typename T> __device__ __forceinline__ uint4v first_of(const T *src, int count) {
    uint4v o = {0u, 0u, 0u, 0u};
    if (count >= 16 / (int)sizeof(T)) {
        __builtin_memcpy(&o, src, 16);
        return o;
    }
    const uint32_t c = (uint32_t)max(count, 0) * (uint32_t)sizeof(T);
    const char *from = reinterpret_cast<const char *>(src);
    uint64_t p8 = 0;
    uint32_t p4 = 0;
    uint16_t p2 = 0;
    uint8_t p1 = 0;
    if (c & 8u) __builtin_memcpy(&p8, from, 8);
    if (c & 4u) __builtin_memcpy(&p4, from + (c & 8u), 4);
    if (sizeof(T) < 4 && (c & 2u)) __builtin_memcpy(&p2, from + (c & 12u), 2);
    if (sizeof(T) < 2 && (c & 1u)) p1 = (uint8_t)from[c & 14u];
    uint64_t v = p1;
    if (c & 2u) v = v << 16 | p2;
    if (c & 4u) v = v << 32 | p4;
    const uint64_t lo = c & 8u ? p8 : v, hi = c & 8u ? v : 0u;
    return uint4v{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
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
//  * A tile reads 1 KB of each operand from LDS per half a stage (both halves at addresses a constant apart; the rows of G
//    once for tiles of one window), and its sums stay in a wavefront's registers for the whole range.  The other wavefronts
//    of the SIMD, three of them, cover the way from LDS: operands fetched a tile ahead took registers, and no less time.
//  * CKPT: X is a checkpoint.  Its codes stay as they are in LDS, and a lane widens its 8 codes of a tile by 4 conversions that
//    take the exponent along: exact but for fp16 values below its normal range.  Exponents come 16 at a time.
//  * Rows are 32-bit byte offsets from a place that moves on by a stage: a load takes no arithmetic.  FAR: G or X reaches over
//    4 GB, and rows are numbers, whose addresses of 64 bits are formed again for every load.
//  * LDS begins with a checkpoint's exponents, then X, then G, so that the places of both operands of a tile fit one register.
//  * The last stage of a row may be short; zeros stand behind its last token.
//  * Ranges of tokens are summed by a second kernel, in order; with one range the sums go straight to their places.
// Measured: 4096 x 4096, 10 % in 16 x 16 blocks, bf16, 8192 tokens from a checkpoint: 107 us with the second kernel's 9 (inputs in
// rotation), 256 TFLOP/s of kept products; 256 x 2304, 25 % in 4 x 4 blocks, 12544 tokens: 38 us.  What bounds it: the stages'
// parts, one behind the other.  Of the first: 11 us before and after the stages, 27 for the way into LDS and its barriers, 42 for
// the products (LDS has 31 % of its cycles taken), 12 in which loads are waited for; loads by themselves take 40.  Two stages in
// LDS, which would overlap them, leave room for half the rows: regions are smaller and read rows more often (143 us, and 41).
template <typename T, bool CKPT, bool FAR, int TILES, int GS, int XS>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(GradArgs a) {
    constexpr int E = 16 / (int)sizeof(T);       // tokens of a 16-byte piece
    constexpr int STAGE = 8 * E;                 // tokens of a stage
    constexpr int XB = CKPT ? STAGE : kRowBytes; // bytes of a row of X
    constexpr int GH = kRowBytes / 2, XH = XB / 2; // of half a stage
    // Halves lie 64 bytes more apart than their rows take: the 8 lanes that LDS serves together write one row's pieces of both
    // halves (or two or four rows of codes), which would meet in the same banks.
    constexpr int G_HALF = GS * GH + 64, X_HALF = XS * XH + 64, X_AREA = CKPT ? 8 * XS : 0, G_AREA = X_AREA + 2 * X_HALF;
    constexpr int XL = XB / 16;                  // lanes that load it
    constexpr int GR = kThreads / 8, XR = kThreads / XL; // rows at once
    constexpr int PG = (GS + GR - 1) / GR, PX = (XS + XR - 1) / XR; // loads per lane
    static_assert(XS <= kThreads, "a lane per row for the exponents");
    static_assert((G_AREA + G_HALF) / 2 <= 65536 && X_HALF <= 65536 && G_AREA % 16 == 0, "places of 16 bits");
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
    const int region = (int)(pair % a.n_regions);
    const int32_t *reg = a.regions + 4 * region;
    const int first = reg[0], tiles = reg[1], g_slots = reg[2], x_slots = reg[3];
    // (lists of one length, filled up with some row: to read them takes nothing but the region's number)
    const int32_t *rows_g = a.rows + (int64_t)region * (a.slots_g + a.slots_x), *rows_x = rows_g + a.slots_g;

    const int all = (int)(((int64_t)a.N + STAGE - 1) / STAGE), full = a.N / STAGE;
    const int s0 = split * a.per_split, s1 = split == a.splits - 1 ? all : s0 + a.per_split, f1 = min(s1, full);

    // this lane's rows: pass i takes row list entries i GR + thread / 8 (of X: i XR + thread / XL), at a place a constant further on
    uint32_t g_row[PG], x_row[PX];
    const uint32_t gq = threadIdx.x % 8, xq = threadIdx.x % XL;
    const int gr = (int)threadIdx.x / 8, xr = (int)threadIdx.x / XL;
    const int64_t g_pitch = a.ldg * (int)sizeof(T), x_pitch = a.ldx * (CKPT ? 1 : (int)sizeof(T));
    const char *gbase = static_cast<const char *>(a.G) + (int64_t)s0 * kRowBytes, *xbase = static_cast<const char *>(a.X) + (int64_t)s0 * XB;
    auto piece = [&](uint32_t &row, const char *base, int64_t pitch, uint32_t q) {
        asm volatile("" : "+v"(row));            // (or all addresses are kept, in registers that there are not)
        if constexpr (FAR) return base + ((int64_t)row * pitch + 16 * q);
        else return base + row;
    };
    auto g_piece = [&](int i) { return piece(g_row[i], gbase, g_pitch, gq); };
    auto x_piece = [&](int i) { return piece(x_row[i], xbase, x_pitch, xq); };
    auto g_place = [&](uint32_t slot, uint32_t q) { return G_AREA + q / 4 * G_HALF + place<GH>(slot, q % 4); };
    auto x_place = [&](uint32_t slot, uint32_t q) { return X_AREA + q / (XL / 2) * X_HALF + place<XH>(slot, q % (XL / 2)); };
    const uint32_t gu = g_place((uint32_t)gr, gq), xu = x_place((uint32_t)xr, xq);
    static_assert(GR % 16 == 0 && XR % 16 == 0, "the rows of two passes differ by a multiple of 16: their places by a constant");
#pragma unroll
    for (int i = 0; i < PG; ++i) {
        g_row[i] = (uint32_t)rows_g[min(i * GR + gr, a.slots_g - 1)];
        if (!FAR) g_row[i] = g_row[i] * (uint32_t)g_pitch + 16 * gq;
    }
#pragma unroll
    for (int i = 0; i < PX; ++i) {
        x_row[i] = (uint32_t)rows_x[min(i * XR + xr, a.slots_x - 1)];
        if (!FAR) x_row[i] = x_row[i] * (uint32_t)x_pitch + 16 * xq;
    }
    // exponents: lane r has up to 16 neighbouring ones of row r, the next stage's first.  Those after a range's first 16 have 16
    // at least before them.
    constexpr int SG = STAGE / 32;               // groups of a stage: 2 or 1
    const int groups = (int)(((int64_t)a.N + 31) / 32);
    [[maybe_unused]] const uint8_t *sp = nullptr;
    [[maybe_unused]] uint4v exps = {0u, 0u, 0u, 0u};
    [[maybe_unused]] int have = 0;               // stages that are left in them
    [[maybe_unused]] auto fetch_exps = [&](int s) {
        const int group = s * SG;
        __builtin_memcpy(&exps, sp + min(group, groups - 16), 16);
        // (a row's last ones lie behind others that were there before: 32-bit words, then bytes move down, in place)
        const int past = group + 16 - groups;
        if (past > 0) {
            for (int k = past >> 2; k > 0; --k) exps = uint4v{exps[1], exps[2], exps[3], 0u};
#pragma unroll
            for (int k = 0; k < 4; ++k) exps[k] = __builtin_amdgcn_alignbyte(k < 3 ? exps[k < 3 ? k + 1 : 3] : 0u, exps[k], (uint32_t)past & 3u);
        }
        have = 16 / SG;
    };
    // a stage's exponents as the floats that conversions take, two for each row
    [[maybe_unused]] auto put_exps = [&]() {
        const uint32_t b0 = exps[0] & 0xffu, b1 = SG == 2 ? (exps[0] >> 8) & 0xffu : b0;
        if ((int)threadIdx.x < x_slots) lds_put(8 * threadIdx.x, uint2v{b0 << 23, b1 << 23});
#pragma unroll
        for (int k = 0; k < 4; ++k) exps[k] = exps[k] >> (8 * SG) | (k < 3 ? exps[k < 3 ? k + 1 : 3] << (32 - 8 * SG) : 0u);
        --have;
    };
    if constexpr (CKPT) {
        sp = a.S + (int64_t)rows_x[min((int)threadIdx.x, a.slots_x - 1)] * a.lds;
        exps = first_of(sp + s0 * SG, groups - s0 * SG);
        have = 16 / SG;
    }

    uint4v hg[PG], hx[PX];
    if (s0 < f1) {
#pragma unroll
        for (int i = 0; i < PG; ++i)
            if (i * GR < g_slots) __builtin_memcpy(&hg[i], g_piece(i), 16);
#pragma unroll
        for (int i = 0; i < PX; ++i)
            if (i * XR < x_slots) __builtin_memcpy(&hx[i], x_piece(i), 16);
    }

    // ---- this wavefront's tiles: places of this lane's pieces of the first half
    // (what is left over goes to the first wavefronts, one to each SIMD in turn)
    const int per = tiles / kGradWaves, more_of = tiles % kGradWaves;
    const int my0 = wave * per + min(wave, more_of), mine = per + (wave < more_of ? 1 : 0);
    // (half of G's, X's behind X_AREA << 16)
    uint32_t places[TILES], fresh = 0, before = 0; // (fresh, bit t: tile t's rows of G are not those of tile t - 1)
    float4v acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const uint32_t o = t < mine ? a.ops[(int64_t)(first + my0 + t) * 16 + n] : 0u, x = o >> 16;
        const uint32_t pb = CKPT ? place<XH>(x, g * E / 16) + g * E % 16 : place<XH>(x, g);
        places[t] = (G_AREA + place<GH>(o & 0xffffu, g)) / 2 | pb << 16;
        if (t == 0 || __any((o & 0xffffu) != before)) fresh |= 1u << t;
        before = o & 0xffffu;
        acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    auto multiply = [&]() {
        uint4v x[2];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if (t >= mine) break;
            uint32_t at = places[t];
            asm volatile("" : "+v"(at));         // (or the addresses of all tiles are kept in registers that there are not)
            const uint32_t pa = (at & 0xffffu) * 2u, pb = at >> 16;
            if (fresh >> t & 1u) {
#pragma unroll
                for (int u = 0; u < 2; ++u) x[u] = lds_get<uint4v>(pa, u * G_HALF);
            }
            typedef __attribute__((__vector_size__(CKPT ? E : 16))) uint32_t piece_t;
            piece_t c[2];
            [[maybe_unused]] uint2v e;
#pragma unroll
            for (int u = 0; u < 2; ++u) c[u] = lds_get<piece_t>(pb, X_AREA + u * X_HALF);
            if constexpr (CKPT) e = lds_get<uint2v>(pb / XH * 8u);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint4v y;
                if constexpr (CKPT) {
                    T w[E];
                    uint32_t codes[E / 4];
                    __builtin_memcpy(codes, &c[u], sizeof codes);
                    e4m3_to<T, E>(codes, __builtin_bit_cast(float, (uint32_t)e[u]), w);
                    __builtin_memcpy(&y, w, 16);
                } else {
                    __builtin_memcpy(&y, &c[u], 16);
                }
                acc[t] = product<T>(x[u], y, acc[t]);
            }
        }
    };

    for (int s = s0; s < f1; ++s) {
        if (s > s0) lds_barrier();               // (all of the stage before has been read; loads stay in flight)
        if constexpr (CKPT) {
            put_exps();
            if (have == 0 && s + 1 < s1) fetch_exps(s + 1);
        }
        const bool more = s + 1 < f1;
        gbase += kRowBytes;
        xbase += XB;
#pragma unroll
        for (int i = 0; i < PG; ++i) {
            if (i * GR >= g_slots) continue;
            if (i * GR + gr < g_slots) lds_put(gu, hg[i], i * (GR * GH));
            if (more) __builtin_memcpy(&hg[i], g_piece(i), 16);
        }
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            if (i * XR >= x_slots) continue;
            if (i * XR + xr < x_slots) lds_put(xu, hx[i], i * (XR * XH));
            if (more) __builtin_memcpy(&hx[i], x_piece(i), 16);
        }
        lds_barrier();
        multiply();
    }
    if (f1 < s1) {
        // the stage behind the last full one, in the last range
        const int n0 = full * STAGE;
        __syncthreads();
        if constexpr (CKPT) put_exps();
        for (int p = threadIdx.x; p < (g_slots + (CKPT ? 0 : x_slots)) * 8; p += kThreads) {
            const int slot = p / 8, q = p % 8;
            const bool in_g = slot < g_slots;
            const T *src = in_g ? static_cast<const T *>(a.G) + (int64_t)rows_g[slot] * a.ldg : static_cast<const T *>(a.X) + (int64_t)rows_x[slot - g_slots] * a.ldx;
            const uint4v o = first_of(src + n0 + q * E, a.N - n0 - q * E);
            lds_put(in_g ? g_place((uint32_t)slot, (uint32_t)q) : x_place((uint32_t)(slot - g_slots), (uint32_t)q), o);
        }
        if constexpr (CKPT)
            for (int p = threadIdx.x; p < x_slots * XL; p += kThreads) {
                const int slot = p / XL, q = p % XL, col = n0 + q * 16;
                const uint8_t *src = static_cast<const uint8_t *>(a.X) + (int64_t)rows_x[slot] * a.ldx;
                const uint4v codes = first_of(src + col, a.N - col);
                lds_put(x_place((uint32_t)slot, (uint32_t)q), codes);
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
    // (8 at a time: one after the other, each would wait for memory)
    for (int s = 0; s < a.splits; s += 8) {
        float4v v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const float4v *>(a.part + ((int64_t)min(s + k, a.splits - 1) * a.n_tiles * 64 + i) * 4);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (s + k < a.splits) sum += v[k];
    }
    const uint4v to = *reinterpret_cast<const uint4v *>(a.inv + i * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if ((int32_t)to[e] >= 0) a.out[to[e]] = a.accumulate ? a.out[to[e]] + sum[e] : sum[e];
}

template <typename T, bool CKPT, bool FAR, int SHAPE> ubp_status launch_one(GradArgs a, hipStream_t st, bool dry) {
    constexpr GradShape S = kGradShapes[SHAPE];
    constexpr auto kernel = &weight_grad_kernel<T, CKPT, FAR, S.tiles, S.g_slots, S.x_slots>;
    constexpr int STAGE = kRowBytes / (int)sizeof(T);
    static LdsLimit limit;
    const ubp_status rc = limit.raise(reinterpret_cast<const void *>(kernel), true);
    if (rc != UBP_OK || dry) return rc;
    const int64_t grid = 8 * (((int64_t)a.n_regions * a.splits + 7) / 8);
    if (grid * kThreads >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED; // (a launch's threads are counted in 32 bits)
    static_assert(kGradUnit % STAGE == 0, "a range is whole stages");
    a.per_split /= STAGE;
    constexpr size_t lds = 256 + (size_t)S.g_slots * kRowBytes + (size_t)S.x_slots * (CKPT ? STAGE + 8 : kRowBytes);
    static_assert(lds <= 160 * 1024, "a stage fits LDS");
    return launch_kernel(kernel, dim3((unsigned)grid), dim3(kThreads), lds, st, a);
}

template <typename T, bool CKPT, int SHAPE> ubp_status launch_shape(const GradArgs &a, hipStream_t st, bool dry) {
    if (dry) {
        const ubp_status rc = launch_one<T, CKPT, false, SHAPE>(a, st, dry);
        return rc != UBP_OK ? rc : launch_one<T, CKPT, true, SHAPE>(a, st, dry);
    }
    return a.far_rows ? launch_one<T, CKPT, true, SHAPE>(a, st, dry) : launch_one<T, CKPT, false, SHAPE>(a, st, dry);
}
template <typename T, bool CKPT> ubp_status launch_t(const GradArgs &a, int shape, hipStream_t st, bool dry) {
    static_assert(kNumGradShapes == 3, "their instantiations");
    switch (shape) {
    case 0: return launch_shape<T, CKPT, 0>(a, st, dry);
    case 1: return launch_shape<T, CKPT, 1>(a, st, dry);
    case 2: return launch_shape<T, CKPT, 2>(a, st, dry);
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
