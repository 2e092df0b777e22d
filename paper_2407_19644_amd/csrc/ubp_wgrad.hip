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

// General kernel: rows of any alignment and pitch.
// One workgroup = one region (at most 8 T tiles of 16 rows of G x 16 rows of X) and one range of tokens.  Both operands of
// the matrix instruction have the tokens along their inner dimension, as G and X have them in memory, so that a tile may
// pair any rows: nothing is transposed, and only tiles that keep weights are formed.
//  * A step = 64 bytes of every row that the region needs, through registers into one of two LDS buffers: the next step's
//    loads are all in flight while this one is multiplied.  Rows that no tile asks for (they fill up 16) hold some row of
//    the matrix: what they give is not stored.
//  * A tile reads 1 KB of each operand from LDS per step, two tiles ahead, and its sums stay in a wavefront's registers for
//    the whole range.
//  * The last step of a row may be short; it is staged token by token, zeros behind the last one.
//  * Ranges of tokens are summed by a second kernel, in order; with one range the sums go straight to their places.
// CKPT: X is a checkpoint (8 bits and an exponent per 32 tokens), widened to T's type on its way into LDS, which is exact
// but for fp16 values below its normal range.
template <typename T, bool CKPT, int TILES, int GS, int XS>
__global__ __launch_bounds__(kThreads, 2) void weight_grad_kernel(GradArgs a) {
    constexpr int E = 16 / (int)sizeof(T);       // tokens of a 16-byte piece
    constexpr int STEP = 4 * E;                  // tokens of a step
    constexpr int XL = CKPT ? STEP / 16 : 4;     // lanes that load a row of X
    constexpr int GR = kThreads / 4, XR = kThreads / XL; // rows at once
    constexpr int PG = (GS + GR - 1) / GR, QX = (XS + XR - 1) / XR; // loads per lane
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
    const int first = reg[0], tiles = reg[1], g_slots = reg[3], x_slots = reg[4] - reg[3];
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

    const int all_steps = (a.N + STEP - 1) / STEP, full = a.N / STEP;
    const int s0 = split * a.per_split, s1 = split == a.splits - 1 ? all_steps : s0 + a.per_split;
    const uint32_t buffer = (uint32_t)a.slots * kRowBytes;

    // this lane's rows: slot i of a pass is row list entry i GR + thread / 4 (the last one again behind the end)
    const char *gp[PG], *xp[QX];
    const uint8_t *sp[QX];
    uint32_t gu[PG], xu[QX];
    const int gq = threadIdx.x & 3, xq = threadIdx.x % XL;
#pragma unroll
    for (int i = 0; i < PG; ++i) {
        const int slot = min(i * GR + (int)threadIdx.x / 4, g_slots - 1);
        gp[i] = static_cast<const char *>(a.G) + ((int64_t)rows[slot] * a.ldg + (int64_t)s0 * STEP + gq * E) * (int)sizeof(T);
        gu[i] = 16u * unit_of((uint32_t)slot, (uint32_t)gq);
    }
#pragma unroll
    for (int i = 0; i < QX; ++i) {
        const int slot = g_slots + min(i * XR + (int)threadIdx.x / XL, x_slots - 1);
        const int64_t row = rows[slot];
        if constexpr (CKPT) {
            xp[i] = static_cast<const char *>(a.X) + row * a.ldx + (int64_t)s0 * STEP + xq * 16;
            sp[i] = a.S + row * a.lds + ((int64_t)s0 * STEP >> 5);
            xu[i] = (uint32_t)slot;
        } else {
            xp[i] = static_cast<const char *>(a.X) + (row * a.ldx + (int64_t)s0 * STEP + xq * E) * (int)sizeof(T);
            xu[i] = 16u * unit_of((uint32_t)slot, (uint32_t)xq);
        }
    }
    uint4v hg[PG], hx[QX];
    uint32_t hs[QX];
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < PG; ++i) {
            __builtin_memcpy(&hg[i], gp[i], 16);
            gp[i] += kRowBytes;
        }
#pragma unroll
        for (int i = 0; i < QX; ++i) {
            __builtin_memcpy(&hx[i], xp[i], 16);
            xp[i] += CKPT ? STEP : kRowBytes;
            if constexpr (CKPT) hs[i] = sp[i][((int64_t)s * STEP >> 5) - ((int64_t)s0 * STEP >> 5)];
        }
    };
    auto put_codes = [&](uint32_t at, uint32_t slot, int q16, const uint32_t (&codes)[4], uint32_t byte) {
        // 16 values: 16 / E pieces
        T w[16];
        e4m3_to<T, 16>(codes, byte, w);
#pragma unroll
        for (int h = 0; h < 16 / E; ++h) {
            uint4v o;
            __builtin_memcpy(&o, w + h * E, 16);
            *reinterpret_cast<uint4v *>(smem + at + 16u * unit_of(slot, (uint32_t)(q16 * (16 / E) + h))) = o;
        }
    };
    auto put = [&](uint32_t at) {
#pragma unroll
        for (int i = 0; i < PG; ++i) *reinterpret_cast<uint4v *>(smem + at + gu[i]) = hg[i];
#pragma unroll
        for (int i = 0; i < QX; ++i) {
            if constexpr (CKPT) {
                const uint32_t codes[4] = {hx[i][0], hx[i][1], hx[i][2], hx[i][3]};
                put_codes(at, xu[i], xq, codes, hs[i]);
            } else {
                *reinterpret_cast<uint4v *>(smem + at + xu[i]) = hx[i];
            }
        }
    };
    // the step behind the last full one
    auto put_short = [&](uint32_t at) {
        const int n0 = full * STEP;
        for (int p = threadIdx.x; p < (g_slots + (CKPT ? 0 : x_slots)) * 4; p += kThreads) {
            const int slot = p >> 2, q = p & 3;
            const T *src = slot < g_slots ? static_cast<const T *>(a.G) + (int64_t)rows[slot] * a.ldg
                                          : static_cast<const T *>(a.X) + (int64_t)rows[slot] * a.ldx;
            T w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] = (T)0.f;
                if (n0 + q * E + e < a.N) w[e] = src[n0 + q * E + e];
            }
            uint4v o;
            __builtin_memcpy(&o, w, 16);
            *reinterpret_cast<uint4v *>(smem + at + 16u * unit_of((uint32_t)slot, (uint32_t)q)) = o;
        }
        if constexpr (CKPT)
            for (int p = threadIdx.x; p < x_slots * XL; p += kThreads) {
                const int slot = g_slots + p / XL, q = p % XL;
                const int64_t row = rows[slot];
                const uint8_t *src = static_cast<const uint8_t *>(a.X) + row * a.ldx;
                uint32_t codes[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (n0 + q * 16 + e < a.N) codes[e / 4] |= (uint32_t)src[n0 + q * 16 + e] << (8 * (e & 3));
                put_codes(at, (uint32_t)slot, q, codes, a.S[row * a.lds + (n0 >> 5)]);
            }
    };

    if (s0 < s1) {
        if (s0 < full) {
            fetch(s0);
            put(0u);
        } else {
            put_short(0u);
        }
    }
    __syncthreads();
    uint32_t at = 0u;
    for (int s = s0; s < s1; ++s) {
        const int next = s + 1;
        if (next < s1 && next < full) fetch(next);
        {
            uint4v x[2][2], y[2][2];
            auto load = [&](int t) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    x[(t >> 1) & 1][h] = *reinterpret_cast<const uint4v *>(smem + at + 16u * (ops[t + h] & 0xffffu));
                    y[(t >> 1) & 1][h] = *reinterpret_cast<const uint4v *>(smem + at + 16u * (ops[t + h] >> 16));
                }
            };
            load(0);
#pragma unroll
            for (int t = 0; t < TILES; t += 2) {
                if (t >= mine) break;
                if (t + 2 < TILES) load(t + 2);
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[t + h] = product<T>(x[(t >> 1) & 1][h], y[(t >> 1) & 1][h], acc[t + h]);
            }
        }
        at = buffer - at;
        if (next < s1) {
            if (next < full) put(at);
            else put_short(at);
        }
        __syncthreads();
    }

#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        if (t >= mine) continue;
        store_tile(a, acc[t], split, first + my0 + t, lane);
    }
}

// ------------------------------------------------------------------ rows of 16-byte pieces, many tokens
constexpr int kStreamLoaders = 4;
constexpr int kStreamThreads = 64 * (kGradWaves + kStreamLoaders);
constexpr int kBlock = 128;                      // tokens that 4 exponent bytes cover

// The same regions and sums, with wavefronts that do nothing but start loads straight into a ring of LDS stages, several
// stages ahead; 8 wavefronts multiply.  One barrier per stage: behind it the stage's rows are there and the stage before it is free.
// A checkpoint's codes stay as they are in LDS (half of the bytes on the way there and half of the reads of X), and a lane
// widens its 8 codes of a tile with 4 conversions that take the exponent along; the exponents of its tiles come
// straight from memory, 4 groups at a time, a block of 128 tokens ahead.
// A range is a whole number of blocks; the tokens behind the last block are staged one by one.
template <typename T, bool CKPT, int TILES>
__global__ __launch_bounds__(kStreamThreads) void weight_grad_stream_kernel(GradArgs a) {
    constexpr int E = 16 / (int)sizeof(T);
    constexpr int STAGE = 4 * E;                 // tokens of a stage: 64 bytes of a row
    constexpr int SPB = kBlock / STAGE;          // stages of a block
    constexpr int XB = CKPT ? STAGE : kRowBytes; // bytes of a row of X in LDS
    constexpr int XROWS = 1024 / XB;             // rows of X that a load of a wavefront covers
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, n = lane & 15;
    const int64_t pairs = (int64_t)a.n_regions * a.splits;
    const int xcd = blockIdx.x & 7;
    const int64_t pair = (pairs * xcd >> 3) + (blockIdx.x >> 3);
    if (pair >= (pairs * (xcd + 1) >> 3)) return;
    const int split = (int)(pair / a.n_regions);
    const int32_t *reg = a.regions + 8 * (pair % a.n_regions);
    const int first = reg[0], tiles = reg[1], g_slots = reg[3], x_slots = reg[4] - reg[3];
    const int32_t *rows = a.rows + reg[2];
    const int s0 = split * a.per_split, f1 = min(s0 + a.per_split, a.N / kBlock * SPB);
    const int stages = max(0, f1 - s0);
    const bool last = split == a.splits - 1;
    const uint32_t x_area = (uint32_t)a.slots_g * kRowBytes, stage_bytes = (uint32_t)a.stage_bytes;
    const int ring = a.ring;

    const int per = (tiles + kGradWaves - 1) / kGradWaves;
    const int my0 = wave * per, mine = wave < kGradWaves ? min(per, tiles - my0) : 0;
    float4v acc[TILES];
    uint32_t ops[TILES];                         // bytes of a stage: this lane's piece of the rows of G | of X << 16
    [[maybe_unused]] uint32_t exps[TILES];       // offset of this lane's row in S
    auto multiply = [&](uint32_t at, [[maybe_unused]] const uint32_t (&words)[TILES], [[maybe_unused]] int shift) {
        struct Operands {
            uint4v x;
            uint32_t y[CKPT ? E / 4 : 4];
        };
        Operands o[2][2];
        auto load = [&](int t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                o[(t >> 1) & 1][h].x = *reinterpret_cast<const uint4v *>(smem + at + (ops[t + h] & 0xffffu));
                __builtin_memcpy(o[(t >> 1) & 1][h].y, __builtin_assume_aligned(smem + at + (ops[t + h] >> 16), CKPT ? E : 16), sizeof o[0][0].y);
            }
        };
        load(0);
#pragma unroll
        for (int t = 0; t < TILES; t += 2) {
            if (t >= mine) break;
            if (t + 2 < TILES) load(t + 2);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Operands &p = o[(t >> 1) & 1][h];
                uint4v y;
                if constexpr (CKPT) {
                    T w[E];
                    e4m3_to<T, E>(p.y, (words[t + h] >> shift) & 0xffu, w);
                    __builtin_memcpy(&y, w, 16);
                } else {
                    __builtin_memcpy(&y, p.y, 16);
                }
                acc[t + h] = product<T>(p.x, y, acc[t + h]);
            }
        }
    };

    if (wave >= kGradWaves) {
        // ---- loads: number j = me, me + loaders, ..: 16 rows of G each, then XROWS rows of X each
        const int me = wave - kGradWaves;
        const int n_g = g_slots / 16, n_all = n_g + (x_slots + XROWS - 1) / XROWS;
        constexpr int LOADS = (kGradSlots / 16 + kStreamLoaders) / kStreamLoaders;
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
        uint32_t off[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int j = me + i * kStreamLoaders;
            if (j < n_g) {
                const int slot = 16 * j + (lane >> 2);
                off[i] = (uint32_t)rows[slot] * (uint32_t)a.ldg * (uint32_t)sizeof(T) + 16u * ((lane & 3) ^ ((slot >> 2) & 3));
            } else {
                constexpr int L = XB / 16;        // lanes of a row
                const int slot = XROWS * (j - n_g) + lane / L;
                const uint32_t row = (uint32_t)rows[g_slots + min(slot, x_slots - 1)];
                uint32_t q = (uint32_t)(lane % L);
                if constexpr (L == 4) q ^= (uint32_t)((slot >> 2) & 3);
                if constexpr (L == 2) q ^= (uint32_t)((slot >> 3) & 1);
                off[i] = row * (uint32_t)a.ldx * (CKPT ? 1u : (uint32_t)sizeof(T)) + 16u * q;
            }
        }
        const int mine_loads = (n_all - me + kStreamLoaders - 1) / kStreamLoaders;
        const char *gb = static_cast<const char *>(a.G) + (int64_t)s0 * kRowBytes;
        const char *xb = static_cast<const char *>(a.X) + (int64_t)s0 * XB;
        uint32_t slot_at = 0;
        auto issue = [&]() {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int j = me + i * kStreamLoaders;
                if (j < n_g) load16_to_lds(gb, off[i], lds0 + slot_at + (uint32_t)j * 1024u);
                else if (j < n_all) load16_to_lds(xb, off[i], lds0 + slot_at + x_area + (uint32_t)(j - n_g) * 1024u);
            }
            gb += kRowBytes;
            xb += XB;
            slot_at = slot_at + stage_bytes == (uint32_t)ring * stage_bytes ? 0u : slot_at + stage_bytes;
        };
        const int ahead = min(ring - 1, stages);
        for (int k = 0; k < ahead; ++k) issue();
        for (int s = 0; s < stages; ++s) {
            wait_vmcnt_at_most((min(s + ring - 1, stages) - (s + 1)) * mine_loads);
            asm volatile("s_barrier" ::: "memory");
            if (s + ring - 1 < stages) issue();
        }
    } else {
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
            const uint32_t o = t < mine ? a.ops[(int64_t)(first + my0 + t) * 16 + n] : (uint32_t)g_slots << 16;
            const uint32_t gr = o & 0xffffu, xr = (o >> 16) - (uint32_t)g_slots;
            const uint32_t xu = XB == 64 ? 16u * unit_of(xr, (uint32_t)g)
                              : XB == 32 ? 32u * xr + 16u * ((uint32_t)(g >> 1) ^ ((xr >> 3) & 1u)) + 8u * (g & 1) : 16u * xr + 4u * g;
            ops[t] = 16u * unit_of(gr, (uint32_t)g) | (x_area + xu) << 16;
            if constexpr (CKPT) exps[t] = (uint32_t)rows[g_slots + xr] * (uint32_t)a.lds;
        }
        uint32_t now[TILES], next[TILES];
        const uint8_t *sb = a.S + (((int64_t)s0 * STAGE) >> 5);
        auto fetch = [&]() {
            if constexpr (CKPT) {
#pragma unroll
                for (int t = 0; t < TILES; ++t) __builtin_memcpy(&next[t], sb + exps[t], 4);
            }
        };
        if (stages > 0) fetch();
        uint32_t at = 0;
        for (int s = 0; s < stages; ++s) {
            if (CKPT && s % SPB == 0) {
#pragma unroll
                for (int t = 0; t < TILES; ++t) now[t] = next[t];
                if (s + SPB < stages) sb += 4;
                fetch();                          // (behind the last block: it again)
            }
            lds_barrier();
            multiply(at, now, (s % SPB) * STAGE / 32 * 8);
            at = at + stage_bytes == (uint32_t)ring * stage_bytes ? 0u : at + stage_bytes;
        }
    }
    // ---- the tokens behind the last block
    if (last) {
        for (int n0 = a.N / kBlock * kBlock; n0 < a.N; n0 += STAGE) {
            __syncthreads();
            for (int p = threadIdx.x; p < (g_slots + (CKPT ? 0 : x_slots)) * 4; p += kStreamThreads) {
                const int slot = p >> 2, q = p & 3;
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
                const uint32_t to = in_g ? 16u * unit_of((uint32_t)slot, (uint32_t)q) : x_area + 16u * unit_of((uint32_t)(slot - g_slots), (uint32_t)q);
                *reinterpret_cast<uint4v *>(smem + to) = o;
            }
            if constexpr (CKPT)
                for (int p = threadIdx.x; p < x_slots * (XB / 16); p += kStreamThreads) {
                    const int slot = p / (XB / 16);
                    uint32_t q = (uint32_t)(p % (XB / 16));
                    const int col = n0 + (int)q * 16;
                    const uint8_t *src = static_cast<const uint8_t *>(a.X) + (int64_t)rows[g_slots + slot] * a.ldx;
                    uint4v codes = {0u, 0u, 0u, 0u};
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (col + e < a.N) codes[e / 4] |= (uint32_t)src[col + e] << (8 * (e & 3));
                    if constexpr (XB == 32) q ^= (uint32_t)((slot >> 3) & 1);
                    *reinterpret_cast<uint4v *>(smem + x_area + (uint32_t)slot * XB + 16u * q) = codes;
                }
            __syncthreads();
            if (wave < kGradWaves) {
                uint32_t words[TILES];
#pragma unroll
                for (int t = 0; t < TILES; ++t) words[t] = CKPT ? a.S[exps[t] + (uint32_t)(n0 >> 5)] : 0u;
                multiply(0u, words, 0);
            }
        }
    }
    if (wave >= kGradWaves) return;

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

template <typename T, bool CKPT, int SHAPE> ubp_status launch_one(const GradArgs &a, bool stream, hipStream_t st, bool dry) {
    constexpr GradShape S = kGradShapes[SHAPE];
    constexpr auto general = &weight_grad_kernel<T, CKPT, S.tiles, S.g_slots, S.x_slots>;
    constexpr auto streamed = &weight_grad_stream_kernel<T, CKPT, S.tiles>;
    static LdsLimit limits[2];
    ubp_status rc = limits[0].raise(reinterpret_cast<const void *>(general));
    if (rc == UBP_OK) rc = limits[1].raise(reinterpret_cast<const void *>(streamed));
    if (rc != UBP_OK || dry) return rc;
    const int64_t grid = 8 * (((int64_t)a.n_regions * a.splits + 7) / 8);
    if (grid * kStreamThreads >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED; // (a launch's threads are counted in 32 bits)
    if (!stream) return launch_kernel(general, dim3((unsigned)grid), dim3(kThreads), (size_t)2 * a.slots * kRowBytes, st, a);
    GradArgs b = a;
    const int x_bytes = !CKPT ? a.slots_x * kRowBytes : ((a.slots_x + 63) / 64 * 64) * (64 / (int)sizeof(T));
    b.stage_bytes = a.slots_g * kRowBytes + x_bytes;
    b.ring = std::min(kGradMaxRing, 160 * 1024 / b.stage_bytes);
    return launch_kernel(streamed, dim3((unsigned)grid), dim3(kStreamThreads), (size_t)b.ring * b.stage_bytes, st, b);
}

template <typename T, bool CKPT> ubp_status launch_t(const GradArgs &a, int shape, bool stream, hipStream_t st, bool dry) {
    static_assert(kNumGradShapes == 3, "their instantiations");
    switch (shape) {
    case 0: return launch_one<T, CKPT, 0>(a, stream, st, dry);
    case 1: return launch_one<T, CKPT, 1>(a, stream, st, dry);
    case 2: return launch_one<T, CKPT, 2>(a, stream, st, dry);
    }
    return UBP_ERR_UNSUPPORTED;
}

} // namespace

bool weight_grad_streams(const GradArgs &a, ubp_dtype dtype, bool checkpoint) {
    const int64_t size = dtype_size(dtype), x_size = checkpoint ? 1 : size;
    const int64_t rows_g = (int64_t)a.M * a.ldg * size, rows_x = (int64_t)a.K * a.ldx * x_size;
    return a.blocks > 0 && reinterpret_cast<uintptr_t>(a.G) % 16 == 0 && reinterpret_cast<uintptr_t>(a.X) % 16 == 0 && a.ldg * size % 16 == 0 &&
           a.ldx * x_size % 16 == 0 && std::max({a.ldg, a.ldx, a.lds}) < (int64_t(1) << 31) && rows_g < (int64_t(1) << 32) &&
           rows_x < (int64_t(1) << 32) && (int64_t)a.K * a.lds < (int64_t(1) << 32);
}

ubp_status launch_weight_grad(const GradArgs &a, ubp_dtype dtype, bool checkpoint, int shape, void *stream, bool dry) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    GradArgs b = a;
    const bool streams = !dry && weight_grad_streams(a, dtype, checkpoint);
    // a range in tokens -> in steps, of 64 bytes of a row of the layer's type
    b.per_split = a.per_split / (64 / (int)dtype_size(dtype));
    switch (dtype) {
    case UBP_F32: return checkpoint ? launch_t<float, true>(b, shape, streams, st, dry) : launch_t<float, false>(b, shape, streams, st, dry);
    case UBP_F16: return checkpoint ? launch_t<_Float16, true>(b, shape, streams, st, dry) : launch_t<_Float16, false>(b, shape, streams, st, dry);
    case UBP_BF16: return checkpoint ? launch_t<__bf16, true>(b, shape, streams, st, dry) : launch_t<__bf16, false>(b, shape, streams, st, dry);
    }
    return UBP_ERR_INVALID_ARG;
}

ubp_status launch_weight_sum(const GradArgs &a, void *stream) {
    const int64_t grid = (a.n_tiles * 64 + 255) / 256;
    if (grid * 256 >= (int64_t(1) << 32)) return UBP_ERR_UNSUPPORTED;
    return launch_kernel(&weight_sum_kernel, dim3((unsigned)grid), dim3(256), 0, static_cast<hipStream_t>(stream), a);
}

} // namespace ubp
