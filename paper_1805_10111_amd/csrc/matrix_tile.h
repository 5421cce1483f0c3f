// One tile of a matrix product on the matrix cores, the part that all products of many-class models share.
//
//   out[i][j] = sum_k x(i, k) y(j, k),   i = XT rows of x, j = YT rows of y
//
// A thread ends up with four neighbouring i (the rows of an output element are 4 (lane / 16) + 0..3) of one j (lane % 16) per 16 x 16
// subtile: x is given the index along which the result is stored, or summed up, contiguously.
//
// Either operand is stored along k (row-major rows i, k contiguous), or across it (row-major rows k, i contiguous); the latter
// reaches the matrix cores through the transposing reads of LDS, so nothing is ever transposed in memory.
// A stage is 128 bytes of k: 64 numbers of 16 bits, 256 of 4.  Two stages of both operands lie in LDS, filled by loads that go there
// directly; while one is multiplied the other is on its way.
//
// What bounds it: the matrix cores.  256 x 256 with eight wavefronts (a wavefront multiplies 128 x 64: 12 reads of LDS for 32
// products) needs 96 KB of LDS reads per 1024 cycles of matrix-core work, and each byte of memory is used for 256 products.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "dq_common.h"

namespace dq {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr int kStageBytes = 128;               // of k, per row of an operand stored along k
constexpr int kStageRows = 64;                 // of k, for an operand stored across it (16-bit numbers)

// An operand in memory.  Its row i (row k where it is stored across k) begins at p + i * ld bytes; rows is how many there are:
// reads past the last are turned to the last, whose products the caller drops (i) or meets with zeros of the other operand (k).
struct Operand {
    const char *p;
    int64_t ld;            // bytes, a multiple of 16
    int64_t rows;
    int32_t cols;          // stored across k: how many i there are (a multiple of 8); unused otherwise
    int64_t plane;         // bytes from one part of a number to the next (float32 as three bfloat16), 0 otherwise
    const uint8_t *scales; // 4-bit numbers: four scales per 64 bytes of a row, from row to row ld_scales bytes
    int64_t ld_scales;
};

// float32 numbers are carried as three bfloat16 (24 bits of significand between them): x y = the products of the parts whose
// exponents add up to at least that of the last bit, six of nine, smallest first.  Two bits per step: which part of x, of y.
constexpr int kPartSteps = 6;
constexpr uint32_t kPartsX = 2u | 0u << 2 | 1u << 4 | 1u << 6 | 0u << 8 | 0u << 10;
constexpr uint32_t kPartsY = 0u | 2u << 2 | 1u << 4 | 0u << 6 | 1u << 8 | 0u << 10;

struct MulBf16 {
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ f32x4 mul(i32x4 x, i32x4 y, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    }
};
struct MulF16 {
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ f32x4 mul(i32x4 x, i32x4 y, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    }
};

// 128 numbers of 4 bits: a lane holds 32 of them, one block, and the low byte of sx, sy is that block's scale.
struct MulMx4 {
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ f32x4 mul(i32x4 x, i32x4 y, f32x4 c, uint32_t sx, uint32_t sy)
    {
        const i32x8 a{x[0], x[1], x[2], x[3], 0, 0, 0, 0}, b{y[0], y[1], y[2], y[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, static_cast<int>(sx), 0, static_cast<int>(sy));
    }
};

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;
typedef __attribute__((address_space(3))) i16x4 *LdsQuad;

__device__ __forceinline__ void load_to_lds(const char *from, char *to)
{
    __builtin_amdgcn_global_load_lds((GlobalPtr)from, (LdsPtr)to, 16, 0, 0);
}

// The stage that is on its way has arrived, in every wavefront, and every wavefront is done with the one before.
__device__ __forceinline__ void stage_arrived()
{
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    __syncthreads();
}

// The loads of one operand's stages.  ACROSS: stored across k.
// LDS holds a stage as it lies in memory, its 16-byte chunks permuted within a row so that no two of the lanes that read together
// meet a bank: along k, chunk c of row r at c ^ (r / 2) % 8 (16 lanes read 16 rows of 128 bytes); across k, 32 bytes at a time,
// pair c of row k at c ^ (k % 4 + 4 (k / 8 % 2)) (32 lanes read rows k .. k + 3 and k + 8 .. k + 11).
template <int T, bool ACROSS, int THREADS>
struct StageLoads {
    static constexpr int kChunks = (T * 8 + THREADS - 1) / THREADS;
    static constexpr int kRowChunks = ACROSS ? T / 8 : 8;
    static constexpr int kPairMask = T / 16 >= 8 ? 7 : T / 16 - 1;
    uint32_t off[kChunks];
    int64_t ld;

    __device__ __forceinline__ void init(const Operand &o, int64_t i0)
    {
        ld = o.ld;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int id = threadIdx.x + i * THREADS, row = id / kRowChunks, slot = id % kRowChunks;
            if constexpr (ACROSS) {
                const int pair = (slot >> 1) ^ (((row & 3) | ((row >> 1) & 4)) & kPairMask);
                const int col = min(static_cast<int>(i0) + (pair * 2 + (slot & 1)) * 8, o.cols - 8);
                off[i] = static_cast<uint32_t>(col) * 2u;
            } else {
                const int64_t r = i0 + row < o.rows ? row : o.rows - 1 - i0;
                off[i] = static_cast<uint32_t>(r * o.ld) + static_cast<uint32_t>(slot ^ ((row >> 1) & 7)) * 16u;
            }
        }
    }
    // base: where the stage's k begins (row k0, or byte k0 of row i0).  left: how much of k there is from there on (rows, or bytes; a
    // multiple of 64 bytes).
    __device__ __forceinline__ void issue(const char *base, int64_t left, char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int id = threadIdx.x + i * THREADS, first = id & ~(kWave - 1);
            if (kChunks * THREADS > T * 8 && first >= T * 8) break;
            uint32_t at = off[i];
            if constexpr (ACROSS) {
                const int row = id / kRowChunks;
                at += static_cast<uint32_t>(left < kStageRows ? min(row, static_cast<int>(left) - 1) : row) * static_cast<uint32_t>(ld);
            } else if (left < kStageBytes) {
                const int row = id / 8, chunk = (id % 8) ^ ((row >> 1) & 7);
                at -= static_cast<uint32_t>(chunk & 4) * 16u;
            }
            load_to_lds(base + at, lds + first * 16);
        }
    }
};

// What a lane reads from a stage for subtile `sub` and 32 numbers of k.
template <int T, bool ACROSS>
__device__ __forceinline__ i32x4 stage_part(const char *lds, int sub, int half)
{
    const int lane = threadIdx.x & (kWave - 1), j = lane & 15, g = lane >> 4;
    if constexpr (ACROSS) {
        constexpr int mask = T / 16 >= 8 ? 7 : T / 16 - 1;
        const int f = ((j >> 2) | ((g & 1) << 2)) & mask;
        const char *at = lds + (half * 32 + g * 8 + (j >> 2)) * (T * 2) + ((sub ^ f) * 32) + (j & 3) * 8;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)at);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(at + 4 * T * 2));
        return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        return *reinterpret_cast<const i32x4 *>(lds + (sub * 16 + j) * kStageBytes + (((half * 4 + g) ^ (j >> 1)) * 16));
    }
}

// WX x WY wavefronts share the tile.  Each of them multiplies SX x SY subtiles.
template <class Mul, int XT, int YT, int WX, int WY, bool XS, bool YS>
struct TileProduct {
    static constexpr int kThreads = WX * WY * kWave;
    static constexpr int SX = XT / 16 / WX, SY = YT / 16 / WY;
    f32x4 acc[SX][SY];

    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    static __device__ __forceinline__ int sub_x(int m) { return (wave() % WX) * SX + m; }
    static __device__ __forceinline__ int sub_y(int n) { return (wave() / WX) * SY + n; }
    // index within the tile of a lane's four results of subtile (m, n)
    static __device__ __forceinline__ int at_x(int m) { return sub_x(m) * 16 + ((threadIdx.x & 63) >> 4) * 4; }
    static __device__ __forceinline__ int at_y(int n) { return sub_y(n) * 16 + (threadIdx.x & 15); }

    // The scales of a stage's blocks: of both halves, a lane's own block's in the low byte.
    struct Scales {
        uint32_t x[2][Mul::kScaled ? SX : 1], y[2][Mul::kScaled ? SY : 1];
    };
    template <int S>
    static __device__ __forceinline__ void load_scales(const Operand &o, int64_t row0, int64_t group, int64_t groups, uint32_t (&out)[2][S])
    {
#pragma unroll
        for (int m = 0; m < S; ++m) {
            const uint8_t *const row = o.scales + min(row0 + m * 16 + (threadIdx.x & 15), o.rows - 1) * o.ld_scales;
            out[0][m] = *reinterpret_cast<const uint32_t *>(row + group * 4);
            out[1][m] = *reinterpret_cast<const uint32_t *>(row + min(group + 1, groups - 1) * 4);
        }
    }

    __device__ __forceinline__ void multiply(const char *xs, const char *ys, int halves, const Scales &scales)
    {
        const int mine = ((threadIdx.x & 63) >> 4) * 8;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half && halves < 2) break;
            i32x4 y[SY];
#pragma unroll
            for (int n = 0; n < SY; ++n) y[n] = stage_part<YT, YS>(ys, sub_y(n), half);
#pragma unroll
            for (int m = 0; m < SX; ++m) {
                const i32x4 x = stage_part<XT, XS>(xs, sub_x(m), half);
#pragma unroll
                for (int n = 0; n < SY; ++n) {
                    if constexpr (Mul::kScaled) acc[m][n] = Mul::mul(x, y[n], acc[m][n], scales.x[half][m] >> mine, scales.y[half][n] >> mine);
                    else acc[m][n] = Mul::mul(x, y[n], acc[m][n]);
                }
            }
        }
    }

    // k0 .. k1 (in pairs of bytes, k0 a multiple of 64, k1 of 32) of rows i0.. of x and j0.. of y.  steps: 1, or kPartSteps for parts.
    __device__ __forceinline__ void run(const Operand &x, const Operand &y, int64_t i0, int64_t j0, int64_t k0, int64_t k1, int steps)
    {
        __shared__ __attribute__((aligned(1024))) char xs0[XT * kStageBytes], xs1[XT * kStageBytes];
        __shared__ __attribute__((aligned(1024))) char ys0[YT * kStageBytes], ys1[YT * kStageBytes];
        StageLoads<XT, XS, kThreads> lx;
        StageLoads<YT, YS, kThreads> ly;
        lx.init(x, i0);
        ly.init(y, j0);
#pragma unroll
        for (int m = 0; m < SX; ++m)
#pragma unroll
            for (int n = 0; n < SY; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        const char *const px = x.p + (XS ? k0 * x.ld : i0 * x.ld + k0 * 2), *const py = y.p + (YS ? k0 * y.ld : j0 * y.ld + k0 * 2);
        const int per = static_cast<int>((k1 - k0 + 63) / 64), stages = per * steps;
        const int64_t dx = XS ? kStageRows * x.ld : kStageBytes, dy = YS ? kStageRows * y.ld : kStageBytes;
        int at = 0, part = 0;                   // the next stage to be loaded: stage `at` of part product `part`
        const char *nx = px + (steps > 1 ? (kPartsX & 3) * x.plane : 0), *ny = py + (steps > 1 ? (kPartsY & 3) * y.plane : 0);
        auto load = [&](char *xs, char *ys, Scales &scales) {
            const int64_t k = k0 + static_cast<int64_t>(at) * 64;
            if constexpr (Mul::kScaled) {
                load_scales(x, i0 + sub_x(0) * 16, k / 32, k1 / 32, scales.x);
                load_scales(y, j0 + sub_y(0) * 16, k / 32, k1 / 32, scales.y);
            }
            lx.issue(nx, XS ? x.rows - k : (k1 - k) * 2, xs);
            ly.issue(ny, YS ? y.rows - k : (k1 - k) * 2, ys);
            nx += dx;
            ny += dy;
            if (++at == per) {
                at = 0;
                ++part;
                nx = px + ((kPartsX >> (2 * part)) & 3) * x.plane;
                ny = py + ((kPartsY >> (2 * part)) & 3) * y.plane;
            }
        };
        const int last = (k1 - k0) % 64 ? 1 : 2;      // halves of the last stage of a part product
        int done = 0;
        auto halves = [&] { return ++done == per ? (done = 0, last) : 2; };
        Scales s0, s1;
        if (stages) load(xs0, ys0, s0);
        stage_arrived();
        for (int s = 0; s < stages; s += 2) {
            if (s + 1 < stages) load(xs1, ys1, s1);
            multiply(xs0, ys0, halves(), s0);
            stage_arrived();
            if (s + 1 >= stages) break;
            if (s + 2 < stages) load(xs0, ys0, s0);
            multiply(xs1, ys1, halves(), s1);
            stage_arrived();
        }
    }
};

typedef unsigned short u16;
typedef __attribute__((ext_vector_type(4))) unsigned short u16x4;

// ---- numbers of the three types ------------------------------------------------
template <int TYPE>
struct Num;
template <>
struct Num<DQ_F32> {
    typedef float Mem;
    typedef MulBf16 Mul;                         // of its parts
    static __device__ __forceinline__ float load(Mem v) { return v; }
    static __device__ __forceinline__ Mem store(float v) { return v; }
};
template <>
struct Num<DQ_F16> {
    typedef u16 Mem;
    typedef MulF16 Mul;
    static __device__ __forceinline__ float load(Mem v) { return static_cast<float>(__builtin_bit_cast(_Float16, v)); }
    static __device__ __forceinline__ Mem store(float v) { return __builtin_bit_cast(u16, static_cast<_Float16>(v)); }
};
template <>
struct Num<DQ_BF16> {
    typedef u16 Mem;
    typedef MulBf16 Mul;
    static __device__ __forceinline__ float load(Mem v) { return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16); }
    static __device__ __forceinline__ Mem store(float v) { return __builtin_bit_cast(u16, static_cast<__bf16>(v)); }
};
typedef Num<DQ_BF16> Part;                       // of a float32

// Four neighbouring results of one row.
template <int TYPE>
__device__ __forceinline__ void store_four(typename Num<TYPE>::Mem *to, f32x4 v, int have, bool vector)
{
    typedef typename Num<TYPE>::Mem Mem;
    typedef __attribute__((ext_vector_type(4))) Mem Quad;
    Mem r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = Num<TYPE>::store(v[i]);
    if (vector && have >= 4) {
        *reinterpret_cast<Quad *>(to) = Quad{r[0], r[1], r[2], r[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) to[i] = r[i];
    }
}

// vector stores of four results where every row allows them
static bool four_at_once(const void *p, int64_t ld, int wide) { return reinterpret_cast<uintptr_t>(p) % (4 * wide) == 0 && ld % 4 == 0; }

// Which tile a block takes: the blocks of a die (every eighth) take neighbouring tiles, in groups of kGroup rows of y tiles, so that
// those at work at one time share both operands in the die's 4 MB of L2.
__device__ __forceinline__ void tile_of_block(int block, int tiles_x, int tiles_y, int &tx, int &ty)
{
    constexpr int kXcds = 8, kGroup = 8;
    const int total = tiles_x * tiles_y, each = total / kXcds, more = total % kXcds, xcd = block % kXcds;
    const int t = xcd * each + min(xcd, more) + block / kXcds;
    const int span = kGroup * tiles_x, group = t / span, first = group * kGroup, high = min(kGroup, tiles_y - first), in = t % span;
    ty = first + in % high;
    tx = in / high;
}

}  // namespace dq
