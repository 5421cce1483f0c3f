// One tile of a matrix product on the matrix cores, the part that all products of many-class models share.
//
//   out[i][j] = sum_k x(i, k) y(j, k),   i = XT rows of x, j = YT rows of y
//
// A thread ends up with four neighbouring i (the rows of an output element are 4 (lane / 16) + 0..3) of one j (lane % 16) per 16 x 16
// subtile: x is given the index along which the result is stored, or summed up, contiguously.
//
// Either operand is stored along k (row-major rows i, k contiguous), or across it (row-major rows k, i contiguous); the latter
// reaches the matrix cores through the transposing reads of LDS, so nothing is ever transposed in memory.
// A step is 64 bytes of k: 32 numbers of 16 bits, 128 of 4; a stage is H steps.  LDS holds a ring of two to four stages, filled by loads
// that go there directly: while one is multiplied, the others are on their way.  One step is right where the matrix cores bound
// (large tiles, short stages); where memory does (few rows), rows are read 128 bytes at a time.
//
// What bounds it: the matrix cores.  256 x 256 with eight wavefronts (a wavefront multiplies 128 x 64: 12 reads of LDS for 32
// products) needs 96 KB of LDS reads per 1024 cycles of matrix-core work, which LDS does in 400, and each byte of memory is used for
// 256 products.  A step takes 1.3 times the 1024 cycles; at 1.7 to 1.8 GHz, which is what the clocks are held to under this
// load, that is 1440 to 1475 TFLOP/s in bfloat16 (n = 8192 rows of 47236 classes times 4096 columns, where a tile is 1476 steps).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "dq_common.h"
#include "launch_sizes.h"

namespace dq {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr int kStepBytes = 64;                 // of k in a product of the matrix cores, per row of an operand stored along k
constexpr int kStepRows = 32;                  // of k, for an operand stored across it (16-bit numbers)

// An operand in memory.  Its row i (row k where it is stored across k) begins at p + i * ld bytes; rows is how many there are.
// Nothing outside of it matters: rows past the last are zeros, and k past its end.
struct Operand {
    const char *p;
    int64_t ld;            // bytes, a multiple of 16
    int64_t rows;
    int32_t cols;          // numbers of a row (pairs of bytes), a multiple of 8.  Along k those behind them are zeros, whatever lies there
    int64_t plane;         // bytes from one part of a number to the next (float32 as three bfloat16), 0 otherwise
    const uint8_t *scales; // 4-bit numbers: four scales per 64 bytes of a row, from row to row ld_scales bytes
    int64_t ld_scales;
};

// float32 numbers are carried as three bfloat16 (24 bits of significand between them): x y = the products of the parts whose
// exponents add up to at least that of the last bit, six of nine, smallest first: which part of x, of y.  All parts of a stage lie in
// LDS together, so that each is brought there once for the products it has a share in.
constexpr int kPartProducts = 6;
constexpr int kPartsX[kPartProducts] = {2, 0, 1, 1, 0, 0}, kPartsY[kPartProducts] = {0, 2, 1, 0, 1, 0};

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

// 128 numbers of 4 bits: a lane holds 32 of them, one block; byte m of sx, n of sy is that block's scale.
struct MulMx4 {
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ f32x4 mul(i32x4 x, i32x4 y, f32x4 c, int sx, int m, int sy, int n)
    {
        const i32x8 a{x[0], x[1], x[2], x[3], 0, 0, 0, 0}, b{y[0], y[1], y[2], y[3], 0, 0, 0, 0};
#define DQ_MX4(M, N) case M * 4 + N: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, M, sx, N, sy)
        switch (m * 4 + n) {                   // (which byte is part of the instruction: m and n are known when it is compiled)
            DQ_MX4(0, 0); DQ_MX4(0, 1); DQ_MX4(0, 2); DQ_MX4(0, 3); DQ_MX4(1, 0); DQ_MX4(1, 1); DQ_MX4(1, 2); DQ_MX4(1, 3);
            DQ_MX4(2, 0); DQ_MX4(2, 1); DQ_MX4(2, 2); DQ_MX4(2, 3); DQ_MX4(3, 0); DQ_MX4(3, 1); DQ_MX4(3, 2); DQ_MX4(3, 3);
        }
#undef DQ_MX4
        return c;
    }
};

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef __attribute__((address_space(3))) i16x4 *LdsQuad;

__device__ __forceinline__ int64_t lesser(int64_t a, int64_t b) { return a < b ? a : b; }      // (min() goes through doubles)

// All but the newest NEWER loads of this wavefront have arrived, in every wavefront, and every wavefront has read what it wanted of
// LDS.  (__syncthreads() would wait for all loads.)
template <int NEWER>
__device__ __forceinline__ void stage_arrived()
{
    static_assert(NEWER < 64, "six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (NEWER & 15) | (NEWER >> 4) << 14);      // vmcnt(NEWER), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The loads of one operand's stages.  ACROSS: stored across k.
// LDS holds a stage as it lies in memory, its 16-byte chunks permuted within a row so that no two of the lanes that read together
// meet a bank: along k, chunk c of row r at c ^ chunk_swap(r); across k, 32 bytes at a time, pair c of row k at c ^ (k % 4 +
// 4 (k / 8 % 2)) (32 lanes read rows k .. k + 3 and k + 8 .. k + 11).
//
// 16-byte reads go by sixteen lanes, which are 0 to 3, 12 to 15 and 20 to 27, and the others of 32 (measured: which lanes of a read take
// longer if they meet in one of 64 banks).  Lane 16 g + j reads chunk g of row j; so in a group chunks of one number come from rows 0 to 3
// and 12 to 15, those of the next from rows 4 to 11.  (With chunk c at c ^ (r H / 4), as if sixteen neighbours read together,
// half of the LDS's cycles were conflicts.)
template <int H>
__device__ __forceinline__ int chunk_swap(int row)
{
    return H == 1 ? (row >> 2) & 2 : (row & 2) | ((row >> 1) & 4);
}
// EDGE: rows may end inside of a step (which costs a comparison a load: 2% of a large product).
template <int T, bool ACROSS, int THREADS, int H, bool EDGE>
struct StageLoads {
    static constexpr int kAll = T * 4 * H;                                       // 16-byte chunks of a stage
    static constexpr int kChunks = (kAll + THREADS - 1) / THREADS;               // loads of a thread per stage
    static constexpr int kSurely = kAll / THREADS;                               // ... of any thread
    static constexpr int kRowChunks = ACROSS ? T / 8 : 4 * H;
    static constexpr int kPairMask = T / 16 >= 8 ? 7 : T / 16 - 1;
    uint32_t off[kChunks];

    // The loads of `planes` parts of numbers are asked for in slices; how many of any thread are in the first.
    static constexpr int slice_of(int plane, int i, int planes, int slices) { return (plane * kChunks + i) * slices / (planes * kChunks); }
    static constexpr int first(int planes, int slices)
    {
        int n = 0;
        for (int p = 0; p < planes; ++p)
            for (int i = 0; i < kSurely; ++i) n += slice_of(p, i, planes, slices) == 0;
        return n;
    }

    __device__ __forceinline__ void init(const Operand &o)
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int id = threadIdx.x + i * THREADS, row = id / kRowChunks, slot = id % kRowChunks;
            int at;
            if constexpr (ACROSS) at = (((slot >> 1) ^ (((row & 3) | ((row >> 1) & 4)) & kPairMask)) * 2 + (slot & 1)) * 16;
            else at = (slot ^ chunk_swap<H>(row)) * 16;
            off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(o.ld) + static_cast<uint32_t>(at);
        }
    }
    // Those of a plane that are in this slice; to: where this wavefront's first one goes.  wide: bytes of k there are yet; a stage may end
    // behind them, and what lies there (the next row, or what a wider matrix holds between the rows) is not read but zeros are.
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t from, char *ring, int to, int plane, int planes, int slice, int slices, int wide) const
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            if (slice_of(plane, i, planes, slices) != slice) continue;
            if (kChunks != kSurely && static_cast<int>(threadIdx.x) + i * THREADS >= kAll) continue;      // (whole wavefronts)
            uint32_t at = off[i];
            if constexpr (!ACROSS && (H > 1 || EDGE)) {
                const int id = threadIdx.x + i * THREADS, row = id / kRowChunks;
                if (((id % kRowChunks) ^ chunk_swap<H>(row)) * 16 >= wide) at = 0x7fffffff;      // behind every buffer
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (LdsPtr)(ring + (to + i * THREADS * 16)), 16, static_cast<int>(at), 0, 0, 0);
        }
    }
};

// Where an operand's next stage lies: a buffer, behind whose end everything reads as zero.  (Loads to LDS go through buffers also
// because the compiler takes those through plain pointers for possible accesses to LDS by address, and then waits for all reads of
// LDS at every use of one.)  Moving on takes a few scalar instructions.
template <int T, bool ACROSS, int H>
struct Reader {
    const char *p;
    int32_t left;                        // across k: rows from here on; along k: bytes from here to the end of the tile's last row
    int32_t ld, edge;                    // across k: bytes of a row, and by how much the last one is shorter
    __device__ __forceinline__ Reader(const Operand &o, int64_t i0, int64_t k0)
    {
        ld = static_cast<int32_t>(o.ld);
        if constexpr (ACROSS) {
            p = o.p + k0 * o.ld + i0 * 2;
            left = static_cast<int32_t>(o.rows - k0);
            edge = static_cast<int32_t>(2 * (o.cols - i0) - o.ld);
        } else {
            p = o.p + i0 * o.ld + k0 * 2;
            left = static_cast<int32_t>((lesser(o.rows - i0, T) - 1) * o.ld + 2 * (o.cols - k0));
            edge = 0;
        }
        // (the same in every lane, which the compiler does not see everywhere: it would go through the lanes in a loop at each load)
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        p = reinterpret_cast<const char *>(static_cast<uint64_t>(same(static_cast<int>(at >> 32))) << 32 | static_cast<uint32_t>(same(static_cast<int>(at))));
        left = same(left);
        ld = same(ld);
        edge = same(edge);
    }
    static __device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }
    // any: whether there is another stage.  plane: bytes further on.
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(bool any, int64_t plane) const
    {
        const int32_t bytes = max(ACROSS ? min(left, kStepRows * H) * ld + edge : left, 0);
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p + plane), 0, any ? bytes : 0, 0x00027000);
    }
    __device__ __forceinline__ void next()
    {
        p += ACROSS ? static_cast<int64_t>(kStepRows * H) * ld : kStepBytes * H;
        left -= ACROSS ? kStepRows * H : kStepBytes * H;
    }
};

// Where in an operand's part of a stage a lane reads of subtile 0 of those of its wavefront (subtiles first ..).
template <int T, bool ACROSS, int H>
__device__ __forceinline__ int part_address(int first)
{
    const int lane = threadIdx.x & (kWave - 1), j = lane & 15, g = lane >> 4;
    if constexpr (ACROSS) {
        constexpr int mask = T / 16 >= 8 ? 7 : T / 16 - 1;
        return (g * 8 + (j >> 2)) * (T * 2) + ((first ^ (((j >> 2) | ((g & 1) << 2)) & mask)) * 32) + (j & 3) * 8;
    } else {
        return (first * 16 + j) * kStepBytes * H + ((g ^ chunk_swap<H>(j)) * 16);
    }
}
// ... and what it reads of step `half` and subtile m of them (there are a power of two of them, their first a multiple of it).  An operand's part of the
// ring begins `from` in.  (One addition to the array: the compiler follows an address to its array through a few additions only.)
template <int T, bool ACROSS, int H>
__device__ __forceinline__ i32x4 stage_part(const char *ring, int from, int address, int half, int m)
{
    if constexpr (ACROSS) {
        const int at = address ^ (m * 32);
        from += half * kStepRows * T * 2;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(ring + (from + at)));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(ring + (from + 4 * T * 2 + at)));
        return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        return *reinterpret_cast<const i32x4 *>(ring + (from + m * 16 * kStepBytes * H + (address ^ (half * kStepBytes))));
    }
}

// WX x WY wavefronts share the tile.  Each of them multiplies SX x SY subtiles.
// H steps a stage, R stages in the ring (an even number), P parts of a number.
template <class Mul, int XT, int YT, int WX, int WY, bool XS, bool YS, int H, int R, int P, bool EDGE = false>
struct TileProduct {
    static constexpr int kThreads = WX * WY * kWave;
    static constexpr int SX = XT / 16 / WX, SY = YT / 16 / WY;
    f32x4 acc[SX][SY];
    int address_x, address_y;

    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    static __device__ __forceinline__ int sub_x(int m) { return (wave() % WX) * SX + m; }
    static __device__ __forceinline__ int sub_y(int n) { return (wave() / WX) * SY + n; }
    // index within the tile of a lane's four results of subtile (m, n)
    static __device__ __forceinline__ int at_x(int m) { return sub_x(m) * 16 + ((threadIdx.x & 63) >> 4) * 4; }
    static __device__ __forceinline__ int at_y(int n) { return sub_y(n) * 16 + (threadIdx.x & 15); }

    // Scales of 4-bit numbers.  A step has four blocks a row; LDS holds their scales as [block][row % 16][row / 16], so that what a
    // lane needs for its subtiles are neighbouring bytes.  Thread r brings those of row r (x's rows, then y's): where a stage is one step,
    // of four stages at a time, 16 bytes (each thread's row is a line of its own in the cache, and a line a stage took as long as the codes).
    static constexpr int kScaleBytes = 4 * (XT + YT);       // of a step
    static_assert(!Mul::kScaled || XT + YT <= kThreads, "a thread brings one row's scales");
    struct Scales {
        uint32_t x[H][(SX + 3) / 4], y[H][(SY + 3) / 4];
    };
    struct Brought {
        uint32_t v[H];
    };
    template <int S, int T>
    static __device__ __forceinline__ void read_scales(const uint8_t *lds, int sub, uint32_t (&out)[(S + 3) / 4])
    {
        const int lane = threadIdx.x & 63;
        const uint8_t *const at = lds + (lane >> 4) * T + (lane & 15) * (T / 16) + sub;
#pragma unroll
        for (int i = 0; i < (S + 3) / 4; ++i)
            out[i] = S >= 4 ? reinterpret_cast<const uint32_t *>(at)[i] : S == 2 ? *reinterpret_cast<const uint16_t *>(at) : *at;
    }
    static __device__ __forceinline__ void read_scales(const uint8_t *lds, Scales &s)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            read_scales<SX, XT>(lds + h * kScaleBytes, sub_x(0), s.x[h]);
            read_scales<SY, YT>(lds + h * kScaleBytes + 4 * XT, sub_y(0), s.y[h]);
        }
    }
    static __device__ __forceinline__ Brought load_scales(const uint8_t *row, int64_t stage, int64_t groups)
    {
        Brought b;
#pragma unroll
        for (int h = 0; h < H; ++h) b.v[h] = row ? *reinterpret_cast<const uint32_t *>(row + lesser(stage * H + h, groups - 1) * 4) : 0;
        return b;
    }
    // Those of stages `stage` to stage + 3, or of the row's last four.
    static __device__ __forceinline__ i32x4 load_four(const uint8_t *row, int stage, int groups)
    {
        struct __attribute__((packed, aligned(4))) Four {
            i32x4 v;
        };
        return reinterpret_cast<const Four *>(row + max(min(stage, groups - 4), 0) * 4)->v;
    }
    // Stage s + i's of those of stage s on (behind the last, where codes are zeros: any).
    static __device__ __forceinline__ Brought one_of(const i32x4 &four, int s, int i, int groups)
    {
        const int past = s - (groups - 4);                       // stages of the row's last four that came before s
        uint32_t v = static_cast<uint32_t>(four[i]);
#pragma unroll
        for (int by = 1; by + i < 4; ++by) v = past == by ? static_cast<uint32_t>(four[i + by]) : v;
        Brought b{};
        b.v[0] = v;
        return b;
    }
    static __device__ __forceinline__ void write_scales(uint8_t *lds, const Brought &b)
    {
        const bool in_x = threadIdx.x < XT;
        const int r = in_x ? threadIdx.x : threadIdx.x - XT, rows = in_x ? XT : YT;
        if (XT + YT < kThreads && r >= rows) return;
        if constexpr (H == 1) {
            // Of the 64 rows of a wavefront, rows 16 apart lie in one word: the lanes that hold them exchange bytes, and lane 16 q + j writes
            // block q's of rows j, j + 16, j + 32 and j + 48 (byte by byte four lanes met in each word).
            static_assert(XT % kWave == 0 && YT % kWave == 0, "a wavefront brings rows of one operand");
            const auto pair = __builtin_amdgcn_permlane16_swap(b.v[0], b.v[0], false, false);          // rows of lanes 0 and 2, 1 and 3
            const auto even = __builtin_amdgcn_permlane32_swap(pair[0], pair[0], false, false), odd = __builtin_amdgcn_permlane32_swap(pair[1], pair[1], false, false);
            const uint32_t q = (threadIdx.x & 63) >> 4, pick = 0x0c0c0400u + q * 0x0101u;              // byte q of the second, then of the first
            const uint32_t low = __builtin_amdgcn_perm(odd[0], even[0], pick), high = __builtin_amdgcn_perm(odd[1], even[1], pick);
            *reinterpret_cast<uint32_t *>(lds + (in_x ? 0 : 4 * XT) + q * rows + (r & 15) * (rows / 16) + (r >> 6) * 4) = low | high << 16;
            return;
        }
        uint8_t *const at = lds + (in_x ? 0 : 4 * XT) + (r & 15) * (rows / 16) + (r >> 4);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) at[h * kScaleBytes + i * rows] = static_cast<uint8_t>(b.v[h] >> (8 * i));
    }

    // A stage is multiplied in parts: H steps, kQ of x's subtiles at a time; what a part multiplies has been read from LDS a part before.
    static constexpr int kQ = SX < 4 ? SX : 4, kPer = SX / kQ, kParts = H * kPer;
    static constexpr int kPlaneX = XT * kStepBytes * H, kPlaneY = YT * kStepBytes * H, kY = P * kPlaneX;      // where y's part of a stage begins
    __device__ __forceinline__ void read_part(const char *ring, int part, i32x4 (&x)[P][kQ], i32x4 (&y)[P][SY]) const
    {
        const int half = part / kPer, q = part % kPer;
        if (q == 0)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int n = 0; n < SY; ++n) y[p][n] = stage_part<YT, YS, H>(ring, kY + p * kPlaneY, address_y, half, n);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int m = 0; m < kQ; ++m) x[p][m] = stage_part<XT, XS, H>(ring, p * kPlaneX, address_x, half, q * kQ + m);
    }
    __device__ __forceinline__ void multiply_part(const i32x4 (&x)[P][kQ], const i32x4 (&y)[P][SY], int part, const Scales &scales)
    {
        const int half = part / kPer, q = part % kPer;
#pragma unroll
        for (int i = 0; i < (P > 1 ? kPartProducts : 1); ++i)
#pragma unroll
            for (int m = 0; m < kQ; ++m)
#pragma unroll
                for (int n = 0; n < SY; ++n) {
                    const int at = q * kQ + m;
                    f32x4 &c = acc[at][n];
                    if constexpr (Mul::kScaled)
                        c = Mul::mul(x[0][m], y[0][n], c, static_cast<int>(scales.x[half][at / 4]), at % 4, static_cast<int>(scales.y[half][n / 4]), n % 4);
                    else if constexpr (P > 1)
                        c = Mul::mul(x[kPartsX[i]][m], y[kPartsY[i]][n], c);
                    else
                        c = Mul::mul(x[0][m], y[0][n], c);
                }
    }
    // In what order a part's instructions are issued: the next part's reads of LDS between the first products, so that each has the
    // rest of the part to arrive (left to itself the compiler puts them right before their use).
    template <int READS, int PRODUCTS>
    static __device__ __forceinline__ void order_part()
    {
        constexpr int kLds = 0x100, kMatrix = 0x8, kEach = READS > PRODUCTS ? 1 : PRODUCTS / READS > 2 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < (READS < PRODUCTS ? READS : PRODUCTS); ++i) {
            __builtin_amdgcn_sched_group_barrier(kLds, READS > PRODUCTS ? READS / PRODUCTS : 1, 0);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kEach, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, PRODUCTS, 0);
    }

    __device__ __forceinline__ void run(const Operand &x, const Operand &y, int64_t i0, int64_t j0, int64_t k0, int64_t k1)
    {
        run(x, y, i0, j0, k0, k1, [] {});
    }

    static constexpr int kRingBytes = P * (XT + YT) * kStepBytes * H;
    // the first stage's memory; the results pass through it
    static __device__ __forceinline__ char *first_ring()
    {
        __shared__ __attribute__((aligned(1024))) char ring0[kRingBytes];
        return ring0;
    }

    // Stores the tile row by row j, value(m, n) the four results of subtile (m, n) in memory's type: out: where the tile's first row
    // begins, rows, cols: how many of the tile's rows and of their columns there are.  A lane's four results are 8 or 16 bytes of one of sixteen
    // rows; each wavefront turns them, through its part of LDS, into up to 256 neighbouring bytes of a row.  (The
    // gradient of a 20011 x 1001 float16 model, on 256 x 256 tiles: written four numbers at a time 83 us, so 50.)
    template <class Mem, class Value>
    __device__ __forceinline__ void store(Mem *out, int64_t ld, int64_t rows, int64_t cols, Value value) const
    {
        typedef __attribute__((ext_vector_type(4))) Mem Quad;
        struct __attribute__((packed, aligned(sizeof(Mem)))) Chunk {
            i32x4 v;
        };
        constexpr int kSize = sizeof(Mem), kCols = SX * 16 < 256 / kSize ? SX * 16 : 256 / kSize, kSub = kCols / 16, kCh = kCols * kSize / 16;
        constexpr int kEach = 16 / kSize;                         // numbers of a chunk
        static_assert(16 * kCols * kSize * WX * WY <= kRingBytes, "a part of the first stage for each wavefront");
        __syncthreads();
        char *const mine = first_ring() + wave() * 16 * kCols * kSize;
        const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
#pragma unroll
        for (int n = 0; n < SY; ++n)
#pragma unroll
            for (int group = 0; group < SX / kSub; ++group) {
#pragma unroll
                for (int m = 0; m < kSub; ++m) {
                    const int at = (m * 16 + g * 4) * kSize, chunk = at / 16 ^ (j & (kCh - 1));
                    *reinterpret_cast<Quad *>(mine + j * kCols * kSize + chunk * 16 + at % 16) = value(group * kSub + m, n);
                }
#pragma unroll
                for (int i = 0; i < (16 * kCh + 63) / 64; ++i) {
                    const int id = i * 64 + lane, r = id / kCh, chunk = id % kCh;
                    if (16 * kCh < 64 && r >= 16) continue;
                    const i32x4 v = *reinterpret_cast<const i32x4 *>(mine + r * kCols * kSize + (chunk ^ (r & (kCh - 1))) * 16);
                    const int64_t row = sub_y(n) * 16 + r, col = sub_x(group * kSub) * 16 + chunk * kEach;
                    if (row >= rows || col >= cols) continue;
                    Mem *const to = out + row * ld + col;
                    if (col + kEach <= cols) {
                        reinterpret_cast<Chunk *>(to)->v = v;
                    } else {
                        typedef __attribute__((ext_vector_type(kEach))) Mem All;
                        const All each = __builtin_bit_cast(All, v);
#pragma unroll
                        for (int e = 0; e < kEach; ++e)
                            if (col + e < cols) to[e] = each[e];
                    }
                }
            }
    }

    // k0 .. k1 (in pairs of bytes, multiples of 32) of rows i0.. of x and j0.. of y.  meanwhile(): what is done when the first stages have
    // been asked for.
    template <class Meanwhile>
    __device__ __forceinline__ void run(const Operand &x, const Operand &y, int64_t i0, int64_t j0, int64_t k0, int64_t k1, Meanwhile meanwhile)
    {
        // (an array of its own for each stage: the compiler keeps apart what is read and what is arriving by the array, up to seven)
        static_assert(R >= 2 && R <= 4, "arrays for up to four stages");
        __shared__ __attribute__((aligned(1024))) char ring1[kRingBytes], ring2[R > 2 ? kRingBytes : 16], ring3[R > 3 ? kRingBytes : 16];
        char *const ring0 = first_ring();
        __shared__ __attribute__((aligned(16))) uint8_t scales0[Mul::kScaled ? kScaleBytes * H : 16], scales1[Mul::kScaled ? kScaleBytes * H : 16];
        typedef StageLoads<XT, XS, kThreads, H, EDGE> LoadsX;
        typedef StageLoads<YT, YS, kThreads, H, EDGE> LoadsY;
        LoadsX lx;
        LoadsY ly;
        lx.init(x);
        ly.init(y);
#pragma unroll
        for (int m = 0; m < SX; ++m)
#pragma unroll
            for (int n = 0; n < SY; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int stages = static_cast<int>((k1 - k0 + 32 * H - 1) / (32 * H));
        if (stages <= 0) return;
        address_x = part_address<XT, XS, H>(sub_x(0));
        address_y = part_address<YT, YS, H>(sub_y(0));
        Reader<XT, XS, H> rx(x, i0, k0);
        Reader<YT, YS, H> ry(y, j0, k0);
        // stages to be loaded yet, bytes of k that they hold of a row (4-bit rows end with a group of 128 numbers, one step)
        int coming = stages, wide_x = static_cast<int>(XS ? 0 : lesser(k1, x.cols) - k0) * 2, wide_y = static_cast<int>(YS ? 0 : lesser(k1, y.cols) - k0) * 2;
        // Loads of a stage, asked for in kSlices slices: right behind the barrier that frees its place in the ring, and a part later.
        // Behind the last stage they find nothing and bring zeros, so that every wavefront has as many loads under way as ever.
        constexpr int kSlices = kParts > 1 && R > 2 ? 2 : 1;
        const int to = wave() * kWave * 16;
        auto load = [&](char *ring, int slice) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                lx.issue(rx.buffer(coming > 0, p * x.plane), ring, p * kPlaneX + to, p, P, slice, kSlices, wide_x);
                ly.issue(ry.buffer(coming > 0, p * y.plane), ring, kY + p * kPlaneY + to, p, P, slice, kSlices, wide_y);
            }
            if (slice + 1 < kSlices) return;
            --coming;
            wide_x -= kStepBytes * H;
            wide_y -= kStepBytes * H;
            rx.next();
            ry.next();
        };
        static_assert(H == 1 || H * kPer % 2 == 0, "parity");
        i32x4 px[2][P][kQ], py[2][P][SY];       // of a part and of the next: x by the part, y by the step
        Scales scales{}, scales_next{};
        Brought brought[2] = {}, scales_at[2] = {};      // scales on their way to LDS, by the stage; of the first two stages
        const uint8_t *row = nullptr;
        const int64_t groups = k1 / 32;
        i32x4 four{}, four_next{};              // of this turn of the ring's stages and of the next
        constexpr bool kFours = Mul::kScaled && H == 1;
        static_assert(!kFours || (R == 4 && XT + YT == kThreads), "a turn is four stages, every thread has a row");
        if constexpr (kFours) {
            const int t = threadIdx.x;
            row = t < XT ? x.scales + lesser(i0 + t, x.rows - 1) * x.ld_scales : y.scales + lesser(j0 + t - XT, y.rows - 1) * y.ld_scales;
            if (groups >= 4) {
                four = load_four(row, 0, static_cast<int>(groups));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) four[i] = *reinterpret_cast<const int *>(row + min(i, static_cast<int>(groups) - 1) * 4);
                row = reinterpret_cast<const uint8_t *>(x.p);       // (for the loop, which asks for a next turn's without a branch: some 16 bytes)
            }
            scales_at[0].v[0] = four[0];
            scales_at[1].v[0] = four[1];
        } else if constexpr (Mul::kScaled) {
            const int t = threadIdx.x;
            row = t < XT ? x.scales + lesser(i0 + t, x.rows - 1) * x.ld_scales : t < XT + YT ? y.scales + lesser(j0 + t - XT, y.rows - 1) * y.ld_scales : nullptr;
            scales_at[0] = load_scales(row, 0, groups);
            scales_at[1] = load_scales(row, 1, groups);
            brought[0] = load_scales(row, 2, groups);
            brought[1] = load_scales(row, 3, groups);
        }
        auto load_all = [&](char *ring) {
#pragma unroll
            for (int slice = 0; slice < kSlices; ++slice) load(ring, slice);
        };
        auto ring = [&](int i) { return i == 0 ? ring0 : i == 1 ? ring1 : i == 2 ? ring2 : ring3; };
#pragma unroll
        for (int i = 0; i < R - 1; ++i) load_all(ring(i));
        load(ring(R - 1), 0);
        meanwhile();
        if constexpr (Mul::kScaled) {
            write_scales(scales0, scales_at[0]);
            write_scales(scales1, scales_at[1]);
        }
        // loads that every wavefront has under way per stage, of a first slice
        constexpr int kEach = P * (LoadsX::kSurely + LoadsY::kSurely), kFirst = LoadsX::first(P, kSlices) + LoadsY::first(P, kSlices);
        stage_arrived<(R - 2) * kEach + kFirst>();
        read_part(ring0, 0, px[0], py[0]);
        if constexpr (Mul::kScaled) read_scales(scales0, scales);
        // Stage s out of `now`; `next` holds the next one, the second slice of `later` is still to be asked for.
        auto stage = [&](char *now, char *next, char *later, uint8_t *ss, uint8_t *sn, int u, int s) {
            const int parity = u & 1;
            constexpr int kPerX = P * (XS ? 2 : 1), kPerY = P * (YS ? 2 : 1), kProducts = (P > 1 ? kPartProducts : 1) * kQ * SY;
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                __builtin_amdgcn_sched_barrier(0);
                const int mine = (kParts & 1 ? parity : 0) ^ (part & 1), yours = (H & 1 ? parity : 0) ^ (part / kPer & 1);
                const int y_next = (part + 1) % kPer ? yours : yours ^ 1;
                if (part + 1 < kParts) {
                    read_part(now, part + 1, px[mine ^ 1], py[y_next]);
                    if (part == 0 && kSlices > 1) load(later, 1);
                } else {
                    stage_arrived<(R - 2) * kEach>();                    // the next stage's; what was asked for since then is on its way
                    if constexpr (Mul::kScaled) {
                        read_scales(sn, scales_next);                    // written before this barrier
                        // stage s + 2's; what was there was read before it
                        if constexpr (kFours) {
                            const int turn = s - u;
                            const int most = max(static_cast<int>(groups), 4);
                            write_scales(ss, u < 2 ? one_of(four, turn, (u + 2) & 3, most) : one_of(four_next, turn + 4, (u + 2) & 3, most));
                            if (u == 0) four_next = load_four(row, turn + 4, static_cast<int>(groups));
                            if (u == 3) four = four_next;
                        } else {
                            write_scales(ss, brought[parity]);
                            brought[parity] = load_scales(row, s + 4, groups);
                        }
                    }
                    read_part(next, 0, px[mine ^ 1], py[y_next]);        // (after the last stage: zeros)
                    load(now, 0);
                }
                multiply_part(px[mine], py[yours], part, scales);
                if ((part + 1) % kPer) order_part<kQ * kPerX, kProducts>();
                else order_part<kQ * kPerX + SY * kPerY, kProducts>();
            }
            if constexpr (Mul::kScaled) scales = scales_next;
        };
        constexpr int kTurn = R % 2 ? 2 * R : R;          // stages after which ring and parity are where they were
        auto step = [&](int u, int s) {
            stage(ring(u % R), ring((u + 1) % R), ring((u + R - 1) % R), u & 1 ? scales1 : scales0, u & 1 ? scales0 : scales1, u, s + u);
        };
        // (Whole turns in a loop without exits: with them the compiler loses track of what has arrived where the loop begins again, and waits
        // there for all but one of the loads: 8192 x 47236 x 4096 in bfloat16 2.65 ms for its scores instead of 2.75.)
        int s = 0;
        for (; s + kTurn <= stages; s += kTurn) {
#pragma unroll
            for (int u = 0; u < kTurn; ++u) step(u, s);
        }
#pragma unroll
        for (int u = 0; u < kTurn - 1; ++u) {
            if (s + u >= stages) break;
            step(u, s);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);     // nothing is on its way to LDS any more
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

template <int TYPE>
using Quad = __attribute__((ext_vector_type(4))) typename Num<TYPE>::Mem;
template <int TYPE>
__device__ __forceinline__ Quad<TYPE> quad_of(f32x4 v)
{
    return Quad<TYPE>{Num<TYPE>::store(v[0]), Num<TYPE>::store(v[1]), Num<TYPE>::store(v[2]), Num<TYPE>::store(v[3])};
}

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

// (Which sizes of tiles there are and the rules that choose them: launch_sizes.h.)
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

// The launch of a kernel in a tile's size: `what`, then x, y, the wavefronts that share them, steps a stage, stages in the ring, parts of a number
// (kInParts: float32's three).  The callers list the sizes that their rules give.
#define DQ_TILE_Large(parts) 256, parts ? 128 : 256, 2, 4, 1, parts ? 2 : 4, parts ? 3 : 1
#define DQ_TILE_Half(parts) 256, 128, 2, 2, 1, 3, 1
#define DQ_TILE_Middle(parts) 128, parts ? 64 : 128, 2, 2, 1, parts ? 2 : 4, parts ? 3 : 1
#define DQ_TILE_Few(parts) 64, 64, 2, 2, parts ? 1 : 2, 4, parts ? 3 : 1
#define DQ_TILE_Fewest(parts) 64, 16, 4, 1, parts ? 1 : 2, 4, parts ? 3 : 1
#define DQ_TILE_FewestAcross(parts) 128, 16, 4, 1, parts ? 1 : 2, 4, parts ? 3 : 1
constexpr TileSize kTileFewestAcross = kTileFewest;
#define DQ_TILE_LAUNCH(kernel, what, size, ...) kernel<what, DQ_TILE_##size(kInParts)><<<grid, threads_of(kTile##size), 0, st>>>(__VA_ARGS__)

}  // namespace dq
