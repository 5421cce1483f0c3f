// One tile of a product of two matrices in 8-bit blocks, on the matrix cores:  out[i][j] = sum_b 2^(sx_ib + sy_jb) sum_{k in block b} x(i, k) y(j, k).
//
// 32 x 32 results from 64 numbers an instruction, which takes the two rows' scales along; a stage is a block of every row, 128 bytes, in a ring of two or four.
// LDS holds it as it lies in memory, the eight 16-byte chunks of row r at c ^ (r / 2 % 8): of the sixteen lanes that read together (0 to 3, 12 to 15 and 20 to 27 of 32, or
// the others) those whose rows begin at the same banks then read different chunks.  A lane holds chunks 2 h and 2 h + 1 of either half of row lane % 32, h = lane / 32,
// and of a result the four neighbouring i at 8 q + 4 h, q = 0 .. 3, of column j = lane % 32.
// Rings of two where the matrix cores bound, for one large tile or two middle ones to a compute unit; four where there is one middle tile to a unit, for a stage there
// takes as long as its loads, divided by those under way.  (Stages of half a block in rings of four, whose loads are of half a line of the cache, took 5%
// longer at 8192 x 47236 x 4096 and 8% at 8192 x 8192 x 8192; middle tiles, 5003 x 1001 x 2049, 25 us, whole blocks 20.)
//
// The scales of two blocks are brought at a time, by the thread whose row they are of, a turn of the ring ahead, and lie in LDS as [row % 32][row / 32], so
// that a lane reads those of all its subtiles at once.
//
// What is rounded: of the eight products that the matrix cores take together, what is less than 2^-13 of the power of two of the largest is left out (measured:
// each product is cut towards zero there; what comes of it is added up in float32).  Sums of 128 normally distributed codes are 1.5 10^-5 off in norm, a
// hundredth of bfloat16's rounding and a thirteenth of float16's; float32 results are not made here.
#pragma once

#include "fp8_codes.h"

namespace dq {

typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __forceinline__ int chunk_swap8(int row) { return row >> 1 & 7; }

template <int T, int THREADS>
struct Fp8Loads {
    static constexpr int kRow = 8, kChunks = T * kRow / THREADS;      // 16-byte loads of a thread per stage
    static_assert(T * kRow % THREADS == 0, "as many of every thread");
    uint32_t off[kChunks];
    __device__ __forceinline__ void init(int64_t ld)
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int id = threadIdx.x + i * THREADS, row = id / kRow, slot = id % kRow;
            off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(ld) + static_cast<uint32_t>((slot ^ chunk_swap8(row)) * 16);
        }
    }
    // Slice 0 or 1 of them.
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t from, char *ring, int to, int slice) const
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            if (i * 2 / kChunks == slice)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (LdsPtr)(ring + (to + i * THREADS * 16)), 16, static_cast<int>(off[i]), 0, 0, 0);
    }
    static constexpr int first() { return (kChunks + 1) / 2; }
};

// WX x WY wavefronts share the tile, each has SX x SY subtiles of 32 x 32.  R stages in the ring.
template <int XT, int YT, int WX, int WY, int R>
struct Fp8Tile {
    static constexpr int kThreads = WX * WY * kWave, SX = XT / 32 / WX, SY = YT / 32 / WY, kBytes = kGroup8;
    static constexpr int kRing = (XT + YT) * kBytes, kY = XT * kBytes;
    static_assert(XT + YT == kThreads && SX % 2 == 0 && SY % 2 == 0, "a thread brings one row's scales; a lane reads them in words");
    f32x16 acc[SX][SY];

    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    static __device__ __forceinline__ int sub_x(int m) { return (wave() % WX) * SX + m; }
    static __device__ __forceinline__ int sub_y(int n) { return (wave() / WX) * SY + n; }
    static __device__ __forceinline__ char *first_ring()
    {
        __shared__ __attribute__((aligned(1024))) char ring0[kRing];
        return ring0;
    }
    static __device__ __forceinline__ char *second_ring()
    {
        __shared__ __attribute__((aligned(1024))) char ring1[kRing];
        return ring1;
    }
    static __device__ __forceinline__ i32x8 read(const char *ring, int from, int address, int half)
    {
        // (chunk 2 h + 1 lies where chunk 2 h does with its lowest bit turned, the second half's with their third)
        address ^= half * 64;
        const i32x4 lo = *reinterpret_cast<const i32x4 *>(ring + (from + address)), hi = *reinterpret_cast<const i32x4 *>(ring + (from + (address ^ 16)));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    template <int M, int N>
    static __device__ __forceinline__ f32x16 multiply(i32x8 x, i32x8 y, f32x16 c, int sx, int sy)
    {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 0, 0, M, sx, N, sy);
    }
    // (which byte of a word of scales is part of the instruction)
    static __device__ __forceinline__ f32x16 multiply(i32x8 x, i32x8 y, f32x16 c, int sx, int m, int sy, int n)
    {
        switch (m * 4 + n) {
        case 0: return multiply<0, 0>(x, y, c, sx, sy);
        case 1: return multiply<0, 1>(x, y, c, sx, sy);
        case 2: return multiply<0, 2>(x, y, c, sx, sy);
        case 3: return multiply<0, 3>(x, y, c, sx, sy);
        case 4: return multiply<1, 0>(x, y, c, sx, sy);
        case 5: return multiply<1, 1>(x, y, c, sx, sy);
        case 6: return multiply<1, 2>(x, y, c, sx, sy);
        case 7: return multiply<1, 3>(x, y, c, sx, sy);
        case 8: return multiply<2, 0>(x, y, c, sx, sy);
        case 9: return multiply<2, 1>(x, y, c, sx, sy);
        case 10: return multiply<2, 2>(x, y, c, sx, sy);
        case 11: return multiply<2, 3>(x, y, c, sx, sy);
        case 12: return multiply<3, 0>(x, y, c, sx, sy);
        case 13: return multiply<3, 1>(x, y, c, sx, sy);
        case 14: return multiply<3, 2>(x, y, c, sx, sy);
        default: return multiply<3, 3>(x, y, c, sx, sy);
        }
    }

    // Rows i0.. of x and j0.. of y, blocks g0 (an even number) to g1.
    __device__ __forceinline__ void run(const dq_fp8 &x, const dq_fp8 &y, int64_t i0, int64_t j0, int g0, int g1)
    {
        constexpr int kQ = 2, kPer = SX / kQ, kParts = kPer * 2;
        __shared__ __attribute__((aligned(1024))) char ring2[R > 2 ? kRing : 16], ring3[R > 2 ? kRing : 16];
        static_assert(R == 2 || R == 4, "arrays for up to four stages");
        __shared__ __attribute__((aligned(16))) u16 scales[2][XT + YT];
        char *const ring0 = first_ring(), *const ring1 = second_ring();
        auto ring = [&](int i) { return i == 0 ? ring0 : i == 1 ? ring1 : i == 2 ? ring2 : ring3; };
        typedef Fp8Loads<XT, kThreads> LoadsX;
        typedef Fp8Loads<YT, kThreads> LoadsY;
        LoadsX lx;
        LoadsY ly;
        lx.init(x.ld_codes);
        ly.init(y.ld_codes);
#pragma unroll
        for (int m = 0; m < SX; ++m)
#pragma unroll
            for (int n = 0; n < SY; ++n) acc[m][n] = f32x16{};
        const int groups = g1, stages = g1 - g0;
        const Operand ox{reinterpret_cast<const char *>(x.codes), x.ld_codes, x.n, groups * 64, 0, nullptr, 0}, oy{reinterpret_cast<const char *>(y.codes), y.ld_codes, y.n, groups * 64, 0, nullptr, 0};
        Reader<XT, false, 2> rx(ox, i0, g0 * 64);
        Reader<YT, false, 2> ry(oy, j0, g0 * 64);
        int coming = stages;
        const int to = wave() * kWave * 16, lane = threadIdx.x & 63;
        auto load = [&](char *at, int slice) {
            lx.issue(rx.buffer(coming > 0, 0), at, to, slice);
            ly.issue(ry.buffer(coming > 0, 0), at, kY + to, slice);
            if (slice == 0) return;
            --coming;
            rx.next();
            ry.next();
        };
        const int r = threadIdx.x, address = (lane & 31) * kBytes + (((lane >> 5) * 2 ^ chunk_swap8(lane & 31)) * 16);
        const uint8_t *const row = r < XT ? x.scales + lesser(i0 + r, x.n - 1) * x.ld_scales : y.scales + lesser(j0 + r - XT, y.n - 1) * y.ld_scales;
        const int place = r < XT ? (r & 31) * (XT / 32) + (r >> 5) : XT + ((r - XT) & 31) * (YT / 32) + ((r - XT) >> 5);
        // two blocks' scales (behind the last, where codes are zeros: any)
        auto bring = [&](int pair) { return *reinterpret_cast<const u16 *>(row + min(g0 / 2 + pair, (groups - 1) / 2) * 2); };
        u16 coming_scales = bring(1);
        scales[0][place] = bring(0);
        struct Scales {
            uint32_t x[SX / 2], y[SY / 2];
        } now_scales{}, next_scales{};
        auto read_scales = [&](int pair, Scales &s) {
            const u16 *const at = scales[pair & 1];
#pragma unroll
            for (int i = 0; i < SX / 2; ++i) s.x[i] = reinterpret_cast<const uint32_t *>(at + (lane & 31) * (XT / 32) + sub_x(0))[i];
#pragma unroll
            for (int i = 0; i < SY / 2; ++i) s.y[i] = reinterpret_cast<const uint32_t *>(at + XT + (lane & 31) * (YT / 32) + sub_y(0))[i];
        };
#pragma unroll
        for (int i = 0; i < R - 1; ++i) {
            load(ring(i), 0);
            load(ring(i), 1);
        }
        load(ring(R - 1), 0);
        constexpr int kEach = LoadsX::kChunks + LoadsY::kChunks, kFirst = LoadsX::first() + LoadsY::first();
        i32x8 px[2][kQ], py[2][SY];
        auto read_part = [&](const char *at, int part, i32x8 (&ax)[kQ], i32x8 (&ay)[SY]) {
            const int half = part / kPer, q = part % kPer;
            if (q == 0)
#pragma unroll
                for (int n = 0; n < SY; ++n) ay[n] = read(at, kY + sub_y(n) * 32 * kBytes, address, half);
#pragma unroll
            for (int m = 0; m < kQ; ++m) ax[m] = read(at, sub_x(q * kQ + m) * 32 * kBytes, address, half);
        };
        stage_arrived<(R - 2) * kEach + kFirst>();
        read_part(ring0, 0, px[0], py[0]);
        read_scales(0, now_scales);
        // Stage u of turn `turn`.
        auto stage = [&](int u, int turn) {
            char *const now = ring(u), *const next = ring((u + 1) % R), *const later = ring((u + R - 1) % R);
            const int block = u % 2, pair = turn * (R / 2) + u / 2;
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                __builtin_amdgcn_sched_barrier(0);
                const int mine = part & 1, half = part / kPer, q = part % kPer;
                if (part == 0) load(later, 1);
                if (part + 1 < kParts) {
                    read_part(now, part + 1, px[mine ^ 1], py[(part + 1) / kPer]);
                } else {
                    stage_arrived<(R - 2) * kEach>();
                    if (block == 0) {                  // the next two blocks' scales: who read what lay there did so long ago
                        scales[(pair + 1) & 1][place] = coming_scales;
                        coming_scales = bring(pair + 2);
                    }
                    if (block == 1) read_scales(pair + 1, next_scales);
                    read_part(next, 0, px[mine ^ 1], py[0]);
                    load(now, 0);
                }
#pragma unroll
                for (int m = 0; m < kQ; ++m)
#pragma unroll
                    for (int n = 0; n < SY; ++n) {
                        const int at = q * kQ + m;
                        acc[at][n] = multiply(px[mine][m], py[half][n], acc[at][n], static_cast<int>(now_scales.x[at / 2]), 2 * (at & 1) + block,
                                              static_cast<int>(now_scales.y[n / 2]), 2 * (n & 1) + block);
                    }
                // the next part's reads of LDS between the products
                constexpr int kLds = 0x100, kMatrix = 0x8, kProducts = kQ * SY;
                const bool both = (part + 1) % kPer == 0;
#pragma unroll
                for (int i = 0; i < kProducts; ++i) {
                    if (!both) __builtin_amdgcn_sched_group_barrier(kLds, 2 * kQ / kProducts > 0 ? 2 * kQ / kProducts : 1, 0);
                    else __builtin_amdgcn_sched_group_barrier(kLds, (2 * (kQ + SY) + kProducts - 1) / kProducts, 0);
                    __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
                }
            }
            if (block == 1) now_scales = next_scales;
        };
        int turn = 0;
        for (; R * turn + R <= stages; ++turn) {
#pragma unroll
            for (int u = 0; u < R; ++u) stage(u, turn);
        }
#pragma unroll
        for (int u = 0; u < R - 1; ++u) {
            if (R * turn + u >= stages) break;
            stage(u, turn);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);      // nothing is on its way to LDS any more
    }

    // The sums in float32, row by row j.
    __device__ __forceinline__ void store_sums(float *out, int64_t ld, int64_t rows, int64_t cols) const
    {
        const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
#pragma unroll
        for (int n = 0; n < SY; ++n)
#pragma unroll
            for (int m = 0; m < SX; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16 &c = acc[m][n];
                    const int64_t row = sub_y(n) * 32 + j, col = sub_x(m) * 32 + 8 * q + 4 * h;
                    if (row < rows && col < cols)
                        store_four<DQ_F32>(out + row * ld + col, f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]}, static_cast<int>(lesser(cols - col, 4)), ld % 4 == 0);
                }
    }

    // Stores the tile row by row j (16 bits a number): each wavefront turns 32 rows of all its columns at a time, through its part of the first two stages, into
    // as many neighbouring bytes a row as it has (256 of a large tile), which go past the cache.  8192 x 47236 x 4096, whose rows begin anywhere: 128 bytes at a time
    // 26 us more, not past the cache 112 more (nothing stored: 132 less).
    template <int TYPE>
    __device__ __forceinline__ void store(typename Num<TYPE>::Mem *out, int64_t ld, int64_t rows, int64_t cols) const
    {
        typedef typename Num<TYPE>::Mem Mem;
        constexpr int kWide = SX * 64, kCh = kWide / 16;             // bytes and chunks of a row
        static_assert(sizeof(Mem) == 2 && 32 * kWide * WX * WY <= 2 * kRing, "a part of the first two stages for each wavefront");
        struct __attribute__((packed, aligned(2))) Chunk {
            i32x4 v;
        };
        __syncthreads();
        constexpr int kHalf = WX * WY / 2;
        char *const mine = (wave() < kHalf ? first_ring() : second_ring()) + wave() % kHalf * 32 * kWide;
        const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
#pragma unroll
        for (int n = 0; n < SY; ++n) {
#pragma unroll
            for (int m = 0; m < SX; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16 &c = acc[m][n];
                    const f32x4 v{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
                    const int chunk = m * 4 + q;                     // sixteen bytes: the eight numbers at 32 m + 8 q, h the half
                    *reinterpret_cast<i32x2 *>(mine + j * kWide + (chunk ^ (j & (kCh - 1))) * 16 + h * 8) = __builtin_bit_cast(i32x2, quad_of<TYPE>(v));
                }
#pragma unroll
            for (int i = 0; i < kCh / 2; ++i) {
                const int id = i * 64 + lane, r = id / kCh, chunk = id % kCh;
                const i32x4 v = *reinterpret_cast<const i32x4 *>(mine + r * kWide + (chunk ^ (r & (kCh - 1))) * 16);
                const int64_t row = sub_y(n) * 32 + r, col = sub_x(0) * 32 + chunk * 8;
                if (row >= rows || col >= cols) continue;
                Mem *const at = out + row * ld + col;
                if (col + 8 <= cols) {
                    __builtin_nontemporal_store(v, &reinterpret_cast<Chunk *>(at)->v);
                } else {
                    typedef __attribute__((ext_vector_type(8))) Mem All;
                    const All each = __builtin_bit_cast(All, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < cols) at[e] = each[e];
                }
            }
        }
    }
};

}  // namespace dq
