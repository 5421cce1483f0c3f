// A matrix update orthogonalized by Newton-Schulz products: its singular values all brought near 1, its singular vectors kept.
//   X = G / |G|_F, then `steps` times, on the shorter side:  A = X X^T,  B = b A + c A^2,  X = a X + B X
// with the odd polynomial a s + b s^3 + c s^5, a, b, c = 3.4445, -4.7750, 2.0315, that takes (0, 1] into 0.68 .. 1.21 within five steps.
//
// Where G has more rows than columns, everything is done on its transpose, which is never made: A = X^T X, X = a X + X B.
//
// Two ways.  Step by step, as the formulas say: products of s^2 l (s the shorter side, l the longer) two or three times a step.  Or, 16-bit types, through the small
// matrices alone: with Q = a + B, A of the next step is Q A Q, and X after all steps is P X, P the product of the Q: s^2 l once for A, twice (P in two parts) for P X, and
// four products of s^3 a step, which is less where l is more than 1.2 s (float16 goes that way always).  P is held less a^steps times one, and Q less a:
// what is held then is as small as A is where a matrix has nothing.
//
// What is rounded to what.  An error E of A or Q acts as (1 + E) X, which turns and stretches what is there by E; an error added to X puts
// something where a matrix of low rank has nothing, and every later step makes that 3.4445 times as large, 485 times in five.  So everything is the sum of two float16, 22
// bits: X, A and B = b A + c A^2.  (X in one float16: 0.001 off where all singular values count, 0.1 for one direction; in one bfloat16 0.012 and 0.75.  A and B in one,
// 11 bits: roundings that go either way leave 0.0012 in norm, but those of a matrix whose numbers share their significands are all the same and left 0.006, more than
// bfloat16's own half step; five steps of 4096 x 4096 took 2.4 ms so, and 4.0 in two.)  Through the small matrices X is the matrix that was given, exactly, and A, B and P
// are two float16 each: 10^-5 (singular values of one size) to 8 10^-4 (one direction: P X adds up 485 times its result in float32).  X, A, B and P are held times 2^14,
// 2^14, 2^12 (through the small matrices 2^13) and 2^6, so that entries of a matrix of 2^28 numbers are normal float16 ones and P's of five steps (up to 485) in range.
//
// float32 goes step by step: two float16, and three products of their four, are at worst four times float32's rounding, but the sums' and the steps' own
// roundings are the larger part, 2 10^-6 to 10^-4 in norm as in float32 throughout (256 x 1000 of noise 2.2 and 2.1 10^-6, of rank 1 1.26 and 1.21 10^-4; three
// numbers by 5000 1.1 10^-6 and 5 10^-7).  Three bfloat16 parts, six products, were no nearer there than 0.3 to 0.8 times and took 1.2 to 1.8 times as long (20958 x 2048
// 7.1 and 4.0 ms, 1000 x 1000 393 and 275 us).
#include <algorithm>
#include <type_traits>

#include "row_items.h"

namespace dq {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kNormBlocks = 1024;
// Numbers are held in one or two float16, times powers of two (step by step).
typedef Num<DQ_F16> Half;
constexpr float kUpX = 16384.0f, kUpA = 16384.0f, kUpB = 4096.0f;

// What lies in front of the workspace: the blocks' sums of squares, and what X of the first step is to be multiplied by.
struct OrthogonalHead {
    double square[kNormBlocks];
    float rest;
    float unused[3];
};

// A matrix in the workspace, row by row, in planes of parts of its numbers that are `next` numbers apart.
struct Parts {
    u16 *p;
    int64_t ld, next;
};

template <int TYPE>
__global__ __launch_bounds__(256) void orthogonal_square_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, uint32_t d, int64_t ld, OrthogonalHead *__restrict__ head)
{
    __shared__ double room[4];
    const uint32_t per = (d + 7) / 8;
    const int64_t total = n * per;
    double sum = 0.0;
    for (int64_t first = blockIdx.x * 256ll + threadIdx.x; first < total; first += 4 * 256ll * kNormBlocks) {
        float x[4][8];
        Eight<TYPE> asked[4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t i = first + u * 256ll * kNormBlocks, row = i / per;
            if (i < total) asked[u] = ask_eight<TYPE>(v + row * ld, static_cast<uint32_t>(i - row * per) * 8, d);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) values_of<TYPE>(asked[u], x[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += static_cast<double>(x[u][e]) * x[u][e];
    }
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) sum += __shfl_xor(sum, by);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) head->square[blockIdx.x] = room[0] + room[1] + room[2] + room[3];
}

// X of the first step: rows x cols numbers (with zeros behind the matrix's), eight a thread.  16-bit types: times the power of two that brings the norm
// to 2^13 .. 2^14, exactly (the rest of the way is `rest`); float32: over the norm.
template <int TYPE>
__global__ __launch_bounds__(256) void orthogonal_pack_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, uint32_t d, int64_t ld, OrthogonalHead *__restrict__ head,
                                                              Parts x, int64_t rows, uint32_t cols, uint32_t *__restrict__ status)
{
    __shared__ double room[4];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kNormBlocks; i += 256) sum += head->square[i + threadIdx.x];
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) sum += __shfl_xor(sum, by);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = sum;
    __syncthreads();
    const double norm = sqrt(room[0] + room[1] + room[2] + room[3]);
    const bool finite = __builtin_isfinite(norm);
    const int up = norm > 0.0 && finite ? 14 - (ilogb(norm) + 1) : 0;
    const double over = norm > 0.0 ? 1.0 / norm : 0.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        head->rest = norm > 0.0 && finite ? static_cast<float>(ldexp(over, 14 - up)) : 1.0f;
        if (!finite && status) atomicOr(status, 1u);
    }
    const uint32_t per = cols / 8;
    const int64_t total = rows * per;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += 256ll * gridDim.x) {
        const int64_t row = i / per;
        const uint32_t c = static_cast<uint32_t>(i - row * per) * 8;
        float y[8] = {};
        if (row < n && c < d) load_eight<TYPE>(v + row * ld, c, d, y);
        u16 *const to = x.p + row * x.ld + c;
        if constexpr (TYPE == DQ_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = finite ? static_cast<float>(y[e] * over * kUpX) : __uint_as_float(0x7fc00000u);
            store_eight<DQ_F16>(to, y, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] -= Half::load(Half::store(y[e]));
            store_eight<DQ_F16>(to + x.next, y, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = finite ? ldexpf(y[e], up) : __uint_as_float(0x7fc00000u);
            store_eight<DQ_F16>(to, y, 8);
        }
    }
}

constexpr float kUpQ = 8192.0f, kUpP = 64.0f;                       // through the small matrices
constexpr int kStepsOfP = 5;

// A product's tile: PX, PY parts of a number of x and y.
template <int SIZE, int PX, int PY, bool XS, bool YS>
struct Shape {
    static constexpr int XT = SIZE == kTileLarge ? 256 : SIZE == kTileMiddle ? 128 : 64, YT = XT;
    static constexpr int WX = 2, WY = SIZE == kTileLarge ? 4 : 2, R = SIZE == kTileFew ? 4 : PX + PY == 2 ? 4 : PX + PY == 3 ? 3 : 2;
    static constexpr int kThreads = WX * WY * kWave;
    typedef TileProduct<typename Half::Mul, XT, YT, WX, WY, XS, YS, 1, R, PX, false, PY> Tile;
};

// tile.acc = two * tile.acc + one * (the sum of `count` parts of a matrix of `rows` rows and `cols` columns, whole chunks of eight, from the tile's first
// number on).  Sixteen rows' 16-byte chunks at a time, which pass through LDS to the lanes that hold their results; all of a part's are asked for together.
// (Four numbers at a time, each waited for, took as long as the product: 47236 x 4096, 2.1 of 4.1 ms.)
template <class Tile>
__device__ __forceinline__ void add_old(Tile &tile, const u16 *p, int64_t ld, int64_t next, int count, int64_t rows, int64_t cols, float one, float two)
{
    constexpr int SX = Tile::SX, SY = Tile::SY, kCols = SX * 16 < 128 ? SX * 16 : 128, kSub = kCols / 16, kCh = kCols / 8, kLoads = 16 * kCh / 64, kGroups = SX / kSub;
    static_assert(16 * kCh % 64 == 0, "whole loads");
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    char *const mine = Tile::first_ring() + Tile::wave() * 16 * kCols * 2;
    i32x4 coming[SY][kGroups][kLoads];
    auto ask = [&](int part, int n) {
#pragma unroll
        for (int group = 0; group < kGroups; ++group)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int id = i * 64 + lane;
                const int64_t row = Tile::sub_y(n) * 16 + id / kCh, col = Tile::sub_x(group * kSub) * 16 + id % kCh * 8;
                coming[n][group][i] = i32x4{0, 0, 0, 0};
                if (row < rows && col < cols) coming[n][group][i] = *reinterpret_cast<const i32x4 *>(p + part * next + row * ld + col);
            }
    };
    if (count) {
#pragma unroll
        for (int n = 0; n < SY; ++n) ask(0, n);
    }
#pragma unroll
    for (int m = 0; m < SX; ++m)
#pragma unroll
        for (int n = 0; n < SY; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) tile.acc[m][n][e] *= two;
    if (!count) return;
    __syncthreads();
    for (int part = 0; part < count; ++part) {
#pragma unroll
        for (int n = 0; n < SY; ++n) {
#pragma unroll
            for (int group = 0; group < kGroups; ++group) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int id = i * 64 + lane, r = id / kCh, chunk = id % kCh;
                    *reinterpret_cast<i32x4 *>(mine + r * kCols * 2 + (chunk ^ (r & (kCh - 1))) * 16) = coming[n][group][i];
                }
#pragma unroll
                for (int m = 0; m < kSub; ++m) {
                    const int at = (m * 16 + g * 4) * 2, chunk = at / 16 ^ (j & (kCh - 1));
                    const u16x4 q = __builtin_bit_cast(u16x4, *reinterpret_cast<const i32x2 *>(mine + j * kCols * 2 + chunk * 16 + at % 16));
#pragma unroll
                    for (int e = 0; e < 4; ++e) tile.acc[group * kSub + m][n][e] += one * Half::load(q[e]);
                }
            }
            if (part + 1 < count) ask(part + 1, n);
        }
    }
}

// Stores the tile's values in PARTS parts, `next` numbers apart.
template <int PARTS, class Tile>
__device__ __forceinline__ void store_parts(Tile &tile, u16 *out, int64_t ld, int64_t next, int64_t rows, int64_t cols)
{
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        tile.store(out + part * next, ld, rows, cols, [&](int m, int n) {
            u16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = tile.acc[m][n][e];
                r[e] = Half::store(v);
                if (part + 1 < PARTS) tile.acc[m][n][e] = v - Half::load(r[e]);
            }
            return r;
        });
    }
}

// A symmetric product S = X Y^T (of matrices that commute) and what becomes of it:  to = two S + one old + more also;  rest: S is of the first X, which wants
// `rest` twice.
struct GramJob {
    Operand x, y;
    const OrthogonalHead *rest;
    float two, one, more;
    Parts old, also, to;
    __device__ __forceinline__ float factor() const { return rest ? two * rest->rest * rest->rest : two; }
};
struct GramJobs {
    GramJob job[2];
};

// 64 x 64 of S, patch (bx, by) with bx >= by, and what mirrors it: above the diagonal nothing is computed, so that the results are symmetric to the last bit (where they
// were not, a matrix of rank 1 came out 2 10^-3 off instead of 2 10^-4).  A thread has sixteen numbers: four neighbours in each of four rows.
template <int OUT>
struct Added {                                                       // what is added to a thread's, as it lies in memory: asked for long before
    u16x4 old[4][OUT], also[4][OUT];
    __device__ __forceinline__ Added(const GramJob &job, int bx, int by, int64_t side)
    {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t row = by * 64 + threadIdx.x / 16 + 16 * u, col = bx * 64 + threadIdx.x % 16 * 4;
            const bool in = row < side && col < side;                // (side is a multiple of 32)
#pragma unroll
            for (int part = 0; part < OUT; ++part) {
                old[u][part] = also[u][part] = u16x4{0, 0, 0, 0};
                if (job.old.p && in) old[u][part] = *reinterpret_cast<const u16x4 *>(job.old.p + part * job.old.next + row * job.old.ld + col);
                if (job.also.p && in) also[u][part] = *reinterpret_cast<const u16x4 *>(job.also.p + part * job.also.next + row * job.also.ld + col);
            }
        }
    }
};
template <int OUT>
__device__ __forceinline__ void gram_end(const GramJob &job, const Added<OUT> &added, f32x4 (&v)[4], float (*turned)[65], int bx, int by, int64_t side)
{
    const int c = threadIdx.x % 16 * 4, r0 = threadIdx.x / 16;
    const float two = job.factor();
    auto add = [&](f32x4 &x, const u16x4 (&of)[OUT], float times) {
        f32x4 old{};
#pragma unroll
        for (int part = 0; part < OUT; ++part)
#pragma unroll
            for (int e = 0; e < 4; ++e) old[e] += Half::load(of[part][e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += times * old[e];
    };
    auto put = [&](f32x4 x, int64_t row, int64_t col) {
        if (row >= side || col >= side) return;
#pragma unroll
        for (int part = 0; part < OUT; ++part) {
            u16x4 q;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                q[e] = Half::store(x[e]);
                x[e] -= Half::load(q[e]);
            }
            *reinterpret_cast<u16x4 *>(job.to.p + part * job.to.next + row * job.to.ld + col) = q;
        }
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t row = by * 64 + r0 + 16 * u, col = bx * 64 + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] *= two;
        add(v[u], added.old[u], job.one);
        add(v[u], added.also[u], job.more);
#pragma unroll
        for (int e = 0; e < 4; ++e) turned[r0 + 16 * u][c + e] = v[u][e];
        if (bx != by) put(v[u], row, col);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = r0 + 16 * u;                                   // row bx * 64 + i of the mirror; at the diagonal one half gives way to the other
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = bx == by && c + e > i ? turned[i][c + e] : turned[c + e][i];
        put(x, bx * 64 + i, by * 64 + c);
    }
}

// How a product's factors are read: both along k, both across it (X^T X), or x across and y along it, which of symmetric matrices is the same and the fastest
// (rows of 512 bytes instead of 64 at a time).
enum { kAlong = 0, kMixed = 1, kAcross = 3 };

// All of it at once, a patch a block.  1024 x 1024 over 1024 in two parts 17 us: some 0.4 a stage of 32, whatever is multiplied.
template <int IN, int OUT, int HOW>
__global__ __launch_bounds__((Shape<kTileFew, IN, IN, (HOW & 1) != 0, (HOW & 2) != 0>::kThreads)) void orthogonal_gram_kernel(GramJobs jobs, int64_t k, int64_t side)
{
    typedef typename Shape<kTileFew, IN, IN, (HOW & 1) != 0, (HOW & 2) != 0>::Tile Tile;
    __shared__ float turned[64][65];
    const GramJob &job = jobs.job[blockIdx.z];
    const int bx = static_cast<int>(blockIdx.x), by = static_cast<int>(blockIdx.y);
    if (bx < by) return;
    const Added<OUT> added(job, bx, by, side);
    Tile tile;
    tile.run(job.x, job.y, bx * 64, by * 64, 0, k);
#pragma unroll
    for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
        for (int n = 0; n < Tile::SY; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) turned[Tile::at_y(n)][Tile::at_x(m) + e] = tile.acc[m][n][e];
    __syncthreads();
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] = turned[threadIdx.x / 16 + 16 * u][threadIdx.x % 16 * 4 + e];
    gram_end<OUT>(job, added, v, turned, bx, by, side);              // (a thread writes where it has read)
}

// The sums of one split of k of one tile at the diagonal or below it (i >= j somewhere), whole, to sums[job][split][tile][j][i].  The blocks of a die take
// neighbouring tiles of one split.  4096 x 4096 over 47236 in one part (136 tiles, five splits) 0.65 ms, 1215 TFLOP/s of the half that is made; over 4096 in two
// parts (three products) 0.19 to 0.22.  (The whole square in one round of 256 tiles: 1.1.)
template <int IN, int SIZE, int HOW>
__global__ __launch_bounds__((Shape<SIZE, IN, IN, (HOW & 1) != 0, (HOW & 2) != 0>::kThreads)) void orthogonal_gram_sums_kernel(GramJobs jobs, int64_t k, GramPlan g, float *__restrict__ sums)
{
    typedef Shape<SIZE, IN, IN, (HOW & 1) != 0, (HOW & 2) != 0> S;
    typedef typename S::Tile Tile;
    const int total = gridDim.x, each = total / 8, more = total % 8, die = blockIdx.x % 8, unit = die * each + min(die, more) + blockIdx.x / 8;
    const int part = unit / g.tiles, split = part % g.splits;
    const GramJob &job = jobs.job[part / g.splits];
    int t = unit - part * g.tiles, ty = 0;
    while (t >= g.tiles_x - ty) {
        t -= g.tiles_x - ty;
        ++ty;
    }
    const int64_t i0 = static_cast<int64_t>(t + ty) * S::XT, j0 = static_cast<int64_t>(ty) * S::YT;
    Tile tile;
    tile.run(job.x, job.y, i0, j0, split * g.per_split, lesser(k, (split + 1) * g.per_split));
    tile.store(sums + static_cast<int64_t>(unit) * (S::XT * S::YT), S::XT, S::YT, S::XT, [&](int m, int n) { return tile.acc[m][n]; });
}

// ... added up, a patch a block.
template <int OUT>
__global__ __launch_bounds__(256) void orthogonal_gram_end_kernel(GramJobs jobs, const float *__restrict__ sums, GramPlan g, int64_t side)
{
    __shared__ float turned[64][65];
    int bx = static_cast<int>(blockIdx.x), by = 0;                   // counted row by row
    const int wide = static_cast<int>((side + 63) / 64);
    while (bx >= wide - by) {
        bx -= wide - by;
        ++by;
    }
    bx += by;
    const Added<OUT> added(jobs.job[blockIdx.y], bx, by, side);
    const int tx = bx * 64 / g.dims.x, ty = by * 64 / g.dims.y, r0 = threadIdx.x / 16;
    const int tile = ty * g.tiles_x - gram_before(ty) + tx - ty;
    const int64_t size = static_cast<int64_t>(g.dims.x) * g.dims.y, all = size * g.tiles;
    const float *const from = sums + blockIdx.y * g.splits * all + tile * size + (by * 64 - ty * g.dims.y) * static_cast<int64_t>(g.dims.x) + bx * 64 - tx * g.dims.x + threadIdx.x % 16 * 4;
    f32x4 v[4] = {};
    int s = 0;
    auto sum = [&](auto count) {                                    // of so many splits, asked for together
        constexpr int N = decltype(count)::value;
        for (; s + N <= g.splits; s += N) {
            f32x4 part[N][4];
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) part[i][u] = *reinterpret_cast<const f32x4 *>(from + (s + i) * all + static_cast<int64_t>(r0 + 16 * u) * g.dims.x);
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] += part[i][u];
        }
    };
    sum(std::integral_constant<int, 8>());
    sum(std::integral_constant<int, 4>());
    sum(std::integral_constant<int, 2>());
    sum(std::integral_constant<int, 1>());
    gram_end<OUT>(jobs.job[blockIdx.y], added, v, turned, bx, by, side);
}

// Bound by the matrix cores: 47236 x 4096 by 4096 x 4096 in two parts 2.75 ms, 1150 TFLOP/s with the ends of 2960 tiles (both factors along k: 2.95).
// X = one X + two B X (TALL: X B, B read across k, as it is symmetric), PX and PY parts of a number of the product's x and y, `parts` of X that are added; in the last step in the result's type.
template <int TYPE, int SIZE, bool TALL, int PX, int PY>
__global__ __launch_bounds__((Shape<SIZE, PX, PY, true, false>::kThreads)) void orthogonal_update_kernel(Operand x, Operand y, int64_t k, Parts old, int parts, int64_t rows, int64_t cols,
                                                                                                         float one, float two, const OrthogonalHead *__restrict__ head, int tiles_x, int tiles_y,
                                                                                                         Parts now, void *__restrict__ out, int64_t ldo, int64_t out_rows, int64_t out_cols)
{
    typedef Shape<SIZE, PX, PY, true, false> S;
    typedef typename S::Tile Tile;
    typedef typename Num<TYPE>::Mem Mem;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * S::XT, j0 = static_cast<int64_t>(ty) * S::YT;
    Tile tile;
    tile.run(x, y, i0, j0, 0, k);
    const float scale = (head ? head->rest : 1.0f) * (out ? 1.0f / kUpX : 1.0f);
    add_old(tile, old.p + j0 * old.ld + i0, old.ld, old.next, parts, rows - j0, cols - i0, one * scale, two * scale);
    if (out) tile.template store<true>(static_cast<Mem *>(out) + j0 * ldo + i0, ldo, out_rows - j0, out_cols - i0, [&](int m, int n) { return quad_of<TYPE>(tile.acc[m][n]); });
    else store_parts<2>(tile, now.p + j0 * now.ld + i0, now.ld, now.next, rows - j0, cols - i0);
}

// ---- host ----------------------------------------------------------------------
constexpr int64_t kLongest = 1 << 20, kShortest = 1 << 15;

// Where everything lies.  side: the shorter side in whole steps of the products; rows, cols: X's, with zeros behind the matrix's.  A matrix is held in
// planes, one a part of its numbers.  small: whether the steps go through the small matrices.
struct OrthogonalPlan {
    bool tall, small;
    int64_t side, rows, cols, x_ld, x_next, x_bytes, a_ld, a_next, a_bytes, matrices, sums_bytes;
    GramPlan first, gram, square, pair;      // A of what was given, A of X, products of small matrices, two of them
    int64_t bytes() const { return static_cast<int64_t>(sizeof(OrthogonalHead)) + 2 * x_bytes + matrices * a_bytes + sums_bytes; }
};
// Numbers from one row to the next: 128 bytes off whole multiples of 1024, so that the rows of a tile do not all begin at one channel of the cache.
static int64_t apart(int64_t cols) { return cols % 512 ? cols : cols + 64; }
template <int TYPE>
static OrthogonalPlan plan_of(int64_t n, int64_t d)
{
    OrthogonalPlan p{};
    p.tall = n > d;
    p.side = ceil_div(p.tall ? d : n, 32) * 32;
    p.rows = p.tall ? n : p.side;
    p.cols = p.tall ? p.side : ceil_div(d, 32) * 32;
    p.small = TYPE != DQ_F32 && small_matrices(p.side, std::max(p.rows, p.cols), TYPE == DQ_F16);
    p.x_ld = apart(p.cols);
    p.x_next = p.rows * p.x_ld;
    p.x_bytes = ceil_div(2 * 2 * p.x_next, 16) * 16;
    p.a_ld = apart(p.side);
    p.a_next = p.side * p.a_ld;
    p.a_bytes = 2 * 2 * p.a_next;
    p.matrices = p.small ? 6 : 2;
    const int64_t k = p.tall ? p.rows : p.cols;
    int64_t floats = 0;
    auto plan = [&](int64_t deep, int products, int jobs) {
        const GramPlan g = gram_plan(p.side, deep, products, jobs);
        if (!g.at_once) floats = std::max(floats, g.floats() * jobs);
        return g;
    };
    p.gram = plan(k, 3, 1);
    if (TYPE != DQ_F32) p.first = plan(k, 1, 1);
    p.square = plan(p.side, 3, 1);
    if (p.small) p.pair = plan(p.side, 3, 2);
    p.sums_bytes = 4 * floats;
    return p;
}

static Operand operand_of(const Parts &m, int64_t rows, int64_t cols)
{
    return Operand{reinterpret_cast<const char *>(m.p), m.ld * 2, rows, static_cast<int32_t>(cols), m.next * 2, nullptr, 0};
}

// One or two products over k.  IN, OUT: parts of their factors' and of the results' numbers.
template <int IN, int OUT, int HOW>
static int32_t gram(const OrthogonalPlan &p, const GramPlan &g, int64_t k, float *sums, const GramJobs &jobs, int count, hipStream_t st)
{
    if (g.at_once) {
        const unsigned tiles = static_cast<unsigned>(ceil_div(p.side, 64));
        orthogonal_gram_kernel<IN, OUT, HOW><<<dim3(tiles, tiles, static_cast<unsigned>(count)), 256, 0, st>>>(jobs, k, p.side);
        DQ_LAUNCH_CHECK();
        return DQ_OK;
    }
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(g.tiles) * g.splits * count), patches = static_cast<unsigned>(ceil_div(p.side, 64) * (ceil_div(p.side, 64) + 1) / 2);
    if (g.size == kTileLarge) orthogonal_gram_sums_kernel<IN, kTileLarge, HOW><<<blocks, 512, 0, st>>>(jobs, k, g, sums);
    else if (g.size == kTileMiddle) orthogonal_gram_sums_kernel<IN, kTileMiddle, HOW><<<blocks, 256, 0, st>>>(jobs, k, g, sums);
    else if constexpr (IN == 2 && HOW != kMixed) orthogonal_gram_sums_kernel<IN, kTileFew, HOW><<<blocks, 256, 0, st>>>(jobs, k, g, sums);
    else return DQ_ERR_UNSUPPORTED;                              // (not planned)
    DQ_LAUNCH_CHECK();
    orthogonal_gram_end_kernel<OUT><<<dim3(patches, static_cast<unsigned>(count)), 256, 0, st>>>(jobs, sums, g, p.side);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

// OF_X, OF_B: parts of their numbers that are multiplied; added: parts of X that are added `one` times.
template <int TYPE, bool TALL, int OF_X, int OF_B>
static int32_t update(const OrthogonalPlan &p, const Parts &now, const Parts &b, int added, float one, float two, const Parts &next, const OrthogonalHead *head, void *out, int64_t ldo,
                      int64_t n, int64_t d, hipStream_t st)
{
    constexpr int PX = TALL ? OF_B : OF_X, PY = TALL ? OF_X : OF_B;
    const TileSize size = update_tile(p.cols, p.rows);
    const TileDims t = dims_of(size, false, false);
    const int tiles_x = static_cast<int>(ceil_div(p.cols, t.x)), tiles_y = static_cast<int>(ceil_div(p.rows, t.y));
    const unsigned grid = static_cast<unsigned>(tiles_x) * static_cast<unsigned>(tiles_y);
    const Operand small = operand_of(b, p.side, p.side), large = operand_of(now, p.rows, p.cols);
#define DQ_UPDATE TALL ? small : large, TALL ? large : small, p.side, now, added, p.rows, p.cols, one, two, head, tiles_x, tiles_y, next, out, ldo, n, d
    if (size == kTileLarge) orthogonal_update_kernel<TYPE, kTileLarge, TALL, PX, PY><<<grid, 512, 0, st>>>(DQ_UPDATE);
    else if (size == kTileMiddle) orthogonal_update_kernel<TYPE, kTileMiddle, TALL, PX, PY><<<grid, 256, 0, st>>>(DQ_UPDATE);
    else orthogonal_update_kernel<TYPE, kTileFew, TALL, PX, PY><<<grid, 256, 0, st>>>(DQ_UPDATE);
#undef DQ_UPDATE
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

template <int TYPE, bool TALL>
static int32_t orthogonalize(const OrthogonalPlan &p, const void *v, int64_t n, int64_t d, int64_t ld, int32_t steps, void *out, int64_t ldo, uint32_t *status, char *ws, hipStream_t st)
{
    typedef typename Num<TYPE>::Mem Mem;
    OrthogonalHead *const head = reinterpret_cast<OrthogonalHead *>(ws);
    char *at = ws + sizeof(OrthogonalHead);
    auto take = [&](int64_t bytes, int64_t ld_, int64_t next) {
        const Parts parts{reinterpret_cast<u16 *>(at), ld_, next};
        at += bytes;
        return parts;
    };
    const Parts x[2] = {take(p.x_bytes, p.x_ld, p.x_next), take(p.x_bytes, p.x_ld, p.x_next)};
    Parts m[6] = {};
    for (int i = 0; i < p.matrices; ++i) m[i] = take(p.a_bytes, p.a_ld, p.a_next);
    float *const sums = reinterpret_cast<float *>(at);
    const int64_t k = TALL ? p.rows : p.cols;
    auto whole = [&](const Parts &of) { return operand_of(of, p.rows, p.cols); };
    auto small = [&](const Parts &of) { return operand_of(of, p.side, p.side); };
    orthogonal_square_kernel<TYPE><<<kNormBlocks, 256, 0, st>>>(static_cast<const Mem *>(v), n, static_cast<uint32_t>(d), ld, head);
    DQ_LAUNCH_CHECK();
    const unsigned pack = static_cast<unsigned>(std::min<int64_t>(ceil_div(p.rows * (p.cols / 8), 256), 4096));
    orthogonal_pack_kernel<TYPE><<<pack, 256, 0, st>>>(static_cast<const Mem *>(v), n, static_cast<uint32_t>(d), ld, head, x[0], p.rows, static_cast<uint32_t>(p.cols), status);
    DQ_LAUNCH_CHECK();
    int32_t done = 0;
    if constexpr (TYPE != DQ_F32) {
        if (p.small) {
            const Parts none{}, &a = m[0], &y = m[1];
            Parts all = m[2];                                       // P less its multiple of one
            done = std::min(steps, kStepsOfP);
            constexpr float kTwo = 1.0f / kUpQ;
            float power = 1.0f;                                     // kA to the step
            const GramJob first{whole(x[0]), whole(x[0]), head, kUpA / (kUpX * kUpX), 0.0f, 0.0f, none, none, a};
            if (const int32_t e = gram<1, 2, (TALL ? kAcross : kAlong)>(p, p.first, k, sums, GramJobs{{first, first}}, 1, st)) return e;
            for (int32_t step = 0; step < done; ++step) {
                const Parts &b = step ? m[3] : m[2], &next = step % 2 ? m[4] : m[5];
                const float up = step == 1 ? kUpQ : kUpP;           // (the first B is `all` of one step: held 2^7 times as high as the later ones)
                const GramJob square{small(a), small(a), nullptr, kC * kUpQ / (kUpA * kUpA), kB * kUpQ / kUpA, 0.0f, a, none, b};
                const GramJob once{small(a), small(b), nullptr, kTwo, kA, 0.0f, a, none, y}, twice{small(y), small(b), nullptr, kTwo, kA, 0.0f, y, none, a};
                const GramJob of_all{small(all), small(b), nullptr, kUpP / up * kTwo, kA * kUpP / up, power * kUpP / kUpQ, all, b, next};
                const bool more = step + 1 < done;
                if (const int32_t e = gram<2, 2, kMixed>(p, p.square, p.side, sums, GramJobs{{square, square}}, 1, st)) return e;
                if (more && step && gram_together(p.square)) {
                    if (const int32_t e = gram<2, 2, kMixed>(p, p.pair, p.side, sums, GramJobs{{once, of_all}}, 2, st)) return e;
                } else {
                    if (more)
                        if (const int32_t e = gram<2, 2, kMixed>(p, p.square, p.side, sums, GramJobs{{once, once}}, 1, st)) return e;
                    if (step)
                        if (const int32_t e = gram<2, 2, kMixed>(p, p.square, p.side, sums, GramJobs{{of_all, of_all}}, 1, st)) return e;
                }
                if (more)
                    if (const int32_t e = gram<2, 2, kMixed>(p, p.square, p.side, sums, GramJobs{{twice, twice}}, 1, st)) return e;
                if (step) all = next;
                power *= kA;
            }
            if (const int32_t e = update<TYPE, TALL, 1, 2>(p, x[0], all, 1, power, 1.0f / (done == 1 ? kUpQ : kUpP), x[1], head, done == steps ? out : nullptr, ldo, n, d, st)) return e;
        }
    }
    for (int32_t step = done; step < steps; ++step) {
        const int i = (step - done + (done ? 1 : 0)) & 1;
        const Parts &now = x[i], &next = x[i ^ 1], &a = m[0], &b = m[1];
        const OrthogonalHead *const first = TYPE != DQ_F32 && step == 0 ? head : nullptr;
        void *const last = step + 1 == steps ? out : nullptr;
        const GramJob of_x{whole(now), whole(now), first, kUpA / (kUpX * kUpX), 0.0f, 0.0f, Parts{}, Parts{}, a};
        const GramJob square{small(a), small(a), nullptr, kC * kUpB / (kUpA * kUpA), kB * kUpB / kUpA, 0.0f, a, Parts{}, b};
        auto one_step = [&](auto parts, const GramPlan &plan) -> int32_t {          // parts of X
            constexpr int kOfX = decltype(parts)::value;
            if (const int32_t e = gram<kOfX, 2, (TALL ? kAcross : kAlong)>(p, plan, k, sums, GramJobs{{of_x, of_x}}, 1, st)) return e;
            if (const int32_t e = gram<2, 2, kMixed>(p, p.square, p.side, sums, GramJobs{{square, square}}, 1, st)) return e;
            return update<TYPE, TALL, kOfX, 2>(p, now, b, kOfX, kA, 1.0f / kUpB, next, first, last, ldo, n, d, st);
        };
        if constexpr (TYPE == DQ_BF16) {
            if (step == 0) {                                        // what was given is exact in one
                if (const int32_t e = one_step(std::integral_constant<int, 1>(), p.first)) return e;
                continue;
            }
        }
        if (const int32_t e = one_step(std::integral_constant<int, 2>(), p.gram)) return e;
    }
    return DQ_OK;
}

}  // namespace dq

extern "C" int64_t dq_orthogonalize_bytes(int32_t type, int64_t n, int64_t d)
{
    if (n <= 0 || d <= 0 || !dq::typed(type)) return DQ_ERR_INVALID_ARG;
    if (std::max(n, d) > dq::kLongest || std::min(n, d) > dq::kShortest) return DQ_ERR_UNSUPPORTED;
    return type == DQ_F32 ? dq::plan_of<DQ_F32>(n, d).bytes() : type == DQ_F16 ? dq::plan_of<DQ_F16>(n, d).bytes() : dq::plan_of<DQ_BF16>(n, d).bytes();
}

extern "C" int32_t dq_orthogonalize(const void *v, int32_t type, int64_t n, int64_t d, int64_t ld, int32_t steps, void *out, int64_t ldo, uint32_t *status, void *ws,
                                    int64_t ws_bytes, void *stream)
{
    const int64_t bytes = dq_orthogonalize_bytes(type, n, d);
    if (bytes < 0) return static_cast<int32_t>(bytes);
    if (const int32_t e = dq::check_matrix(v, type, d, ld)) return e;
    if (const int32_t e = dq::check_matrix(out, type, d, ldo)) return e;
    if (steps < 1 || steps > 64 || !ws || !dq::aligned16(ws)) return DQ_ERR_INVALID_ARG;
    if (ws_bytes < bytes) return DQ_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char *const at = static_cast<char *>(ws);
#define DQ_ORTHOGONALIZE(TYPE) \
    { \
        const dq::OrthogonalPlan p = dq::plan_of<TYPE>(n, d); \
        return p.tall ? dq::orthogonalize<TYPE, true>(p, v, n, d, ld, steps, out, ldo, status, at, st) : dq::orthogonalize<TYPE, false>(p, v, n, d, ld, steps, out, ldo, status, at, st); \
    }
    switch (type) {
    case DQ_F32: DQ_ORTHOGONALIZE(DQ_F32)
    case DQ_F16: DQ_ORTHOGONALIZE(DQ_F16)
    default: DQ_ORTHOGONALIZE(DQ_BF16)
    }
#undef DQ_ORTHOGONALIZE
}
