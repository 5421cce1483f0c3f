// Matrices in 8-bit blocks: quantization along rows and along columns, its inverse, and products of two such matrices on the matrix cores,
// which multiply the codes as they are stored and apply the scales.
#include "fp8_codes.h"
#include "fp8_tile.h"

namespace dq {

// A thread takes eight numbers, sixteen neighbouring lanes a block.  Bound by memory: 8192 x 4096 in bfloat16 (101 MB) 19 to 22 us.
template <int TYPE>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, int64_t rows, uint32_t d, int64_t ld,
                                                           uint8_t *__restrict__ codes, int64_t ld_codes, uint8_t *__restrict__ scales,
                                                           int64_t ld_scales, uint32_t *__restrict__ status)
{
    const int64_t row0 = blockIdx.y * rows;
    const uint32_t groups = (d + kGroup8 - 1) / kGroup8, per = groups * 16, total = static_cast<uint32_t>(lesser(rows, n - row0)) * per;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;             // per is a multiple of sixteen: a block's lanes stay together
    if (i >= total) return;
    const Place p = place_of(i, per, row0);
    float x[8];
    load_eight<TYPE>(v + p.row * ld, p.at * 8, d, x);
    uint32_t byte;
    const uint2 code = quantize_eight8(x, byte);
    *reinterpret_cast<uint2 *>(codes + p.row * ld_codes + p.at * 8) = code;
    if ((p.at & 15) == 0) {
        write_scale8(scales + p.row * ld_scales, p.at / 16, groups, byte);
        if (byte == 255 && status) atomicOr(status, 1u);
    }
}

// Both ways from one reading: a block takes 128 rows of 128 columns, a thread ROWS rows of eight columns, which it quantizes twice.  The codes
// along the columns go through LDS, whose 16-byte chunks are permuted within a column so that lanes with neighbouring columns do not meet.  Bound by memory:
// 47236 x 4096 in bfloat16 (777 MB) 155 to 170 us, 4.6 to 5 TB/s (quantized one way after the other 1160 MB).
// A single tile is a chain of waits, shorter with four rows a thread (2049 x 1001, 136 tiles, 7.6 us, with eight 8.9): right for up to a tile to a compute
// unit (2048 x 5120, 640 tiles, 14.0 us, with eight 12.4).
template <int TYPE, int ROWS>
__global__ __launch_bounds__(2048 / ROWS) void fp8_quantize_both_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, uint32_t d, int64_t ld, dq_fp8 q, dq_fp8 qt,
                                                                         uint32_t *__restrict__ status)
{
    constexpr int kWaves = 32 / ROWS;
    __shared__ __attribute__((aligned(16))) uint8_t turned[kGroup8 * kGroup8];
    __shared__ uint32_t tops[kWaves][kGroup8];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, wave = threadIdx.x / kWave;
    const uint32_t groups = (d + kGroup8 - 1) / kGroup8, row_groups = static_cast<uint32_t>(groups8_of(n));
    const uint32_t row_group = blockIdx.x / groups, group = blockIdx.x - row_group * groups, col0 = group * kGroup8 + tx * 8;
    const int64_t row0 = static_cast<int64_t>(row_group) * kGroup8 + ty * ROWS;
    float x[ROWS][8];
    Eight<TYPE> asked[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) asked[i] = ask_eight<TYPE>(v + lesser(row0 + i, n - 1) * ld, col0, d);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        values_of<TYPE>(asked[i], x[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = row0 + i < n ? x[i][e] : 0.0f;
    }
    bool bad = false;
    if (q.codes) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            uint32_t byte;
            const uint2 code = quantize_eight8(x[i], byte);
            if (row0 + i >= n) continue;
            *reinterpret_cast<uint2 *>(q.codes + (row0 + i) * q.ld_codes + col0) = code;
            if (tx == 0) write_scale8(q.scales + (row0 + i) * q.ld_scales, group, groups, byte);
            bad |= byte == 255;
        }
    }
    uint32_t top[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        top[e] = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) top[e] = max(top[e], magnitude(x[i][e]));
        top[e] = max(top[e], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[e]), 16)));
        top[e] = max(top[e], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[e]), 32)));
        if ((threadIdx.x & 48) == 0) tops[wave][tx * 8 + e] = top[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = tx * 8 + e;
        uint32_t all = tops[0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) all = max(all, tops[w][c]);
        const uint32_t byte = scale8_byte(all);
        float column[8] = {};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) column[i] = x[i][e];
        const uint2 code = codes_of_eight(column, byte);
        uint8_t *const to = turned + c * kGroup8 + ((ty * ROWS) ^ ((tx & 7) * 16));
        if constexpr (ROWS == 8) *reinterpret_cast<uint2 *>(to) = code;
        else *reinterpret_cast<uint32_t *>(to) = code.x;
        if (ty == 0 && col0 + e < d) write_scale8(qt.scales + static_cast<int64_t>(col0 + e) * qt.ld_scales, row_group, row_groups, byte);
        bad |= byte == 255;
    }
    if (bad && status) atomicOr(status, 1u);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ROWS / 2; ++i) {
        const int id = i * (2048 / ROWS) + threadIdx.x, c = id >> 3, chunk = id & 7;
        if (group * kGroup8 + c >= d) continue;
        const i32x4 codes = *reinterpret_cast<const i32x4 *>(turned + c * kGroup8 + ((chunk ^ ((c >> 3) & 7)) * 16));
        *reinterpret_cast<i32x4 *>(qt.codes + static_cast<int64_t>(group * kGroup8 + c) * qt.ld_codes + static_cast<int64_t>(row_group) * kGroup8 + chunk * 16) = codes;
    }
}

// The inverse: eight numbers a thread.  47236 x 4096 to bfloat16 (582 MB) 95 to 100 us, 5.8 TB/s with half of the codes in the cache yet.
template <int TYPE>
__global__ __launch_bounds__(256) void fp8_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t ld_codes, const uint8_t *__restrict__ scales,
                                                             int64_t ld_scales, int64_t n, int64_t rows, uint32_t d, typename Num<TYPE>::Mem *__restrict__ out,
                                                             int64_t ld)
{
    const int64_t row0 = blockIdx.y * rows;
    const uint32_t per = (d + 7) / 8, total = static_cast<uint32_t>(lesser(rows, n - row0)) * per, i = blockIdx.x * 256u + threadIdx.x;
    if (i >= total) return;
    const Place p = place_of(i, per, row0);
    const uint2 code = *reinterpret_cast<const uint2 *>(codes + p.row * ld_codes + p.at * 8);
    const uint32_t byte = scales[p.row * ld_scales + p.at / 16];
    // the number times the scale, exact down to float32's smallest (a scale of 255: not a number, times zero too)
    const float scale = byte == 255 ? __uint_as_float(0x7fc00000u) : scale8_value(byte);
    float x[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h ? code.y : code.x, 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h ? code.y : code.x, 1.0f, true);
        x[4 * h] = lo[0] * scale;
        x[4 * h + 1] = lo[1] * scale;
        x[4 * h + 2] = hi[0] * scale;
        x[4 * h + 3] = hi[1] * scale;
    }
    store_eight<TYPE>(out + p.row * ld + p.at * 8, x, static_cast<int>(d - p.at * 8));
}

// Sixteen numbers of a block as bfloat16, which holds them exactly, scale and all.
struct Sixteen {
    i32x4 lo, hi;
};
__device__ __forceinline__ Sixteen sixteen_of(i32x4 codes, float scale)
{
    Sixteen r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = static_cast<uint32_t>(codes[i]);
        const int a = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false)), b = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true));
        (i < 2 ? r.lo : r.hi)[i % 2 * 2] = a;
        (i < 2 ? r.lo : r.hi)[i % 2 * 2 + 1] = b;
    }
    return r;
}
__device__ __forceinline__ float number_scale(uint32_t byte) { return byte == 255 ? __uint_as_float(0x7fc00000u) : scale8_value(byte); }

// Sixteen rows of w times one row of a or two: four wavefronts take every fourth block of k, and their sums are added in LDS, so that a compute unit reads
// whole rows of w one behind the other.  1 x 47236 x 4096 with w in memory, not in the cache: 45 us (4.3 TB/s; strips of 64 47); of sixteen rows, which each
// wavefront would read, 68.  (Which numbers of a block a lane holds is the same for both operands, which is all that a sum needs.)  Bound by w's
// codes, which are read once.  sums: of blocks per_split * blockIdx.y and on, for a second launch.
template <int TYPE>
__global__ __launch_bounds__(256) void fp8_fewest_kernel(dq_fp8 w, dq_fp8 a, int per_split, typename Num<TYPE>::Mem *__restrict__ out, int64_t ld, float *__restrict__ sums)
{
    __shared__ f32x4 shared[4][kWave];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, j = lane & 15, g = lane >> 4;
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 16, x = lesser(i0 + j, w.n - 1), y = lesser(j, a.n - 1);       // (results of rows past the last are not stored)
    const int first = blockIdx.y * per_split, last = min(first + per_split, static_cast<int>(groups8_of(w.d)));
    const uint8_t *const wc = w.codes + x * w.ld_codes + g * 16, *const ws = w.scales + x * w.ld_scales, *const ac = a.codes + y * a.ld_codes + g * 16, *const as = a.scales + y * a.ld_scales;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (int b = first + wave; b < last; b += 4) {
        const float sx = number_scale(ws[b]), sy = number_scale(as[b]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Sixteen p = sixteen_of(*reinterpret_cast<const i32x4 *>(wc + b * kGroup8 + h * 64), sx), q = sixteen_of(*reinterpret_cast<const i32x4 *>(ac + b * kGroup8 + h * 64), sy);
            acc = MulBf16::mul(p.lo, q.lo, acc);
            acc = MulBf16::mul(p.hi, q.hi, acc);
        }
    }
    shared[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int u = 1; u < 4; ++u) acc += shared[u][lane];
    const int64_t i = i0 + g * 4;
    if (j >= a.n || i >= w.n) return;
    const int have = static_cast<int>(lesser(w.n - i, 4));
    if (sums) store_four<DQ_F32>(sums + (blockIdx.y * a.n + j) * w.n + i, acc, have, w.n % 4 == 0);
    else store_four<TYPE>(out + j * ld + i, acc, have, false);
}

// 64 rows of w, sixteen a wavefront, times 16 SY rows of a (64 blockIdx.z and on).  GROUPS blocks of k at a time: the rows' go to LDS as bfloat16, which all wavefronts read, w's stay in
// registers; the next are asked for before these are multiplied.  Bound by w's codes, which are read once: 16 x 47236 x 4096 48 us, 64 66 (loads past the cache: 53 and 72).  sums: of blocks per_split * blockIdx.y and on, for
// a second launch.
template <int TYPE, int SY>
__global__ __launch_bounds__(256) void fp8_few_kernel(dq_fp8 w, dq_fp8 a, int per_split, typename Num<TYPE>::Mem *__restrict__ out, int64_t ld, float *__restrict__ sums)
{
    constexpr int GROUPS = SY == 4 ? 2 : 4, kRow = GROUPS * 256 + 16, kAsked = SY * GROUPS / 2;     // (bytes of a row in LDS: rows 16 bytes apart in the banks)
    __shared__ __attribute__((aligned(16))) char rows[SY * 16 * kRow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, j = lane & 15, g = lane >> 4;
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64 + wave * 16, x = lesser(i0 + j, w.n - 1);       // (results of rows past the last are not stored)
    const int first = blockIdx.y * per_split, last = min(first + per_split, static_cast<int>(groups8_of(w.d)));
    const int64_t row0 = blockIdx.z * kFewRows8;
    const uint8_t *const wc = w.codes + x * w.ld_codes + g * 16, *const ws = w.scales + x * w.ld_scales;
    i32x4 p[GROUPS][2], q[kAsked];
    uint32_t sp[GROUPS], sq[kAsked];
    auto ask = [&](int b) {
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int at = min(b + u, last - 1);                 // (behind the last: it again, times zeros)
            p[u][0] = *reinterpret_cast<const i32x4 *>(wc + at * kGroup8);
            p[u][1] = *reinterpret_cast<const i32x4 *>(wc + at * kGroup8 + 64);
            sp[u] = ws[at];
        }
#pragma unroll
        for (int i = 0; i < kAsked; ++i) {
            const int id = i * 256 + threadIdx.x, chunk = id % (GROUPS * 8), at = min(b + chunk / 8, last - 1);
            const int64_t y = lesser(row0 + id / (GROUPS * 8), a.n - 1);
            q[i] = *reinterpret_cast<const i32x4 *>(a.codes + y * a.ld_codes + at * kGroup8 + chunk % 8 * 16);
            sq[i] = a.scales[y * a.ld_scales + at];
        }
    };
    f32x4 acc[SY] = {};
    ask(first);
    for (int b = first; b < last; b += GROUPS) {
#pragma unroll
        for (int i = 0; i < kAsked; ++i) {
            const int id = i * 256 + threadIdx.x, chunk = id % (GROUPS * 8);
            Sixteen y = sixteen_of(q[i], number_scale(sq[i]));
            if (b + chunk / 8 >= last) y = Sixteen{};
            i32x4 *const to = reinterpret_cast<i32x4 *>(rows + id / (GROUPS * 8) * kRow + chunk * 32);
            to[0] = y.lo;
            to[1] = y.hi;
        }
        Sixteen xs[GROUPS][2];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) xs[u][h] = sixteen_of(p[u][h], b + u < last ? number_scale(sp[u]) : 1.0f);
        __syncthreads();
        if (b + GROUPS < last) ask(b + GROUPS);
#pragma unroll
        for (int u = 0; u < GROUPS; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < SY; ++n) {
                    const i32x4 *const y = reinterpret_cast<const i32x4 *>(rows + (n * 16 + j) * kRow + u * 256 + h * 128 + g * 32);
                    acc[n] = MulBf16::mul(xs[u][h].lo, y[0], acc[n]);
                    acc[n] = MulBf16::mul(xs[u][h].hi, y[1], acc[n]);
                }
        __syncthreads();
    }
    const int64_t i = i0 + g * 4;
    if (i >= w.n) return;
    const int have = static_cast<int>(lesser(w.n - i, 4));
#pragma unroll
    for (int n = 0; n < SY; ++n) {
        const int64_t row = row0 + n * 16 + j;
        if (row >= a.n) continue;
        if (sums) store_four<DQ_F32>(sums + (blockIdx.y * a.n + row) * w.n + i, acc[n], have, w.n % 4 == 0);
        else store_four<TYPE>(out + row * ld + i, acc[n], have, false);
    }
}

// The splits' sums added up, in their order.
template <int TYPE>
__global__ __launch_bounds__(256) void fp8_sum_kernel(const float *__restrict__ sums, int splits, int64_t n, uint32_t c, typename Num<TYPE>::Mem *__restrict__ out, int64_t ld)
{
    const int64_t all = n * c;
    for (int64_t i = (blockIdx.x * 256ll + threadIdx.x) * 4; i < all; i += gridDim.x * 1024ll) {
        const int have = static_cast<int>(lesser(all - i, 4));
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) {
            const float *const from = sums + s * all + i;
            struct __attribute__((packed, aligned(4))) Four {
                f32x4 v;
            };
            if (have == 4) {
                v += reinterpret_cast<const Four *>(from)->v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < have) v[e] += from[e];
            }
        }
        int64_t row = i / c;
        uint32_t col = static_cast<uint32_t>(i - row * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e < have) out[row * ld + col] = Num<TYPE>::store(v[e]);
            if (++col == c) {
                col = 0;
                ++row;
            }
        }
    }
}

// Many rows, results of 16 bits: the codes as they are.  How long it takes goes by the numbers, which draw different power: 8192 x 8192 x 8192, the same product
// again and again, 412 us (2670 TFLOP/s) of normally distributed numbers, 374 of whole ones from -2 to 2, 335 of ones; 8192 x 47236 x 4096 1297, 1201 and 1095 us, of which
// what is stored is some 130 (a pass on new rows into another result, their quantization of 20 us included: 1500).
template <int TYPE, int XT, int YT, int WX, int WY, int R>
__global__ __launch_bounds__(WX *WY *kWave) void fp8_tile_kernel(dq_fp8 w, dq_fp8 a, int per_split, int tiles_x, int tiles_y, typename Num<TYPE>::Mem *__restrict__ out, int64_t ld,
                                                                 float *__restrict__ sums)
{
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, j0 = static_cast<int64_t>(ty) * YT;
    const int first = blockIdx.y * per_split;
    Fp8Tile<XT, YT, WX, WY, R> tile;
    tile.run(w, a, i0, j0, first, min(first + per_split, static_cast<int>(groups8_of(w.d))));
    if (sums) tile.store_sums(sums + (blockIdx.y * a.n + j0) * w.n + i0, w.n, a.n - j0, w.n - i0);
    else tile.template store<TYPE>(out + j0 * ld + i0, ld, a.n - j0, w.n - i0);
}

// Many rows, float32 results: the numbers in bfloat16, which holds them exactly.  8192 x 8192 x 8192 944 us with the 0.4 GB that are written for it, 1165 TFLOP/s.
template <int UNUSED, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave) void fp8_wide_product_kernel(Operand w, Operand a, int64_t k, int64_t per_split, int tiles_x, int tiles_y, float *__restrict__ out, int64_t ld)
{
    typedef TileProduct<MulBf16, XT, YT, WX, WY, false, false, H, R, P> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, j0 = static_cast<int64_t>(ty) * YT;
    Tile tile;
    tile.run(w, a, i0, j0, blockIdx.y * per_split, lesser(k, (blockIdx.y + 1) * per_split));
    tile.store(out + (blockIdx.y * a.rows + j0) * ld + i0, ld, a.rows - j0, w.rows - i0, [&](int m, int n) { return quad_of<DQ_F32>(tile.acc[m][n]); });
}

// ---- host ----------------------------------------------------------------------
template <int TYPE>
static int32_t quantize8(const void *v, int64_t n, int64_t d, int64_t ld, const dq_fp8 *q, const dq_fp8 *qt, uint32_t *status, hipStream_t st)
{
    typedef typename Num<TYPE>::Mem Mem;
    if (qt) {
        const unsigned blocks = static_cast<unsigned>(groups8_of(d) * groups8_of(n));
        if (blocks <= 256) fp8_quantize_both_kernel<TYPE, 4><<<blocks, 512, 0, st>>>(static_cast<const Mem *>(v), n, static_cast<uint32_t>(d), ld, q ? *q : dq_fp8{}, *qt, status);
        else fp8_quantize_both_kernel<TYPE, 8><<<blocks, 256, 0, st>>>(static_cast<const Mem *>(v), n, static_cast<uint32_t>(d), ld, q ? *q : dq_fp8{}, *qt, status);
    } else {
        int64_t rows;
        const dim3 blocks = blocks_of(n, groups8_of(d) * 16, 1, rows);
        fp8_quantize_kernel<TYPE><<<blocks, 256, 0, st>>>(static_cast<const Mem *>(v), n, rows, static_cast<uint32_t>(d), ld, q->codes, q->ld_codes, q->scales, q->ld_scales,
                                                          status);
    }
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
static int32_t quantize8(const void *v, int32_t type, int64_t n, int64_t d, int64_t ld, const dq_fp8 *q, const dq_fp8 *qt, uint32_t *status, hipStream_t st)
{
    switch (type) {
    case DQ_F32: return quantize8<DQ_F32>(v, n, d, ld, q, qt, status, st);
    case DQ_F16: return quantize8<DQ_F16>(v, n, d, ld, q, qt, status, st);
    default: return quantize8<DQ_BF16>(v, n, d, ld, q, qt, status, st);
    }
}

template <int TYPE>
static int32_t dequantize8(const dq_fp8 &q, void *out, int64_t ld, hipStream_t st)
{
    int64_t rows;
    const dim3 blocks = blocks_of(q.n, (q.d + 7) / 8, 1, rows);
    fp8_dequantize_kernel<TYPE><<<blocks, 256, 0, st>>>(q.codes, q.ld_codes, q.scales, q.ld_scales, q.n, rows, static_cast<uint32_t>(q.d),
                                                        static_cast<typename Num<TYPE>::Mem *>(out), ld);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

static int64_t wide_bytes(int64_t n, int64_t d) { return n * groups8_of(d) * kGroup8 * 2; }
// Whether a launch takes the product.
static bool product_fits8(const ProductPlan &p)
{
    return p.few ? launchable(p.tiles_x, 256) : launchable(p.tiles_x * p.tiles_y, threads_of(p.size));
}

// Workspace: the splits' sums; where many rows have float32 results, then w and a in bfloat16.
template <int TYPE>
static int32_t product8(const dq_fp8 &a, const dq_fp8 &w, void *out, int64_t ld, char *ws, hipStream_t st)
{
    typedef typename Num<TYPE>::Mem Mem;
    const ProductPlan p = product_plan(a.n, w.n, groups8_of(w.d), TYPE == DQ_F32);
    const int per = static_cast<int>(p.per_split), tiles_x = static_cast<int>(p.tiles_x), tiles_y = static_cast<int>(p.tiles_y);
    const unsigned splits = static_cast<unsigned>(p.splits);
    float *const sums = splits > 1 ? reinterpret_cast<float *>(ws) : nullptr;
    Mem *const to = static_cast<Mem *>(out);
    if (p.few) {
        const dim3 grid(static_cast<unsigned>(p.tiles_x), splits, static_cast<unsigned>(p.tiles_y));
        if (a.n <= kFewestRows8) fp8_fewest_kernel<TYPE><<<grid, 256, 0, st>>>(w, a, per, to, ld, sums);
        else if (a.n <= 16) fp8_few_kernel<TYPE, 1><<<grid, 256, 0, st>>>(w, a, per, to, ld, sums);
        else if (a.n <= 32) fp8_few_kernel<TYPE, 2><<<grid, 256, 0, st>>>(w, a, per, to, ld, sums);
        else fp8_few_kernel<TYPE, 4><<<grid, 256, 0, st>>>(w, a, per, to, ld, sums);
    } else if constexpr (TYPE == DQ_F32) {
        const int64_t wide = groups8_of(w.d) * kGroup8;
        const dq_fp8 whole_w{w.n, wide, w.codes, w.ld_codes, w.scales, w.ld_scales}, whole_a{a.n, wide, a.codes, a.ld_codes, a.scales, a.ld_scales};
        char *const ww = ws + p.sums_bytes(a.n, w.n), *const wa = ww + wide_bytes(w.n, w.d);
        if (const int32_t e = dequantize8<DQ_BF16>(whole_w, ww, wide, st)) return e;
        if (const int32_t e = dequantize8<DQ_BF16>(whole_a, wa, wide, st)) return e;
        const Operand x{ww, wide * 2, w.n, static_cast<int32_t>(wide), 0, nullptr, 0}, y{wa, wide * 2, a.n, static_cast<int32_t>(wide), 0, nullptr, 0};
        constexpr bool kInParts = false;
        const dim3 grid(static_cast<unsigned>(p.tiles_x * p.tiles_y), splits);
        float *const into = sums ? sums : to;
        const int64_t stride = sums ? w.n : ld;
        if (p.size == kTileLarge) DQ_TILE_LAUNCH(fp8_wide_product_kernel, 0, Large, x, y, wide, p.per_split * kGroup8, tiles_x, tiles_y, into, stride);
        else DQ_TILE_LAUNCH(fp8_wide_product_kernel, 0, Middle, x, y, wide, p.per_split * kGroup8, tiles_x, tiles_y, into, stride);
    } else {
        const dim3 grid(static_cast<unsigned>(p.tiles_x * p.tiles_y), splits);
        if (p.size == kTileLarge) fp8_tile_kernel<TYPE, 256, 256, 2, 4, 2><<<grid, 512, 0, st>>>(w, a, per, tiles_x, tiles_y, to, ld, sums);
        else if (p.tiles_x * p.tiles_y * p.splits <= 256) fp8_tile_kernel<TYPE, 128, 128, 2, 2, 4><<<grid, 256, 0, st>>>(w, a, per, tiles_x, tiles_y, to, ld, sums);
        else fp8_tile_kernel<TYPE, 128, 128, 2, 2, 2><<<grid, 256, 0, st>>>(w, a, per, tiles_x, tiles_y, to, ld, sums);
    }
    DQ_LAUNCH_CHECK();
    if (!sums) return DQ_OK;
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(ceil_div(a.n * w.n, 1024), 4096));
    fp8_sum_kernel<TYPE><<<blocks, 256, 0, st>>>(sums, static_cast<int>(splits), a.n, static_cast<uint32_t>(w.n), to, ld);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
static int32_t product8(const dq_fp8 &a, const dq_fp8 &w, void *out, int32_t type, int64_t ld, void *ws, hipStream_t st)
{
    char *const at = static_cast<char *>(ws);
    switch (type) {
    case DQ_F32: return product8<DQ_F32>(a, w, out, ld, at, st);
    case DQ_F16: return product8<DQ_F16>(a, w, out, ld, at, st);
    default: return product8<DQ_BF16>(a, w, out, ld, at, st);
    }
}

}  // namespace dq

extern "C" int64_t dq_fp8_row_bytes(int64_t d) { return d <= 0 ? DQ_ERR_INVALID_ARG : dq::groups8_of(d) * dq::kGroup8; }
extern "C" int64_t dq_fp8_row_scales(int64_t d) { return d <= 0 ? DQ_ERR_INVALID_ARG : dq::scales8_of(d); }

extern "C" int32_t dq_fp8_quantize(const void *v, int32_t type, int64_t n, int64_t d, int64_t ld, const dq_fp8 *q, const dq_fp8 *qt, uint32_t *status, void *stream)
{
    if ((!q && !qt) || n <= 0 || d <= 0) return DQ_ERR_INVALID_ARG;
    if (q)
        if (const int32_t e = dq::check8(q)) return e;
    if (qt)
        if (const int32_t e = dq::check8(qt)) return e;
    if (qt && !dq::launchable(dq::groups8_of(d) * dq::groups8_of(n), 256)) return DQ_ERR_UNSUPPORTED;
    if ((q && (q->n != n || q->d != d)) || (qt && (qt->n != d || qt->d != n))) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = dq::check_matrix(v, type, d, ld)) return e;
    return dq::quantize8(v, type, n, d, ld, q, qt, status, static_cast<hipStream_t>(stream));
}

extern "C" int32_t dq_fp8_dequantize(const dq_fp8 *q, void *out, int32_t type, int64_t ld, void *stream)
{
    if (const int32_t e = dq::check8(q)) return e;
    if (const int32_t e = dq::check_matrix(out, type, q->d, ld)) return e;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (type) {
    case DQ_F32: return dq::dequantize8<DQ_F32>(*q, out, ld, st);
    case DQ_F16: return dq::dequantize8<DQ_F16>(*q, out, ld, st);
    default: return dq::dequantize8<DQ_BF16>(*q, out, ld, st);
    }
}

extern "C" int64_t dq_fp8_product_bytes(int32_t type, int64_t n, int64_t c, int64_t d)
{
    if (n <= 0 || c <= 0 || d <= 0 || !dq::typed(type)) return DQ_ERR_INVALID_ARG;
    if (n > dq::kMost8 || c > dq::kMost8 || d > dq::kWidest8) return DQ_ERR_UNSUPPORTED;
    const dq::ProductPlan p = dq::product_plan(n, c, dq::groups8_of(d), type == DQ_F32);
    if (!dq::product_fits8(p)) return DQ_ERR_UNSUPPORTED;
    return p.sums_bytes(n, c) + (type == DQ_F32 && !p.few ? dq::wide_bytes(n, d) + dq::wide_bytes(c, d) : 0);
}

extern "C" int32_t dq_fp8_product(const dq_fp8 *a, const dq_fp8 *w, void *out, int32_t type, int64_t ld, void *ws, int64_t ws_bytes, void *stream)
{
    if (const int32_t e = dq::check8(a)) return e;
    if (const int32_t e = dq::check8(w)) return e;
    if (a->d != w->d) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = dq::check_matrix(out, type, w->n, ld)) return e;
    const int64_t bytes = dq_fp8_product_bytes(type, a->n, w->n, a->d);
    if (bytes < 0) return static_cast<int32_t>(bytes);
    if (bytes && (!ws || !dq::aligned16(ws))) return DQ_ERR_INVALID_ARG;
    if (bytes && ws_bytes < bytes) return DQ_ERR_WORKSPACE;
    return dq::product8(*a, *w, out, type, ld, ws, static_cast<hipStream_t>(stream));
}

// Workspace of the scores: the product's, then the rows' codes and scales.
extern "C" int64_t dq_fp8_scores_bytes(int32_t type, int64_t n, int64_t c, int64_t d)
{
    const int64_t bytes = dq_fp8_product_bytes(type, n, c, d);
    return bytes < 0 ? bytes : (bytes + 15) / 16 * 16 + (n * (dq_fp8_row_bytes(d) + dq_fp8_row_scales(d)) + 15) / 16 * 16;
}

extern "C" int32_t dq_fp8_scores(const void *a, int32_t type, int64_t n, int64_t lda, const dq_fp8 *w, void *out, int32_t out_type, int64_t ld, uint32_t *status,
                                 void *ws, int64_t ws_bytes, void *stream)
{
    if (const int32_t e = dq::check8(w)) return e;
    const int64_t product = dq_fp8_product_bytes(out_type, n, w->n, w->d), row = dq_fp8_row_bytes(w->d);
    if (product < 0) return static_cast<int32_t>(product);
    if (const int32_t e = dq::check_matrix(a, type, w->d, lda)) return e;
    if (const int32_t e = dq::check_matrix(out, out_type, w->n, ld)) return e;
    if (!ws || !dq::aligned16(ws)) return DQ_ERR_INVALID_ARG;
    if (ws_bytes < dq_fp8_scores_bytes(out_type, n, w->n, w->d)) return DQ_ERR_WORKSPACE;
    uint8_t *const codes = static_cast<uint8_t *>(ws) + (product + 15) / 16 * 16;
    const dq_fp8 q{n, w->d, codes, row, codes + n * row, dq_fp8_row_scales(w->d)};
    if (const int32_t e = dq::check8(&q)) return e;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (const int32_t e = dq::quantize8(a, type, n, w->d, lda, &q, nullptr, status, st)) return e;
    return dq::product8(q, *w, out, out_type, ld, ws, st);
}
