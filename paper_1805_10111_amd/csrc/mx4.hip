// Models in 4 bits: microscaled quantization (levels +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, one power-of-two scale per 32 neighbours), its
// inverse, and products of two such matrices on the matrix cores, which multiply the codes as they are stored.
#include <algorithm>

#include "dq_common.h"
#include "matrix_tile.h"

namespace dq {

typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kGroup4 = 128;                   // numbers of a row that are stored together: 64 bytes of codes, 4 scales

__host__ __device__ static inline int64_t groups_of(int64_t d) { return (d + kGroup4 - 1) / kGroup4; }

// floor(log2 amax) - 2 as a scale byte: the exponent field less 2, at least 0 (below 2^-125 the largest level is not used); 255 where
// the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits)
{
    const uint32_t e = amax_bits >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// Eight numbers of a row from column c on, zeros behind its end.  (16-byte loads of any alignment to the number.)
template <int TYPE>
__device__ __forceinline__ void load_eight(const typename Num<TYPE>::Mem *row, uint32_t c, uint32_t d, float out[8])
{
    typedef typename Num<TYPE>::Mem Mem;
    if (c + 8 <= d) {
        struct __attribute__((packed, aligned(sizeof(Mem)))) All {
            __attribute__((ext_vector_type(8))) Mem v;
        };
        const All all = *reinterpret_cast<const All *>(row + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = Num<TYPE>::load(all.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = c + e < d ? Num<TYPE>::load(row[c + e]) : 0.0f;
    }
}

// The codes of eight numbers, and the scale byte of the 32 that four neighbouring lanes hold.
__device__ __forceinline__ uint32_t quantize_eight(const float v[8], uint32_t &byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
    byte = scale_byte(top);
    if (byte == 255) return 0;
    const float scale = scale_value(byte);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], scale, 3);
    return code;
}

// Item i of rows of `per` items: its row and place there.  (Rows and items are numbered in 32 bits; where a matrix has more items, in several
// launches' worth of blocks by blockIdx.y.)
struct Place {
    int64_t row;
    uint32_t at;
};
__device__ __forceinline__ Place place_of(uint32_t i, uint32_t per, int64_t row0)
{
    const uint32_t r = i / per;
    return Place{row0 + r, i - r * per};
}

// A thread takes eight numbers: 16 or 32 bytes read, 4 written; four neighbouring lanes share a block.  What bounds it is memory: 47236 x 4096
// in bfloat16 (490 MB) 94 to 108 us on different cards, in float32 (877 MB) 154.  (Two and four items a thread, where one took 94 and 154: 90 to 95 and
// 97 to 100, 160 and 169.)
template <int TYPE>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, int64_t rows, uint32_t d, int64_t ld,
                                                           uint8_t *__restrict__ codes, int64_t ld_codes, uint8_t *__restrict__ scales,
                                                           int64_t ld_scales, uint32_t *__restrict__ status)
{
    const int64_t row0 = blockIdx.y * rows;
    const uint32_t per = (d + kGroup4 - 1) / kGroup4 * 16, total = static_cast<uint32_t>(lesser(rows, n - row0)) * per;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;             // per is a multiple of four: a block's lanes stay together
    if (i >= total) return;
    const Place p = place_of(i, per, row0);
    float x[8];
    load_eight<TYPE>(v + p.row * ld, p.at * 8, d, x);
    uint32_t byte;
    const uint32_t code = quantize_eight(x, byte);
    *reinterpret_cast<uint32_t *>(codes + p.row * ld_codes + p.at * 4) = code;
    if ((p.at & 3) == 0) {
        scales[p.row * ld_scales + p.at / 4] = static_cast<uint8_t>(byte);
        if (byte == 255 && status) atomicOr(status, 1u);
    }
}

// Eight values of a row.
template <int TYPE>
__device__ __forceinline__ void store_eight(typename Num<TYPE>::Mem *to, const float v[8], int have)
{
    typedef typename Num<TYPE>::Mem Mem;
    struct __attribute__((packed, aligned(sizeof(Mem)))) All {
        __attribute__((ext_vector_type(8))) Mem v;
    } all;
#pragma unroll
    for (int e = 0; e < 8; ++e) all.v[e] = Num<TYPE>::store(v[e]);
    if (have >= 8) {
        *reinterpret_cast<All *>(to) = all;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < have) to[e] = all.v[e];
    }
}

// The inverse, AT_ONCE items a thread requested together.  47236 x 4096 to bfloat16 (490 MB): one 107 us, two 98, four 88 (73 right behind the
// quantizer, whose codes are in the cache yet); to float32 (877 MB) 166 to 172, 220 and 228: there the stores are twice as long, and one it is.
template <int TYPE, int AT_ONCE>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t ld_codes, const uint8_t *__restrict__ scales,
                                                             int64_t ld_scales, int64_t n, int64_t rows, uint32_t d, typename Num<TYPE>::Mem *__restrict__ out,
                                                             int64_t ld)
{
    const int64_t row0 = blockIdx.y * rows;
    const uint32_t per = (d + 7) / 8, total = static_cast<uint32_t>(lesser(rows, n - row0)) * per, first = blockIdx.x * (256u * AT_ONCE) + threadIdx.x;
    uint32_t code[AT_ONCE] = {};
    int byte[AT_ONCE] = {};
    Place p[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        const uint32_t i = first + 256u * u;
        p[u] = place_of(i, per, row0);
        if (i >= total) continue;
        code[u] = *reinterpret_cast<const uint32_t *>(codes + p[u].row * ld_codes + p[u].at * 4);
        byte[u] = scales[p[u].row * ld_scales + p[u].at / 4];
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        if (first + 256u * u >= total) continue;
        // levels, exact, times the scale: exact down to float32's smallest number (a scale of 255: not a number, times zero too)
        const float scale = byte[u] == 255 ? __uint_as_float(0x7fc00000u) : scale_value(static_cast<uint32_t>(byte[u]));
        const f32x2 q[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 3)};
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = q[e >> 1][e & 1] * scale;
        store_eight<TYPE>(out + p[u].row * ld + p[u].at * 8, x, static_cast<int>(d - p[u].at * 8));
    }
}

// Few rows: bound by w's codes (1 x 47236 x 4096, 103 MB, 18 us).  Many: 8192 x 47236 x 4096 0.98 to 1.05 ms on different cards, 3020 to 3230
// TFLOP/s, the matrix cores busy 38 % of the time: a step is as many bytes of LDS, and as many cycles of the matrix cores, as in 16 bits, with the
// scales to bring there besides, and takes twice these cycles; a tile is only 32 steps; 200 us are the results' (774 MB in bfloat16).
template <int TYPE, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave) void mx4_product_kernel(Operand w, Operand a, int64_t k, int tiles_x, int tiles_y,
                                                                    typename Num<TYPE>::Mem *__restrict__ out, int64_t ld)
{
    typedef TileProduct<MulMx4, XT, YT, WX, WY, false, false, H, R, P> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, j0 = static_cast<int64_t>(ty) * YT;
    Tile tile;
    tile.run(w, a, i0, j0, 0, k);
    tile.store(out + j0 * ld + i0, ld, a.rows - j0, w.rows - i0, [&](int m, int n) { return quad_of<TYPE>(tile.acc[m][n]); });
}

// ---- host ----------------------------------------------------------------------
constexpr int64_t kMost4 = 1ll << 30;

static int wide_of(int32_t type) { return type == DQ_F32 ? 4 : 2; }
static bool typed(int32_t type) { return type == DQ_F32 || type == DQ_F16 || type == DQ_BF16; }

static int32_t check4(const dq_mx4 *q)
{
    if (!q || q->n <= 0 || q->d <= 0 || !q->codes || !q->scales || !aligned16(q->codes) || reinterpret_cast<uintptr_t>(q->scales) % 4) return DQ_ERR_INVALID_ARG;
    if (q->ld_codes % 16 || q->ld_scales % 4 || q->ld_codes < dq_mx4_row_bytes(q->d) || q->ld_scales < dq_mx4_row_scales(q->d)) return DQ_ERR_INVALID_ARG;
    if (q->n > kMost4 || q->d > (1 << 23) || q->ld_codes > (1 << 23) || q->ld_scales > (1 << 23)) return DQ_ERR_UNSUPPORTED;
    return DQ_OK;
}
static int32_t check_matrix(const void *v, int32_t type, int64_t cols, int64_t ld)
{
    if (!v || !typed(type) || ld < cols || reinterpret_cast<uintptr_t>(v) % wide_of(type)) return DQ_ERR_INVALID_ARG;
    return DQ_OK;
}
// Blocks for n rows of `per` items; rows: how many a blockIdx.y takes.
static dim3 blocks_of(int64_t n, int64_t per, int at_once, int64_t &rows)
{
    rows = std::min<int64_t>(n, std::max<int64_t>((1ll << 31) / per, (n + 65534) / 65535));
    return dim3(static_cast<unsigned>((rows * per + 256 * at_once - 1) / (256 * at_once)), static_cast<unsigned>((n + rows - 1) / rows));
}
template <int TYPE>
static int32_t quantize4(const void *v, int64_t ld, const dq_mx4 &q, uint32_t *status, hipStream_t st)
{
    int64_t rows;
    const dim3 blocks = blocks_of(q.n, groups_of(q.d) * 16, 1, rows);
    mx4_quantize_kernel<TYPE><<<blocks, 256, 0, st>>>(static_cast<const typename Num<TYPE>::Mem *>(v), q.n, rows, static_cast<uint32_t>(q.d), ld,
                                                      q.codes, q.ld_codes, q.scales, q.ld_scales, status);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
static int32_t quantize4(const void *v, int32_t type, int64_t ld, const dq_mx4 &q, uint32_t *status, hipStream_t st)
{
    switch (type) {
    case DQ_F32: return quantize4<DQ_F32>(v, ld, q, status, st);
    case DQ_F16: return quantize4<DQ_F16>(v, ld, q, status, st);
    default: return quantize4<DQ_BF16>(v, ld, q, status, st);
    }
}

template <int TYPE>
static int32_t dequantize4(const dq_mx4 &q, void *out, int64_t ld, hipStream_t st)
{
    constexpr int kAtOnce = TYPE == DQ_F32 ? 1 : 4;
    int64_t rows;
    const dim3 blocks = blocks_of(q.n, (q.d + 7) / 8, kAtOnce, rows);
    mx4_dequantize_kernel<TYPE, kAtOnce><<<blocks, 256, 0, st>>>(q.codes, q.ld_codes, q.scales, q.ld_scales, q.n, rows, static_cast<uint32_t>(q.d),
                                                        static_cast<typename Num<TYPE>::Mem *>(out), ld);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

// Whether a launch takes the product of n rows with c.
static bool product_fits(int64_t n, int64_t c)
{
    const TileSize size = tile_for_rows(c, n, false, false);
    return launchable(tiles_of(c, n, dims_of(size, false, false)), threads_of(size));
}
template <int TYPE>
static int32_t product4(const dq_mx4 &a, const dq_mx4 &w, void *out, int64_t ld, hipStream_t st)
{
    const TileSize size = tile_for_rows(w.n, a.n, false, false);
    const TileDims t = dims_of(size, false, false);
    const int64_t tiles_x = (w.n + t.x - 1) / t.x, tiles_y = (a.n + t.y - 1) / t.y;
    auto operand = [](const dq_mx4 &q) { return Operand{reinterpret_cast<const char *>(q.codes), q.ld_codes, q.n, static_cast<int32_t>(groups_of(q.d) * 32), 0, q.scales, q.ld_scales}; };
    constexpr bool kInParts = false;
    const unsigned grid = static_cast<unsigned>(tiles_x * tiles_y);
#define DQ_PRODUCT operand(w), operand(a), groups_of(a.d) * 32, static_cast<int>(tiles_x), static_cast<int>(tiles_y), static_cast<typename Num<TYPE>::Mem *>(out), ld
    switch (size) {
    case kTileLarge: DQ_TILE_LAUNCH(mx4_product_kernel, TYPE, Large, DQ_PRODUCT); break;
    case kTileMiddle: DQ_TILE_LAUNCH(mx4_product_kernel, TYPE, Middle, DQ_PRODUCT); break;
    case kTileFew: DQ_TILE_LAUNCH(mx4_product_kernel, TYPE, Few, DQ_PRODUCT); break;
    case kTileFewest: DQ_TILE_LAUNCH(mx4_product_kernel, TYPE, Fewest, DQ_PRODUCT); break;
    case kTileHalf: return DQ_ERR_UNSUPPORTED;                   // (not asked for)
    }
#undef DQ_PRODUCT
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
static int32_t product4(const dq_mx4 &a, const dq_mx4 &w, void *out, int32_t type, int64_t ld, hipStream_t st)
{
    switch (type) {
    case DQ_F32: return product4<DQ_F32>(a, w, out, ld, st);
    case DQ_F16: return product4<DQ_F16>(a, w, out, ld, st);
    default: return product4<DQ_BF16>(a, w, out, ld, st);
    }
}

}  // namespace dq

extern "C" int64_t dq_mx4_row_bytes(int64_t d) { return d <= 0 ? DQ_ERR_INVALID_ARG : dq::groups_of(d) * 64; }
extern "C" int64_t dq_mx4_row_scales(int64_t d) { return d <= 0 ? DQ_ERR_INVALID_ARG : dq::groups_of(d) * 4; }

extern "C" int32_t dq_mx4_quantize(const void *v, int32_t type, int64_t ld, const dq_mx4 *q, uint32_t *status, void *stream)
{
    if (const int32_t e = dq::check4(q)) return e;
    if (const int32_t e = dq::check_matrix(v, type, q->d, ld)) return e;
    return dq::quantize4(v, type, ld, *q, status, static_cast<hipStream_t>(stream));
}

extern "C" int32_t dq_mx4_dequantize(const dq_mx4 *q, void *out, int32_t type, int64_t ld, void *stream)
{
    if (const int32_t e = dq::check4(q)) return e;
    if (const int32_t e = dq::check_matrix(out, type, q->d, ld)) return e;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (type) {
    case DQ_F32: return dq::dequantize4<DQ_F32>(*q, out, ld, st);
    case DQ_F16: return dq::dequantize4<DQ_F16>(*q, out, ld, st);
    default: return dq::dequantize4<DQ_BF16>(*q, out, ld, st);
    }
}

extern "C" int32_t dq_mx4_product(const dq_mx4 *a, const dq_mx4 *w, void *out, int32_t type, int64_t ld, void *stream)
{
    if (const int32_t e = dq::check4(a)) return e;
    if (const int32_t e = dq::check4(w)) return e;
    if (a->d != w->d) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = dq::check_matrix(out, type, w->n, ld)) return e;
    if (!dq::product_fits(a->n, w->n)) return DQ_ERR_UNSUPPORTED;
    return dq::product4(*a, *w, out, type, ld, static_cast<hipStream_t>(stream));
}

extern "C" int64_t dq_mx4_scores_bytes(int64_t n, int64_t d)
{
    if (n <= 0 || d <= 0) return DQ_ERR_INVALID_ARG;
    if (n > dq::kMost4 || d > (1 << 23)) return DQ_ERR_UNSUPPORTED;
    return (n * (dq_mx4_row_bytes(d) + dq_mx4_row_scales(d)) + 15) / 16 * 16;
}

extern "C" int32_t dq_mx4_scores(const void *a, int32_t type, int64_t n, int64_t lda, const dq_mx4 *w, void *out, int32_t out_type, int64_t ld,
                                 uint32_t *status, void *ws, int64_t ws_bytes, void *stream)
{
    if (const int32_t e = dq::check4(w)) return e;
    if (n <= 0) return DQ_ERR_INVALID_ARG;
    if (n > dq::kMost4 || !dq::product_fits(n, w->n)) return DQ_ERR_UNSUPPORTED;
    if (const int32_t e = dq::check_matrix(a, type, w->d, lda)) return e;
    if (const int32_t e = dq::check_matrix(out, out_type, w->n, ld)) return e;
    if (!ws || !dq::aligned16(ws)) return DQ_ERR_INVALID_ARG;
    if (ws_bytes < dq_mx4_scores_bytes(n, w->d)) return DQ_ERR_WORKSPACE;
    const int64_t row = dq_mx4_row_bytes(w->d);
    uint8_t *const codes = static_cast<uint8_t *>(ws);
    const dq_mx4 q{n, w->d, codes, row, codes + n * row, dq_mx4_row_scales(w->d)};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (const int32_t e = dq::quantize4(a, type, lda, q, status, st)) return e;
    return dq::product4(q, *w, out, out_type, ld, st);
}
