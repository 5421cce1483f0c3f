// Models in 4 bits: microscaled quantization (levels +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, one power-of-two scale per 32 neighbours), its
// inverse, and products of two such matrices on the matrix cores, which multiply the codes as they are stored.
#include <algorithm>

#include "dq_common.h"
#include "matrix_tile.h"

namespace dq {

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

// Eight numbers of a row from column c on, zeros behind its end.
template <int TYPE>
__device__ __forceinline__ void load_eight(const typename Num<TYPE>::Mem *row, int64_t c, int64_t d, bool vector, float out[8])
{
    typedef typename Num<TYPE>::Mem Mem;
    typedef __attribute__((ext_vector_type(16 / sizeof(Mem)))) Mem Wide;
    constexpr int kPer = 16 / sizeof(Mem);
    if (vector && c + 8 <= d) {
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h) {
            const Wide v = *reinterpret_cast<const Wide *>(row + c + h * kPer);
#pragma unroll
            for (int e = 0; e < kPer; ++e) out[h * kPer + e] = Num<TYPE>::load(v[e]);
        }
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

// A thread takes eight numbers: 16 or 32 bytes read, 4 written; four neighbouring lanes share a block.
template <int TYPE>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const typename Num<TYPE>::Mem *__restrict__ v, int64_t n, int64_t d, int64_t ld, int vector,
                                                           uint8_t *__restrict__ codes, int64_t ld_codes, uint8_t *__restrict__ scales,
                                                           int64_t ld_scales, uint32_t *__restrict__ status)
{
    const int64_t per = groups_of(d) * 16, total = n * per;             // a multiple of four: a block's lanes stay together
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int64_t r = i / per, at = i - r * per;
        float x[8];
        load_eight<TYPE>(v + r * ld, at * 8, d, vector, x);
        uint32_t byte;
        const uint32_t code = quantize_eight(x, byte);
        *reinterpret_cast<uint32_t *>(codes + r * ld_codes + at * 4) = code;
        if ((at & 3) == 0) {
            scales[r * ld_scales + at / 4] = static_cast<uint8_t>(byte);
            if (byte == 255 && status) atomicOr(status, 1u);
        }
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t ld_codes, const uint8_t *__restrict__ scales,
                                                             int64_t ld_scales, int64_t n, int64_t d, typename Num<TYPE>::Mem *__restrict__ out,
                                                             int64_t ld, int vector)
{
    const int64_t per = (d + 7) / 8, total = n * per;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int64_t r = i / per, at = i - r * per;
        const uint32_t code = *reinterpret_cast<const uint32_t *>(codes + r * ld_codes + at * 4);
        const int byte = scales[r * ld_scales + at / 4];
        f32x4 x[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t c = (code >> (4 * e)) & 7u;
            // level = (1 + m / 2) 2^(x - 1), below 1 m / 2
            const float level = c < 2 ? 0.5f * static_cast<float>(c) : __uint_as_float(((c >> 1) + 126u) << 23 | (c & 1u) << 22);
            const float value = ldexpf(level, byte - 127);
            x[e >> 2][e & 3] = byte == 255 ? __uint_as_float(0x7fc00000u) : (code >> (4 * e)) & 8u ? -value : value;
        }
        const int have = static_cast<int>(lesser(8, d - at * 8));
        typename Num<TYPE>::Mem *const to = out + r * ld + at * 8;
        store_four<TYPE>(to, x[0], min(have, 4), vector);
        if (have > 4) store_four<TYPE>(to + 4, x[1], have - 4, vector);
    }
}

template <int TYPE, int XT, int YT, int WX, int WY, int H>
__global__ __launch_bounds__(WX *WY *kWave) void mx4_product_kernel(Operand w, Operand a, int64_t k, int tiles_x, int tiles_y,
                                                                    typename Num<TYPE>::Mem *__restrict__ out, int64_t ld)
{
    typedef TileProduct<MulMx4, XT, YT, WX, WY, false, false, H> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, j0 = static_cast<int64_t>(ty) * YT;
    Tile tile;
    tile.template run<false>(w, a, i0, j0, 0, k);
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
static unsigned blocks_of(int64_t threads) { return static_cast<unsigned>(std::clamp<int64_t>((threads + 255) / 256, 1, 1 << 20)); }
// rows of 8 numbers that can be read 16 bytes at a time
static bool wide_reads(const void *v, int32_t type, int64_t ld) { return aligned16(v) && ld * wide_of(type) % 16 == 0; }

template <int TYPE>
static int32_t quantize4(const void *v, int64_t ld, const dq_mx4 &q, uint32_t *status, hipStream_t st)
{
    mx4_quantize_kernel<TYPE><<<blocks_of(q.n * groups_of(q.d) * 16), 256, 0, st>>>(static_cast<const typename Num<TYPE>::Mem *>(v), q.n, q.d, ld,
                                                                                    wide_reads(v, TYPE, ld), q.codes, q.ld_codes, q.scales, q.ld_scales,
                                                                                    status);
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

template <int TYPE, int kXT, int YT, int WX, int WY, int H>
static int32_t product4(const dq_mx4 &a, const dq_mx4 &w, void *out, int64_t ld, hipStream_t st)
{
    const int64_t tiles_x = (w.n + kXT - 1) / kXT, tiles_y = (a.n + YT - 1) / YT;
    if (tiles_x * tiles_y > kMost4) return DQ_ERR_UNSUPPORTED;
    auto operand = [](const dq_mx4 &q) { return Operand{reinterpret_cast<const char *>(q.codes), q.ld_codes, q.n, static_cast<int32_t>(groups_of(q.d) * 32), 0, q.scales, q.ld_scales}; };
    mx4_product_kernel<TYPE, kXT, YT, WX, WY, H><<<static_cast<unsigned>(tiles_x * tiles_y), WX * WY * kWave, 0, st>>>(
        operand(w), operand(a), groups_of(a.d) * 32, static_cast<int>(tiles_x), static_cast<int>(tiles_y), static_cast<typename Num<TYPE>::Mem *>(out), ld);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
template <int TYPE>
static int32_t product4(const dq_mx4 &a, const dq_mx4 &w, void *out, int64_t ld, hipStream_t st)
{
    switch (tile_for_rows(w.n, a.n)) {
    case kTile256: return product4<TYPE, 256, 256, 2, 4, 1>(a, w, out, ld, st);
    case kTile128: return product4<TYPE, 128, 128, 2, 2, 1>(a, w, out, ld, st);
    case kTile64: return product4<TYPE, 64, 64, 2, 2, 2>(a, w, out, ld, st);
    default: return product4<TYPE, 64, 16, 4, 1, 2>(a, w, out, ld, st);
    }
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
    const int vector = dq::four_at_once(out, ld, dq::wide_of(type));
    const unsigned blocks = dq::blocks_of(q->n * ((q->d + 7) / 8));
    switch (type) {
    case DQ_F32: dq::mx4_dequantize_kernel<DQ_F32><<<blocks, 256, 0, st>>>(q->codes, q->ld_codes, q->scales, q->ld_scales, q->n, q->d, static_cast<float *>(out), ld, vector); break;
    case DQ_F16: dq::mx4_dequantize_kernel<DQ_F16><<<blocks, 256, 0, st>>>(q->codes, q->ld_codes, q->scales, q->ld_scales, q->n, q->d, static_cast<dq::u16 *>(out), ld, vector); break;
    default: dq::mx4_dequantize_kernel<DQ_BF16><<<blocks, 256, 0, st>>>(q->codes, q->ld_codes, q->scales, q->ld_scales, q->n, q->d, static_cast<dq::u16 *>(out), ld, vector); break;
    }
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

extern "C" int32_t dq_mx4_product(const dq_mx4 *a, const dq_mx4 *w, void *out, int32_t type, int64_t ld, void *stream)
{
    if (const int32_t e = dq::check4(a)) return e;
    if (const int32_t e = dq::check4(w)) return e;
    if (a->d != w->d) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = dq::check_matrix(out, type, w->n, ld)) return e;
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
    if (n > dq::kMost4) return DQ_ERR_UNSUPPORTED;
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
