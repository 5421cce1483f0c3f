// Rows over their root mean square, times a gain, after a residual's addition: into the rows' type, or into 8-bit blocks; and the gradients.
//   h = x + r (in the rows' type),  s = 1 / sqrt(mean(h^2) + eps),  y = h s gain
//   u = dy gain,  dx = s (u - h s^2 mean(u h)) + dh,  dgain_j = sum_t dy_tj h_tj s_t
// Sums of a row are held in 64 bits (squares of the types' largest numbers are in their range), the sums over rows in 32.
#include "fp8_codes.h"

namespace dq {

struct NormArgs {
    const void *x, *residual;
    int64_t ldx, ldr, n;
    uint32_t d;
    const float *gain;
    float eps;
};

// Eight numbers of h: rounded to the rows' type where a residual is added.
template <int TYPE>
__device__ __forceinline__ void sum_of(Eight<TYPE> x, Eight<TYPE> r, bool two, float h[8])
{
    values_of<TYPE>(x, h);
    if (!two) return;
    float more[8];
    values_of<TYPE>(r, more);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = Num<TYPE>::load(Num<TYPE>::store(h[e] + more[e]));
}
template <int TYPE>
__device__ __forceinline__ void load_h(const typename Num<TYPE>::Mem *x, const typename Num<TYPE>::Mem *r, uint32_t c, uint32_t d, float h[8])
{
    const Eight<TYPE> a = ask_eight<TYPE>(x, c, d);
    Eight<TYPE> b{};
    if (r) b = ask_eight<TYPE>(r, c, d);
    sum_of<TYPE>(a, b, r, h);
}
__device__ __forceinline__ void load_gain(const float *gain, uint32_t c, uint32_t d, float out[8])
{
    if (gain) {
        load_eight<DQ_F32>(gain, c, d, out);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = 1.0f;
    }
}

// How a row lies over a block's threads: LANES of them share it, each has VEC times eight neighbouring numbers, LANES * 8 apart.  256 threads work on
// 256 / LANES rows at a time (1024 lanes: on one).  A row is read once and stays in registers; rows beyond 24576 numbers are read twice.
//
// What bounds both kernels is memory.  8192 x 4096 in bfloat16: residual and 8-bit blocks (235 MB) 44 us, 5.3 TB/s (256 threads that read rows of any
// length twice: 51); gradients with the residual's (335 MB) 77 us, 4.4 TB/s (181), and 5 for the sums of 1024 blocks' shares of dgain (a column a thread: 112).
template <int LANES, int VEC>
struct RowShape {
    static constexpr int kThreads = LANES > 256 ? LANES : 256, kRows = kThreads / LANES, kLanes = LANES, kVec = VEC;
};

// The sum of a value over the LANES threads of a row, in each of them.  room: a place per wavefront (its turn is over behind the next barrier).
template <int LANES>
__device__ __forceinline__ void row_sum(double (&v)[2], int count, double (*room)[2])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i >= count) break;
#pragma unroll
        for (int by = 1; by < (LANES < kWave ? LANES : kWave); by *= 2) v[i] += __shfl_xor(v[i], by);
    }
    if constexpr (LANES > kWave) {
        if ((threadIdx.x & 63) == 0) {
            room[threadIdx.x / kWave][0] = v[0];
            room[threadIdx.x / kWave][1] = v[1];
        }
        __syncthreads();
        v[0] = v[1] = 0.0;
#pragma unroll
        for (int w = 0; w < LANES / kWave; ++w) {
            v[0] += room[w][0];
            v[1] += room[w][1];
        }
    }
}

// A float32 that lies on the same side of every coarser number as v does, and of the borders between them: cut towards zero, its last bit set where that took
// something away.
__device__ __forceinline__ float side_of(double v)
{
    const float near = static_cast<float>(v);
    const double back = static_cast<double>(near);
    uint32_t bits = __float_as_uint(near);
    if (!(back != v) || (bits & 0x7fffffffu) >= 0x7f800000u) return near;
    if (__builtin_fabs(back) > __builtin_fabs(v)) --bits;
    return __uint_as_float(bits | 1u);
}

// y of eight numbers of h, to where it goes.  Of float32 rows the 8-bit blocks are those of y itself (in 64 bits, as if it were rounded once); of 16-bit rows those of
// its float32 value, which three roundings of 2^-24 make.
template <int TYPE>
__device__ __forceinline__ void put_normed(const float h[8], double scale, const float gain[8], int64_t row, uint32_t c, uint32_t d, typename Num<TYPE>::Mem *out, int64_t ldo,
                                           const dq_fp8 &q, uint32_t *status)
{
    float y[8];
    const float s = static_cast<float>(scale);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = h[e] * s * gain[e];
    if (out && c < d) store_eight<TYPE>(out + row * ldo + c, y, static_cast<int>(d - c));
    if (!q.codes) return;
    if constexpr (TYPE == DQ_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = side_of(h[e] * scale * gain[e]);
    }
    uint32_t byte;
    const uint2 code = quantize_eight8(y, byte);
    *reinterpret_cast<uint2 *>(q.codes + row * q.ld_codes + c) = code;
    if (threadIdx.x % 16 == 0) {
        write_scale8(q.scales + row * q.ld_scales, c / kGroup8, (d + kGroup8 - 1) / kGroup8, byte);
        if (byte == 255 && status) atomicOr(status, 1u);
    }
}

template <int TYPE, int LANES, int VEC>
__global__ __launch_bounds__((RowShape<LANES, VEC>::kThreads)) void norm_kernel(NormArgs p, typename Num<TYPE>::Mem *h_out, int64_t ldh, typename Num<TYPE>::Mem *out, int64_t ldo,
                                                                                dq_fp8 q, uint32_t *__restrict__ status)
{
    typedef typename Num<TYPE>::Mem Mem;
    typedef RowShape<LANES, VEC> Shape;
    __shared__ double room[16][2];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * Shape::kRows + threadIdx.x / LANES;
    if (LANES <= kWave && row >= p.n) return;                       // (a row's lanes are of one wavefront)
    const uint32_t d = p.d, first = threadIdx.x % LANES * 8, end = (d + kGroup8 - 1) / kGroup8 * kGroup8;
    const Mem *const x = static_cast<const Mem *>(p.x) + row * p.ldx, *const r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
    float h[VEC][8], gain[8];
    Eight<TYPE> asked[VEC], added[VEC] = {};
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        asked[v] = ask_eight<TYPE>(x, first + v * LANES * 8, d);
        if (r) added[v] = ask_eight<TYPE>(r, first + v * LANES * 8, d);
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum_of<TYPE>(asked[v], added[v], r, h[v]);
    double square[2] = {};
#pragma unroll
    for (int v = 0; v < VEC; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) square[0] += static_cast<double>(h[v][e]) * h[v][e];
    if (h_out) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            const uint32_t c = first + v * LANES * 8;
            if (c < d) store_eight<TYPE>(h_out + row * ldh + c, h[v], static_cast<int>(d - c));
        }
    }
    row_sum<LANES>(square, 1, room);
    const double mean = square[0] / d + p.eps;
    if (!__builtin_isfinite(mean) && first == 0 && status) atomicOr(status, 1u);
    const double s = 1.0 / sqrt(mean);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        const uint32_t c = first + v * LANES * 8;
        if (c >= end) continue;                                     // (sixteen lanes that share a block go together)
        load_gain(p.gain, c, d, gain);
        put_normed<TYPE>(h[v], s, gain, row, c, d, out, ldo, q, status);
    }
}

// A block a row, of any length: read twice.
template <int TYPE>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs p, typename Num<TYPE>::Mem *h_out, int64_t ldh, typename Num<TYPE>::Mem *out, int64_t ldo, dq_fp8 q,
                                                         uint32_t *__restrict__ status)
{
    typedef typename Num<TYPE>::Mem Mem;
    __shared__ double room[16][2];
    const int64_t row = blockIdx.x;
    const uint32_t d = p.d, end = (d + kGroup8 - 1) / kGroup8 * kGroup8;
    const Mem *x = static_cast<const Mem *>(p.x) + row * p.ldx, *r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
    float h[8], gain[8];
    double square[2] = {};
    for (uint32_t c = threadIdx.x * 8; c < d; c += 8192) {
        load_h<TYPE>(x, r, c, d, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) square[0] += static_cast<double>(h[e]) * h[e];
        if (h_out) store_eight<TYPE>(h_out + row * ldh + c, h, static_cast<int>(d - c));
    }
    row_sum<1024>(square, 1, room);
    const double mean = square[0] / d + p.eps;
    if (!__builtin_isfinite(mean) && threadIdx.x == 0 && status) atomicOr(status, 1u);
    const double s = 1.0 / sqrt(mean);
    if (h_out) {                                        // (it may lie where x or the residual does)
        x = h_out + row * ldh;
        r = nullptr;
    }
    for (uint32_t c = threadIdx.x * 8; c < end; c += 8192) {
        load_h<TYPE>(x, r, c, d, h);
        load_gain(p.gain, c, d, gain);
        put_normed<TYPE>(h, s, gain, row, c, d, out, ldo, q, status);
    }
}

// dx of eight numbers.
__device__ __forceinline__ void gradient_of(const float h[8], const float g[8], const float gain[8], const float more[8], float s, float k, float dx[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) dx[e] = s * (g[e] * gain[e] - h[e] * k) + more[e];
}

// Rows blockIdx.x * kRows .., + gridDim.x * kRows, ...: dx, and the block's share of dgain's sums, held in registers until its last row, then
// added up over the block's rows in LDS.  (Each load is converted where it arrives: asked for all together, as the forward pass does, h, dy and dgain's sums leave
// too few registers, 88 us instead of 77.)
template <int TYPE, int LANES, int VEC>
__global__ __launch_bounds__((RowShape<LANES, VEC>::kThreads)) void norm_grad_kernel(NormArgs p, const typename Num<TYPE>::Mem *dy, int64_t lddy, const typename Num<TYPE>::Mem *dh,
                                                                                     int64_t lddh, typename Num<TYPE>::Mem *dx, int64_t lddx, float *__restrict__ parts)
{
    typedef typename Num<TYPE>::Mem Mem;
    typedef RowShape<LANES, VEC> Shape;
    __shared__ double room[2][16][2];
    __shared__ __attribute__((aligned(16))) float turned[Shape::kRows > 1 ? Shape::kThreads * 8 : 4];
    const uint32_t d = p.d, first = threadIdx.x % LANES * 8;
    float h[VEC][8], g[VEC][8], sum[VEC][8] = {}, gain[8], more[8];
    int turn = 0;
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * Shape::kRows; row0 < p.n; row0 += static_cast<int64_t>(gridDim.x) * Shape::kRows, turn ^= 1) {
        const int64_t row = row0 + threadIdx.x / LANES;
        if (row >= p.n) continue;                                   // (where a row is shared by more than a wavefront there is one at a time)
        const Mem *const x = static_cast<const Mem *>(p.x) + row * p.ldx, *const r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            load_eight<TYPE>(x, first + v * LANES * 8, d, h[v]);
            if (r) {
                load_eight<TYPE>(r, first + v * LANES * 8, d, more);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[v][e] = Num<TYPE>::load(Num<TYPE>::store(h[v][e] + more[e]));
            }
            load_eight<TYPE>(dy + row * lddy, first + v * LANES * 8, d, g[v]);
        }
        double sums[2] = {};
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            load_gain(p.gain, first + v * LANES * 8, d, gain);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[0] += static_cast<double>(h[v][e]) * h[v][e];
                sums[1] += static_cast<double>(g[v][e] * gain[e]) * h[v][e];
            }
        }
        row_sum<LANES>(sums, 2, room[turn]);
        const double mean = sums[0] / d + p.eps;
        const float s = static_cast<float>(1.0 / sqrt(mean)), k = static_cast<float>(sums[1] / d / mean);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            const uint32_t c = first + v * LANES * 8;
            if (c >= d) continue;
            if (parts) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[v][e] += g[v][e] * (h[v][e] * s);
            }
            if (!dx) continue;
            load_gain(p.gain, c, d, gain);
#pragma unroll
            for (int e = 0; e < 8; ++e) more[e] = 0.0f;
            if (dh) load_eight<TYPE>(dh + row * lddh, c, d, more);
            gradient_of(h[v], g[v], gain, more, s, k, g[v]);
            store_eight<TYPE>(dx + row * lddx + c, g[v], static_cast<int>(d - c));
        }
    }
    if (!parts) return;
    float *const part = parts + static_cast<int64_t>(blockIdx.x) * d;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        const uint32_t c = first + v * LANES * 8;
        if constexpr (Shape::kRows > 1) {
            if (v) __syncthreads();
            store_eight<DQ_F32>(turned + threadIdx.x * 8, sum[v], 8);
            __syncthreads();
            if (threadIdx.x >= LANES) continue;
            for (int w = 1; w < Shape::kRows; ++w) {
                load_eight<DQ_F32>(turned + (w * LANES + threadIdx.x) * 8, 0, 8, more);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[v][e] += more[e];
            }
        }
        if (c < d) store_eight<DQ_F32>(part + c, sum[v], static_cast<int>(d - c));
    }
}

// ... of rows of any length, read twice; the block's share of dgain lies in memory while it is added up.
template <int TYPE>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormArgs p, const typename Num<TYPE>::Mem *dy, int64_t lddy, const typename Num<TYPE>::Mem *dh, int64_t lddh,
                                                              typename Num<TYPE>::Mem *dx, int64_t lddx, float *__restrict__ parts)
{
    typedef typename Num<TYPE>::Mem Mem;
    __shared__ double room[2][16][2];
    const uint32_t d = p.d;
    float *const part = parts + static_cast<int64_t>(blockIdx.x) * d;
    float h[8], g[8], gain[8], more[8], sum[8];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x, turn ^= 1) {
        const Mem *const x = static_cast<const Mem *>(p.x) + row * p.ldx, *const r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
        double sums[2] = {};
        for (uint32_t c = threadIdx.x * 8; c < d; c += 8192) {
            load_h<TYPE>(x, r, c, d, h);
            load_eight<TYPE>(dy + row * lddy, c, d, g);
            load_gain(p.gain, c, d, gain);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[0] += static_cast<double>(h[e]) * h[e];
                sums[1] += static_cast<double>(g[e] * gain[e]) * h[e];
            }
        }
        row_sum<1024>(sums, 2, room[turn]);
        const double mean = sums[0] / d + p.eps;
        const float s = static_cast<float>(1.0 / sqrt(mean)), k = static_cast<float>(sums[1] / d / mean);
        for (uint32_t c = threadIdx.x * 8; c < d; c += 8192) {
            load_h<TYPE>(x, r, c, d, h);
            load_eight<TYPE>(dy + row * lddy, c, d, g);
            load_gain(p.gain, c, d, gain);
            if (parts) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
                if (row != blockIdx.x) load_eight<DQ_F32>(part, c, d, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += g[e] * (h[e] * s);
                store_eight<DQ_F32>(part + c, sum, static_cast<int>(d - c));
            }
            if (!dx) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) more[e] = 0.0f;
            if (dh) load_eight<TYPE>(dh + row * lddh, c, d, more);
            gradient_of(h, g, gain, more, s, k, g);
            store_eight<TYPE>(dx + row * lddx + c, g, static_cast<int>(d - c));
        }
    }
}

// Few rows: a block per row leaves most of the chip idle, and a long row is then a chain of waits.  The rows' sums a piece of 2048 columns a block ...
constexpr int64_t kNormPiece = 2048, kFewNormRows = 128;
template <int TYPE>
__global__ __launch_bounds__(256) void norm_grad_sums_kernel(NormArgs p, const typename Num<TYPE>::Mem *dy, int64_t lddy, double (*__restrict__ sums)[2])
{
    typedef typename Num<TYPE>::Mem Mem;
    __shared__ double room[4][2];
    const int64_t row = blockIdx.y;
    const Mem *const x = static_cast<const Mem *>(p.x) + row * p.ldx, *const r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
    const uint32_t c = blockIdx.x * kNormPiece + threadIdx.x * 8;
    double sum[2] = {};
    if (c < p.d) {
        float h[8], g[8], gain[8];
        const Eight<TYPE> asked = ask_eight<TYPE>(dy + row * lddy, c, p.d);
        load_gain(p.gain, c, p.d, gain);
        load_h<TYPE>(x, r, c, p.d, h);
        values_of<TYPE>(asked, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum[0] += static_cast<double>(h[e]) * h[e];
            sum[1] += static_cast<double>(g[e] * gain[e]) * h[e];
        }
    }
    row_sum<256>(sum, 2, room);
    if (threadIdx.x) return;
    double *const to = sums[row * gridDim.x + blockIdx.x];
    to[0] = sum[0];
    to[1] = sum[1];
}
// ... then 64 columns of all rows a block, which has dgain's sums of them to itself: two launches as well.  float32, with and without these two: 64 x 20958 14.2 and
// 20.8 us, 64 x 47236 19.6 and 37.1, 1 x 47236 8.9 and 24.3, 128 x 4096 9.7 and 10.2; 256 x 4096 13.7 and 11.2.  The border goes by rows alone: beyond it, without calls between
// the launches, 129 x 256 are 7.7 and 5.3 us, x 4096 8.5 and 7.5, but x 8192 9.3 and 10.9, x 20958 21.8 and 24.6, x 47236 31.9 and 37.2; 192 x 47236 42.6 and 46.5, 256 x 20958 34.4 and
// 33.4.
template <int TYPE>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(NormArgs p, const typename Num<TYPE>::Mem *dy, int64_t lddy, const typename Num<TYPE>::Mem *dh, int64_t lddh,
                                                                typename Num<TYPE>::Mem *dx, int64_t lddx, const double (*__restrict__ sums)[2], int pieces,
                                                                float *__restrict__ dgain)
{
    typedef typename Num<TYPE>::Mem Mem;
    __shared__ float scale[kFewNormRows], along[kFewNormRows];
    __shared__ __attribute__((aligned(16))) float turned[32][64];
    const int n = static_cast<int>(p.n), first = threadIdx.x / 8;
    const uint32_t d = p.d, at = threadIdx.x % 8 * 8, c = blockIdx.x * 64u + at;
    if (static_cast<int>(threadIdx.x) < n) {
        double sum[2] = {};
        for (int i = 0; i < pieces; ++i) {
            sum[0] += sums[threadIdx.x * pieces + i][0];
            sum[1] += sums[threadIdx.x * pieces + i][1];
        }
        const double mean = sum[0] / d + p.eps;
        scale[threadIdx.x] = static_cast<float>(1.0 / sqrt(mean));
        along[threadIdx.x] = static_cast<float>(sum[1] / d / mean);
    }
    __syncthreads();
    float total[8] = {};
    if (c < d) {
        float gain[8];
        load_gain(p.gain, c, d, gain);
        for (int row = first; row < n; row += 32) {
            const Mem *const x = static_cast<const Mem *>(p.x) + row * p.ldx, *const r = p.residual ? static_cast<const Mem *>(p.residual) + row * p.ldr : nullptr;
            float h[8], g[8], more[8] = {};
            const Eight<TYPE> asked = ask_eight<TYPE>(dy + row * lddy, c, d);
            Eight<TYPE> rest{};
            if (dx && dh) rest = ask_eight<TYPE>(dh + row * lddh, c, d);
            load_h<TYPE>(x, r, c, d, h);
            values_of<TYPE>(asked, g);
            const float s = scale[row];
#pragma unroll
            for (int e = 0; e < 8; ++e) total[e] += g[e] * (h[e] * s);
            if (!dx) continue;
            if (dh) values_of<TYPE>(rest, more);
            gradient_of(h, g, gain, more, s, along[row], g);
            store_eight<TYPE>(dx + row * lddx + c, g, static_cast<int>(d - c));
        }
    }
    store_eight<DQ_F32>(&turned[first][at], total, 8);
    __syncthreads();
    const uint32_t column = blockIdx.x * 64u + threadIdx.x;
    if (threadIdx.x >= 64 || column >= d) return;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += turned[i][threadIdx.x];
    dgain[column] = static_cast<float>(sum);
}

// dgain: the blocks' shares.  A block takes 64 columns, each of its sixteen wavefronts every sixteenth share.
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float *__restrict__ parts, int count, uint32_t d, float *__restrict__ dgain)
{
    __shared__ double room[16][kWave];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / kWave, c = blockIdx.x * 64u + lane;
    double sum = 0.0;
    if (c < d) {
        int i = static_cast<int>(wave);
        for (; i + 7 * 16 < count; i += 8 * 16) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = parts[static_cast<int64_t>(i + 16 * u) * d + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        for (; i < count; i += 16) sum += parts[static_cast<int64_t>(i) * d + c];
    }
    room[wave][lane] = sum;
    __syncthreads();
    if (wave || c >= d) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += room[w][lane];
    dgain[c] = static_cast<float>(sum);
}

// ---- host ----------------------------------------------------------------------
constexpr int64_t kMostRows = 1ll << 30, kWidestNorm = 1ll << 22;

static int32_t check_norm(const dq_norm *p)
{
    if (!p || p->n <= 0 || p->d <= 0 || !(p->eps > 0.0f) || !__builtin_isfinite(p->eps)) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = check_matrix(p->x, p->type, p->d, p->ldx)) return e;
    if (p->residual)
        if (const int32_t e = check_matrix(p->residual, p->type, p->d, p->ldr)) return e;
    if (reinterpret_cast<uintptr_t>(p->gain) % 4) return DQ_ERR_INVALID_ARG;
    if (p->n > kMostRows || p->d > kWidestNorm) return DQ_ERR_UNSUPPORTED;
    return DQ_OK;
}
static NormArgs args_of(const dq_norm &p) { return NormArgs{p.x, p.residual, p.ldx, p.ldr, p.n, static_cast<uint32_t>(p.d), p.gain, p.eps}; }
// The rows' shape by their length: as few lanes as hold it in up to four (two where a row has few) times eight numbers each.
enum NormShape { kNorm16, kNorm32, kNorm64, kNorm64x2, kNorm256, kNorm256x2, kNorm256x4, kNorm1024x2, kNorm1024x3, kNormLong };
static NormShape norm_shape(int64_t d)
{
    return d <= 128 ? kNorm16 : d <= 256 ? kNorm32 : d <= 512 ? kNorm64 : d <= 1024 ? kNorm64x2 : d <= 2048 ? kNorm256 : d <= 4096 ? kNorm256x2 :
           d <= 8192 ? kNorm256x4 : d <= 16384 ? kNorm1024x2 : d <= 24576 ? kNorm1024x3 : kNormLong;
}
static int64_t rows_at_once(int64_t d) { return d <= 128 ? 16 : d <= 256 ? 8 : d <= 1024 ? 4 : 1; }
// Blocks of the gradients: each adds up dgain over its rows.
static int64_t grad_blocks(int64_t n, int64_t d) { return std::min<int64_t>(ceil_div(n, rows_at_once(d)), d <= 8192 ? 1024 : 512); }

// CALL(LANES, VEC) for the shape of rows of d numbers, or LONG.
#define DQ_NORM_SHAPES(d, CALL, LONG) \
    switch (norm_shape(d)) { \
    case kNorm16: CALL(16, 1); break; \
    case kNorm32: CALL(32, 1); break; \
    case kNorm64: CALL(64, 1); break; \
    case kNorm64x2: CALL(64, 2); break; \
    case kNorm256: CALL(256, 1); break; \
    case kNorm256x2: CALL(256, 2); break; \
    case kNorm256x4: CALL(256, 4); break; \
    case kNorm1024x2: CALL(1024, 2); break; \
    case kNorm1024x3: CALL(1024, 3); break; \
    default: LONG; \
    }

template <int TYPE>
static int32_t norm(const dq_norm &p, void *h_out, int64_t ldh, void *out, int64_t ldo, const dq_fp8 *q, uint32_t *status, hipStream_t st)
{
    typedef typename Num<TYPE>::Mem Mem;
    const unsigned blocks = static_cast<unsigned>(ceil_div(p.n, rows_at_once(p.d)));
#define DQ_NORM_ARGS args_of(p), static_cast<Mem *>(h_out), ldh, static_cast<Mem *>(out), ldo, q ? *q : dq_fp8{}, status
#define DQ_NORM(LANES, VEC) norm_kernel<TYPE, LANES, VEC><<<blocks, RowShape<LANES, VEC>::kThreads, 0, st>>>(DQ_NORM_ARGS)
    DQ_NORM_SHAPES(p.d, DQ_NORM, (norm_long_kernel<TYPE><<<blocks, 1024, 0, st>>>(DQ_NORM_ARGS)))
#undef DQ_NORM
#undef DQ_NORM_ARGS
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}
template <int TYPE>
static int32_t norm_grad(const dq_norm &p, const void *dy, int64_t lddy, const void *dh, int64_t lddh, void *dx, int64_t lddx, float *dgain, float *parts, hipStream_t st)
{
    typedef typename Num<TYPE>::Mem Mem;
    if (dgain && p.n <= kFewNormRows) {
        const dim3 pieces(static_cast<unsigned>(ceil_div(p.d, kNormPiece)), static_cast<unsigned>(p.n));
        double(*const sums)[2] = reinterpret_cast<double(*)[2]>(parts);
        norm_grad_sums_kernel<TYPE><<<pieces, 256, 0, st>>>(args_of(p), static_cast<const Mem *>(dy), lddy, sums);
        DQ_LAUNCH_CHECK();
        norm_grad_columns_kernel<TYPE><<<static_cast<unsigned>(ceil_div(p.d, 64)), 256, 0, st>>>(args_of(p), static_cast<const Mem *>(dy), lddy, static_cast<const Mem *>(dh), lddh,
                                                                                                 static_cast<Mem *>(dx), lddx, sums, static_cast<int>(pieces.x), dgain);
        DQ_LAUNCH_CHECK();
        return DQ_OK;
    }
    const unsigned count = static_cast<unsigned>(grad_blocks(p.n, p.d));
#define DQ_NORM_ARGS args_of(p), static_cast<const Mem *>(dy), lddy, static_cast<const Mem *>(dh), lddh, static_cast<Mem *>(dx), lddx, dgain ? parts : nullptr
#define DQ_NORM(LANES, VEC) norm_grad_kernel<TYPE, LANES, VEC><<<count, RowShape<LANES, VEC>::kThreads, 0, st>>>(DQ_NORM_ARGS)
    DQ_NORM_SHAPES(p.d, DQ_NORM, (norm_grad_long_kernel<TYPE><<<count, 1024, 0, st>>>(DQ_NORM_ARGS)))
#undef DQ_NORM
#undef DQ_NORM_ARGS
    DQ_LAUNCH_CHECK();
    if (!dgain) return DQ_OK;
    norm_gain_kernel<<<static_cast<unsigned>((p.d + 63) / 64), 1024, 0, st>>>(parts, static_cast<int>(count), static_cast<uint32_t>(p.d), dgain);
    DQ_LAUNCH_CHECK();
    return DQ_OK;
}

}  // namespace dq

extern "C" int32_t dq_rms_norm(const dq_norm *p, void *h_out, int64_t ldh, void *out, int64_t ldo, const dq_fp8 *q, uint32_t *status, void *stream)
{
    if (const int32_t e = dq::check_norm(p)) return e;
    if (!h_out && !out && !q) return DQ_ERR_INVALID_ARG;
    if (h_out && !p->residual) return DQ_ERR_INVALID_ARG;
    if (h_out)
        if (const int32_t e = dq::check_matrix(h_out, p->type, p->d, ldh)) return e;
    if (out)
        if (const int32_t e = dq::check_matrix(out, p->type, p->d, ldo)) return e;
    if (q) {
        if (const int32_t e = dq::check8(q)) return e;
        if (q->n != p->n || q->d != p->d) return DQ_ERR_INVALID_ARG;
    }
    if (!dq::launchable(dq::ceil_div(p->n, dq::rows_at_once(p->d)), p->d > 8192 ? 1024 : 256)) return DQ_ERR_UNSUPPORTED;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (p->type) {
    case DQ_F32: return dq::norm<DQ_F32>(*p, h_out, ldh, out, ldo, q, status, st);
    case DQ_F16: return dq::norm<DQ_F16>(*p, h_out, ldh, out, ldo, q, status, st);
    default: return dq::norm<DQ_BF16>(*p, h_out, ldh, out, ldo, q, status, st);
    }
}

extern "C" int64_t dq_rms_norm_grad_bytes(int64_t n, int64_t d)
{
    if (n <= 0 || d <= 0) return DQ_ERR_INVALID_ARG;
    if (n > dq::kMostRows || d > dq::kWidestNorm) return DQ_ERR_UNSUPPORTED;
    return n <= dq::kFewNormRows ? n * dq::ceil_div(d, dq::kNormPiece) * 16 : (dq::grad_blocks(n, d) * d * 4 + 15) / 16 * 16;
}

extern "C" int32_t dq_rms_norm_grad(const dq_norm *p, const void *dy, int64_t lddy, const void *dh, int64_t lddh, void *dx_out, int64_t lddx, float *dgain_out, void *ws,
                                    int64_t ws_bytes, void *stream)
{
    if (const int32_t e = dq::check_norm(p)) return e;
    if ((!dx_out && !dgain_out) || reinterpret_cast<uintptr_t>(dgain_out) % 4) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = dq::check_matrix(dy, p->type, p->d, lddy)) return e;
    if (dh)
        if (const int32_t e = dq::check_matrix(dh, p->type, p->d, lddh)) return e;
    if (dx_out)
        if (const int32_t e = dq::check_matrix(dx_out, p->type, p->d, lddx)) return e;
    if (dgain_out) {
        if (!ws || !dq::aligned16(ws)) return DQ_ERR_INVALID_ARG;
        if (ws_bytes < dq_rms_norm_grad_bytes(p->n, p->d)) return DQ_ERR_WORKSPACE;
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float *const parts = static_cast<float *>(ws);
    switch (p->type) {
    case DQ_F32: return dq::norm_grad<DQ_F32>(*p, dy, lddy, dh, lddh, dx_out, lddx, dgain_out, parts, st);
    case DQ_F16: return dq::norm_grad<DQ_F16>(*p, dy, lddy, dh, lddh, dx_out, lddx, dgain_out, parts, st);
    default: return dq::norm_grad<DQ_BF16>(*p, dy, lddy, dh, lddh, dx_out, lddx, dgain_out, parts, st);
    }
}
