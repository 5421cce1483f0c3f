// Models of many classes: softmax cross entropy and distillation from a teacher's largest logits, with gradients.
//
// Both losses are sums  entropy_t + sum_j q_tj (lse_t - z_tj)  over a row's few targets (class, q): a label is one target of weight 1.
// The scores z = a W^T / tau are made tile by tile and never stored:
//   teacher   a teacher's entries in order of class, with their weights q
//   pack      operands that the matrix cores cannot read in place
//   scores    one tile of z: per row its maximum, the sum of exp above it and the targets' sum q z; for gradients the first piece's z too
//   finish    lse and loss of a row from its tiles
//   kept      g = f (exp(z - lse) - q) of the first piece from its z, rounded to 16 bits, where they lie
//   grad      (the other pieces) the tile again, now g
//   da        += g W of the piece, split over its classes where there are few tiles
//   dw        = g^T a of the piece
#include <algorithm>

#include "dq_common.h"
#include "matrix_tile.h"

namespace dq {

constexpr int kNoClass = 0x7fffffff;
constexpr float kF16Unit = 16384.0f;           // g of float16: terms down to 2^-28 of the largest weight stay normal

// The three bfloat16 whose sum is v.  Infinities and NaNs: the first part alone.
__device__ __forceinline__ void parts_of(float v, u16 out[3])
{
    out[0] = Part::store(v);
    const float r = v - Part::load(out[0]);
    const bool whole = __builtin_isfinite(Part::load(out[0]));
    out[1] = whole ? Part::store(r) : 0;
    out[2] = whole ? Part::store(r - Part::load(out[1])) : 0;
}

// ---- targets -------------------------------------------------------------------
// What the kernels know of the rows' targets: k per row, sorted by class; q null for labels.  A class that is not one of the c is no
// target (a label below 0, the end of a row's entries).
struct Targets {
    const int32_t *cls;
    const float *q;
    int32_t k;
    uint32_t c;
    // whether row t has a target: its first one is one
    __device__ __forceinline__ bool used(int64_t t) const { return static_cast<uint32_t>(cls[t * k]) < c; }
    // first target of row t with a class of at least c0
    __device__ __forceinline__ int first(int64_t t, int c0) const
    {
        const int32_t *const row = cls + t * k;
        int lo = 0, hi = k;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (row[mid] < c0) lo = mid + 1;
            else hi = mid;
        }
        return lo;
    }
};

// ---- operands that are not read in place ---------------------------------------
// Rows of [rows][cols] to rows of out_cols 16-bit numbers (three planes of them for float32), zeros behind row and column ends.
// A second copy leaves out the rows without a target.  One thread per eight columns; bound by memory (20011 x 1001 float16, 81 MB moved,
// in 15 us; read number by number 28).
struct Packed {
    const void *v;
    int64_t ld, rows, cols;
    u16 *out, *used;                   // either may be null
    int64_t out_rows, used_rows;       // with the zeros behind them
};
template <int TYPE>
__device__ __forceinline__ void pack_eight(const Packed &j, int64_t out_cols, int64_t i, const Targets &targets)
{
    typedef typename Num<TYPE>::Mem Mem;
    const int64_t each = out_cols / 8, r = i / each, c = (i - r * each) * 8;
    const Mem *const row = static_cast<const Mem *>(j.v) + r * j.ld;
    u16 part[3][8];
    Mem x[8] = {};
    if (r < j.rows) {
        if (c + 8 <= j.cols) {                       // (16-byte loads of any alignment to the number)
            struct __attribute__((packed, aligned(sizeof(Mem)))) All {
                __attribute__((ext_vector_type(8))) Mem v;
            };
            const All all = *reinterpret_cast<const All *>(row + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = all.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < j.cols) x[e] = row[c + e];
        }
    }
    constexpr int kPlanes = TYPE == DQ_F32 ? 3 : 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (TYPE == DQ_F32) {
            u16 p[3];
            parts_of(x[e], p);
            part[0][e] = p[0];
            part[1][e] = p[1];
            part[2][e] = p[2];
        } else {
            part[0][e] = x[e];
        }
    }
    const bool live = j.used && r < j.rows && targets.used(r);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        const i32x4 v = __builtin_bit_cast(i32x4, part[p]);
        if (j.out && r < j.out_rows) *reinterpret_cast<i32x4 *>(j.out + (p * j.out_rows + r) * out_cols + c) = v;
        if (j.used && r < j.used_rows) *reinterpret_cast<i32x4 *>(j.used + (p * j.used_rows + r) * out_cols + c) = live ? v : i32x4{0, 0, 0, 0};
    }
}
// The features and the model in one launch.
template <int TYPE>
__global__ __launch_bounds__(256) void pack_kernel(Packed a, Packed w, int64_t out_cols, int64_t of_a, int64_t total, Targets targets)
{
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        if (i < of_a) pack_eight<TYPE>(a, out_cols, i, targets);
        else pack_eight<TYPE>(w, out_cols, i - of_a, targets);
    }
}

// The largest finite |weight| of the rows that have a target, for float16, one block.  Held to at least 2^-100.  A weight that is not finite
// is its own row's matter, whose g is not finite at any unit: taken into the maximum it would make the others' zeros.
__global__ __launch_bounds__(1024) void weight_max_kernel(const float *__restrict__ weight, int64_t n, Targets targets, float *__restrict__ out)
{
    __shared__ uint32_t top;
    if (threadIdx.x == 0) top = 0;
    __syncthreads();
    uint32_t m = 0;
    for (int64_t t = threadIdx.x; t < n; t += 1024)
        if (targets.used(t)) {
            const uint32_t w = __float_as_uint(weight[t]) & 0x7fffffffu;
            if (w < 0x7f800000u) m = max(m, w);
        }
    atomicMax(&top, m);
    __syncthreads();
    if (threadIdx.x == 0) out[0] = top ? __uint_as_float(max(top, 0x0d800000u)) : 1.0f;
}

// One block of 64 threads per row: q = softmax(logit / tau) over the entries, sorted by class (bitonic, in LDS).
// entropy[t] = sum q log q.  Rows without an entry: all classes kNoClass.  (Differences are scaled, not logits: entries of the type's lowest
// value stay finite at any temperature.)  4096 rows of 64 entries: 12 to 14 us.
constexpr int kTeacherThreads = 64;
__global__ __launch_bounds__(kTeacherThreads) void teacher_kernel(const int32_t *__restrict__ cls_in, const float *__restrict__ logit, int64_t ld,
                                                                  int k, int pow2, int64_t c, float inv_tau, int32_t *__restrict__ cls,
                                                                  float *__restrict__ q, float *__restrict__ entropy,
                                                                  uint32_t *__restrict__ status)
{
    __shared__ int32_t key[DQ_MAX_TEACHER];
    __shared__ float val[DQ_MAX_TEACHER];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x;
    bool far = false;
    float top = -INFINITY;
    for (int j = lane; j < pow2; j += kTeacherThreads) {
        int32_t x = j < k ? cls_in[t * ld + j] : -1;
        if (x >= c) far = true;
        if (x < 0 || x >= c) x = kNoClass;
        const float u = x == kNoClass ? -INFINITY : logit[t * ld + j];
        key[j] = x;
        val[j] = u;
        top = u > top || u != u ? u : top;
    }
    if (far && status) atomicOr(status, 2u);
    for (int o = 32; o; o >>= 1) {
        const float other = __shfl_xor(top, o);
        top = other > top || other != other ? other : top;
    }
    const bool none = top == -INFINITY;
    float sum = 0.0f;
    for (int j = lane; j < pow2; j += kTeacherThreads) {
        if (none) key[j] = kNoClass;
        else if (key[j] != kNoClass) sum += expf((val[j] - top) * inv_tau);
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    const float log_sum = logf(sum);
    float ent = 0.0f;
    for (int j = lane; j < pow2; j += kTeacherThreads) {
        const float l = (val[j] - top) * inv_tau, p = key[j] == kNoClass ? 0.0f : expf(l) / sum;
        val[j] = p;
        ent += p == 0.0f ? 0.0f : p * (l - log_sum);
    }
    for (int o = 32; o; o >>= 1) ent += __shfl_xor(ent, o);
    if (lane == 0) entropy[t] = none ? 0.0f : ent;
    __syncthreads();
    for (int size = 2; size <= pow2; size *= 2)
        for (int step = size / 2; step; step /= 2) {
            for (int i = lane; i < pow2 / 2; i += kTeacherThreads) {
                const int a = i / step * step * 2 + i % step, b = a + step;
                const bool up = !(a & size);
                const int32_t ka = key[a], kb = key[b];
                if (up ? ka > kb : ka < kb) {
                    key[a] = kb;
                    key[b] = ka;
                    const float v = val[a];
                    val[a] = val[b];
                    val[b] = v;
                }
            }
            __syncthreads();
        }
    for (int j = lane; j < k; j += kTeacherThreads) {
        cls[t * k + j] = key[j];
        q[t * k + j] = val[j];
    }
}

// ---- scores --------------------------------------------------------------------
constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147181f;
__device__ __forceinline__ float exp_near(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

constexpr int kEdge = 4;               // with a type: rows that are read in place end inside of a step

// The scores of the first piece stay in the place of its gradients, 16 bits of them in each plane: as they are, in two halves, in float32
// and where there are few rows; else how far they lie below the tile's maximum, in 65535 steps up to a factor of 2^-128 (2^-32 in
// float16), behind which probabilities are zeros.  That is off by half a step, a factor of up to 1 -+ 0.00071 (0.00018, with the conversion's own
// rounding).  With g's rounding, which is up to 0.0039 (0.00049) of a term, terms came out up to 0.0046 (0.00066) off and in root mean squares
// 0.00171 instead of 0.00166 (0.00023 and 0.00021).  The targets' scores, where p - q may cancel, are kept whole.
struct Kept {
    u16 *g;                            // null: none
    int64_t ldg, plane, cols;          // numbers; classes of the piece
    float *target_z;                   // z of the targets' entries, null in calls without gradients
};
template <int TYPE>
struct KeptUnit {
    static constexpr float kRange = TYPE == DQ_F16 ? 32.0f : 128.0f;
    // two numbers, y and top being log2 of probabilities up to a common factor
    static __device__ __forceinline__ uint32_t codes(float top, float y0, float y1)
    {
        const float at = top * (1.0f / kRange);
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(__builtin_fmaf(y0, -1.0f / kRange, at), __builtin_fmaf(y1, -1.0f / kRange, at)));
    }
    // shift: log2 of exp(top - lse); a row whose lse is not a number has no number
    static __device__ __forceinline__ float value(u16 code, float shift)
    {
        return code == 65535 && shift == shift ? 0.0f : __builtin_amdgcn_exp2f(shift - static_cast<float>(code) * (kRange / 65535.0f));
    }
};

// The sums of a tile's row: its maximum, the sum of exp above it, the targets' sum q z; [tile][row].
// Bound by the matrix cores where there are many rows (8192 x 47236 x 4096 in bfloat16 2.67 to 2.84 ms on different cards, 1120 to 1190 TFLOP/s,
// a fifth of it the tiles' ends; 2048 x 20958 x 1000 105 to 109 us), by the model's bytes where there are few (1 x 47236 x 4096 80 us, 4.8 TB/s).
template <int WHAT, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave, 2) void scores_kernel(Operand w, Operand a, int64_t k, int64_t n, int64_t c, float inv_tau, Targets targets,
                                                               int tiles_x, int tiles_y, float2 *__restrict__ sums, float *__restrict__ hits, Kept kept)
{
    constexpr int TYPE = WHAT & 3;
    typedef TileProduct<typename Num<TYPE>::Mul, XT, YT, WX, WY, false, false, H, R, P, (WHAT & kEdge) != 0> Tile;
    __shared__ float3 shared[WX][YT];
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t c0 = static_cast<int64_t>(tx) * XT, t0 = static_cast<int64_t>(ty) * YT;
    const int wave_c0 = static_cast<int>(c0) + Tile::sub_x(0) * 16, wave_end = static_cast<int>(lesser(wave_c0 + Tile::SX * 16, c));
    int entry[Tile::SY], at[Tile::SY];          // the rows' first targets from this wavefront's classes on
    Tile tile;
    tile.run(w, a, c0, t0, 0, k, [&] {
#pragma unroll
        for (int y = 0; y < Tile::SY; ++y) {
            const int64_t t = lesser(t0 + Tile::at_y(y), n - 1);
            entry[y] = targets.first(t, wave_c0);
            at[y] = t0 + Tile::at_y(y) < n && entry[y] < targets.k ? targets.cls[t * targets.k + entry[y]] : kNoClass;
        }
    });
    // Where what is kept is relative, scores are taken in units of a factor of two, which saves a product each.
    constexpr bool kBits = !kept_whole(TYPE == DQ_F32, XT);
    const float unit = kBits ? kLn2 : 1.0f, per_unit = kBits ? inv_tau * kLog2E : inv_tau;
    auto exp_of = [](float v) { return kBits ? __builtin_amdgcn_exp2f(v) : TYPE == DQ_F32 ? expf(v) : exp_near(v); };
    const int lane = threadIdx.x & 63, base = static_cast<int>(c0) + Tile::at_x(0);
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y)
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m) tile.acc[m][y] *= per_unit;
    if (c0 + XT > c) {
#pragma unroll
        for (int y = 0; y < Tile::SY; ++y)
#pragma unroll
            for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (base + 16 * m + i >= c) tile.acc[m][y][i] = -INFINITY;
    }
    float top[Tile::SY], sum[Tile::SY];
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) {
        top[y] = -INFINITY;
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[y] = fmaxf(top[y], tile.acc[m][y][i]);
    }
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) top[y] = fmaxf(top[y], __shfl_xor(top[y], 16));
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) top[y] = fmaxf(top[y], __shfl_xor(top[y], 32));
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) {
        const float from = top[y] == -INFINITY ? 0.0f : top[y];
        sum[y] = 0.0f;
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[y] += exp_of(tile.acc[m][y][i] - from);
    }
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) sum[y] += __shfl_xor(sum[y], 16);
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) sum[y] += __shfl_xor(sum[y], 32);
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) {
        float hit = 0.0f;
        if (__any(at[y] < wave_end)) {
            const int64_t t = t0 + Tile::at_y(y);
            for (int e = entry[y], cls = at[y]; cls < wave_end;) {
                const int rel = cls - base;
                const float q = targets.q ? targets.q[t * targets.k + e] : 1.0f;
                float z = 0.0f;
#pragma unroll
                for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z = rel == 16 * m + i ? tile.acc[m][y][i] : z;
                z *= unit;
                hit += q == 0.0f ? 0.0f : q * z;
                if (kept.target_z && rel >= 0 && rel < Tile::SX * 16 && (rel & 15) < 4) kept.target_z[t * targets.k + e] = z;
                cls = ++e < targets.k ? targets.cls[t * targets.k + e] : kNoClass;
            }
            hit += __shfl_xor(hit, 16);
            hit += __shfl_xor(hit, 32);
        }
        if (lane < 16) shared[Tile::wave() % WX][Tile::at_y(y)] = make_float3(top[y], sum[y], hit);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < YT && t0 + r < n; r += WX * WY * kWave) {
        float all = -INFINITY, total = 0.0f, hit = 0.0f;
#pragma unroll
        for (int x = 0; x < WX; ++x) all = fmaxf(all, shared[x][r].x);
        const float from = all == -INFINITY ? 0.0f : all;
#pragma unroll
        for (int x = 0; x < WX; ++x) {
            const float3 v = shared[x][r];
            total += v.y * exp_of(v.x - from);
            hit += v.z;
        }
        sums[static_cast<int64_t>(tx) * n + t0 + r] = make_float2(all * unit, total);
        hits[static_cast<int64_t>(tx) * n + t0 + r] = hit;
    }
    if (!kept.g || c0 >= kept.cols) return;
    u16 *const to = kept.g + t0 * kept.ldg + c0;
    if constexpr (kept_whole(TYPE == DQ_F32, XT)) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
            tile.store(to + p * kept.plane, kept.ldg, YT, XT, [&](int m, int y) {
                u16x4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = static_cast<u16>(__float_as_uint(tile.acc[m][y][i]) >> (16 * p));
                return r;
            });
    } else {
#pragma unroll
        for (int y = 0; y < Tile::SY; ++y)
#pragma unroll
            for (int x = 0; x < WX; ++x) top[y] = fmaxf(top[y], shared[x][Tile::at_y(y)].x);
        tile.store(to, kept.ldg, YT, XT, [&](int m, int y) {
            const f32x4 v = tile.acc[m][y];
            typedef __attribute__((ext_vector_type(2))) uint32_t Two;
            return __builtin_bit_cast(u16x4, Two{KeptUnit<TYPE>::codes(top[y], v[0], v[1]), KeptUnit<TYPE>::codes(top[y], v[2], v[3])});
        });
    }
}

// What is told of a row when its tiles are through.
struct Finish {
    const float2 *sums;
    const float *hits;
    int slots;                         // tiles
    const float *entropy;
    float tau2;
    float *loss, *lse_out;             // nullable
    uint32_t *status;
    __device__ __forceinline__ void tell(const Targets &targets, int64_t t, float lse, float hit) const
    {
        const bool live = targets.used(t);
        const float value = live ? tau2 * ((entropy ? entropy[t] : 0.0f) + (lse - hit)) : 0.0f;
        if (loss) loss[t] = value;
        if (lse_out) lse_out[t] = lse;
        const bool far = !targets.q && targets.cls[t] >= static_cast<int64_t>(targets.c);       // (a teacher's were looked at before)
        // (a teacher's logits that are not finite, and targets with a score of -inf, show in the loss alone)
        const uint32_t said = (live && !(__builtin_isfinite(lse) && __builtin_isfinite(value)) ? 1u : 0u) | (far ? 2u : 0u);
        if (said && status) atomicOr(status, said);
    }
};

// lse and the targets' sum q z of row t from its tiles; ROWS rows a block of 256, all threads of a row get them.
template <int ROWS>
__device__ __forceinline__ float row_lse(const Finish &f, int64_t n, int64_t t, float &hit)
{
    constexpr int kParts = 256 / ROWS;
    __shared__ float tops[kParts][ROWS];
    __shared__ float2 rest[kParts][ROWS];
    const int row = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    float top = -INFINITY;
    if (t < n)
        for (int s = part; s < f.slots; s += kParts) top = fmaxf(top, f.sums[s * n + t].x);
    tops[part][row] = top;
    __syncthreads();
    for (int o = kParts / 2; o; o /= 2) {
        if (part < o) tops[part][row] = fmaxf(tops[part][row], tops[part + o][row]);
        __syncthreads();
    }
    top = tops[0][row];
    const float from = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    hit = 0.0f;
    if (t < n)
        for (int s = part; s < f.slots; s += kParts) {
            const float2 v = f.sums[s * n + t];
            sum += v.y * expf(v.x - from);
            hit += f.hits[s * n + t];
        }
    rest[part][row] = make_float2(sum, hit);
    __syncthreads();
    for (int o = kParts / 2; o; o /= 2) {
        if (part < o) {
            rest[part][row].x += rest[part + o][row].x;
            rest[part][row].y += rest[part + o][row].y;
        }
        __syncthreads();
    }
    hit = rest[0][row].y;
    return top + logf(rest[0][row].x);
}

// ROWS rows a block, 256 / ROWS threads a row: one where there are few rows, else kFinishRows.
constexpr int kFinishFew = 256, kFinishRows = 16;
static int64_t finish_blocks(int64_t n) { return n <= kFinishFew ? n : (n + kFinishRows - 1) / kFinishRows; }
template <int ROWS>
__global__ __launch_bounds__(256) void finish_kernel(Finish f, int64_t n, Targets targets, float *__restrict__ lse_kept)
{
    const int64_t t = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x % ROWS;
    float hit;
    const float lse = row_lse<ROWS>(f, n, t, hit);
    if (threadIdx.x >= ROWS || t >= n) return;
    f.tell(targets, t, lse, hit);
    if (lse_kept) lse_kept[t] = lse;
}

// ---- gradients -----------------------------------------------------------------
// What a row's gradients are multiplied by in g.
template <int TYPE>
__device__ __forceinline__ float row_factor(const float *weight, const float *weight_max, int64_t t, bool live)
{
    const float f = live && weight ? weight[t] : 1.0f;
    return TYPE == DQ_F16 ? f * (kF16Unit / (weight ? weight_max[0] : 1.0f)) : f;
}

// g of the first piece from what was kept of its scores, in its place: columns 0 .. cols of `rows` rows.  A block takes 2048 columns of
// a row, eight a thread, and then the targets among them.  What bounds it is memory: it reads and writes g once.
// FINISH: the rows' lse are not made by a launch of their own but here, by each block for itself (few rows of few spans: 16 x 1000 x 256
// in float32 34 us a pass, with the launch 38).
template <int TYPE, int XT, bool FINISH>
__global__ __launch_bounds__(256) void kept_kernel(Kept kept, int64_t cols, int64_t rows, int64_t n, Finish finish, Targets targets,
                                                   const float *__restrict__ lse, const float *__restrict__ weight,
                                                   const float *__restrict__ weight_max)
{
    typedef __attribute__((ext_vector_type(8))) u16 Eight;
    constexpr bool kWhole = kept_whole(TYPE == DQ_F32, XT);
    constexpr int kPlanes = TYPE == DQ_F32 ? 3 : 1;
    const int64_t first = blockIdx.x * 2048ll, i = first + threadIdx.x * 8;
    for (int64_t t = blockIdx.y; t < rows; t += gridDim.y) {
        const bool live = t < n && targets.used(t);
        u16 *const row = kept.g + t * kept.ldg;
        float from = 0.0f;
        if constexpr (FINISH) {
            if (t < n) {
                float hit;
                from = row_lse<1>(finish, n, t, hit);
                if (blockIdx.x == 0 && threadIdx.x == 0) finish.tell(targets, t, from, hit);
            }
        } else if (live) {
            from = lse[t];
        }
        const float f = row_factor<TYPE>(weight, weight_max, t, live);
        // (the thread's first entry: every thread looks at its own, which is one trip to memory where a search is one for each halving)
        const int32_t *const cls = targets.cls + t * targets.k;
        const int e0 = static_cast<int>(threadIdx.x), mine = live && e0 < targets.k ? cls[e0] : kNoClass;
        if (i < cols) {
            Eight out[kPlanes] = {};
            if (live) {
                const Eight lo = *reinterpret_cast<const Eight *>(row + i);
                float p[8];
                if constexpr (kWhole) {
                    const Eight hi = *reinterpret_cast<const Eight *>(row + kept.plane + i);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = __uint_as_float(static_cast<uint32_t>(hi[e]) << 16 | lo[e]) - from;
                        p[e] = TYPE == DQ_F32 ? expf(z) : exp_near(z);
                    }
                } else {
                    const float shift = (finish.sums[i / XT * n + t].x - from) * kLog2E;
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = KeptUnit<TYPE>::value(lo[e], shift);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (TYPE == DQ_F32) {
                        u16 part[3];
                        parts_of(f * p[e], part);
#pragma unroll
                        for (int h = 0; h < 3; ++h) out[h][e] = part[h];
                    } else {
                        out[0][e] = Num<TYPE>::store(f * p[e]);
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < kPlanes; ++h) *reinterpret_cast<Eight *>(row + h * kept.plane + i) = out[h];
        }
        __syncthreads();
        if (!live) continue;
        const int end = static_cast<int>(lesser(first + 2048, kept.cols));
        for (int e = e0, j = mine; e < targets.k; e += 256, j = e < targets.k ? cls[e] : kNoClass) {
            if (j < first || j >= end || (e && cls[e - 1] == j)) continue;           // (the first of a class that comes several times takes them all)
            const float z = kept.target_z[t * targets.k + e] - from;
            float v = TYPE == DQ_F32 ? expf(z) : exp_near(z);
            for (int o = e; o < targets.k && cls[o] == j; ++o) v -= targets.q ? targets.q[t * targets.k + o] : 1.0f;
            if constexpr (TYPE == DQ_F32) {
                u16 part[3];
                parts_of(f * v, part);
#pragma unroll
                for (int h = 0; h < 3; ++h) row[h * kept.plane + j] = part[h];
            } else {
                row[j] = Num<TYPE>::store(f * v);
            }
        }
    }
}

// g of another piece of the classes, [rows of the tiles][ldg] in 16 bits (three planes for float32); zeros where there is no row or class.
template <int WHAT, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave, 2) void grad_kernel(Operand w, Operand a, int64_t k, int64_t n, int64_t c, int64_t piece0,
                                                             int64_t piece, float inv_tau, Targets targets, const float *__restrict__ lse,
                                                             const float *__restrict__ weight, const float *__restrict__ weight_max,
                                                             int tiles_x, int tiles_y, u16 *__restrict__ g, int64_t ldg, int64_t plane)
{
    constexpr int TYPE = WHAT & 3;
    typedef TileProduct<typename Num<TYPE>::Mul, XT, YT, WX, WY, false, false, H, R, P, (WHAT & kEdge) != 0> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t c0 = piece0 + static_cast<int64_t>(tx) * XT, t0 = static_cast<int64_t>(ty) * YT;
    Tile tile;
    tile.run(w, a, c0, t0, 0, k);
    const int wave_c0 = static_cast<int>(c0) + Tile::sub_x(0) * 16;
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) {
        const int64_t t = t0 + Tile::at_y(y);
        const bool live = t < n && targets.used(t);
        const int base = static_cast<int>(c0) + Tile::at_x(0);
        const float from = live ? lse[t] : 0.0f;
        const float f = row_factor<TYPE>(weight, weight_max, t, live);
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float z = tile.acc[m][y][i] * inv_tau - from;
                tile.acc[m][y][i] = TYPE == DQ_F32 ? expf(z) : exp_near(z);
            }
        if (live) {
            const int end = min(wave_c0 + Tile::SX * 16, static_cast<int>(c));
            const int32_t *cls = targets.cls + t * targets.k;
            for (int e = targets.first(t, wave_c0); e < targets.k && cls[e] < end; ++e) {
                const int rel = cls[e] - base;
                const float q = targets.q ? targets.q[t * targets.k + e] : 1.0f;
#pragma unroll
                for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) tile.acc[m][y][i] -= rel == 16 * m + i ? q : 0.0f;
            }
        }
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) tile.acc[m][y][i] = live && base + 16 * m + i < c ? f * tile.acc[m][y][i] : 0.0f;
    }
    u16 *const to = g + t0 * ldg + (c0 - piece0);
    if constexpr (TYPE == DQ_F32) {
#pragma unroll
        for (int p = 0; p < 3; ++p)                // (each part is taken off before the next is)
            tile.store(to + p * plane, ldg, YT, XT, [&](int m, int n) {
                u16x4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = tile.acc[m][n][i];
                    r[i] = Part::store(v);
                    tile.acc[m][n][i] = __builtin_isfinite(Part::load(r[i])) ? v - Part::load(r[i]) : 0.0f;
                }
                return r;
            });
    } else {
        tile.store(to, ldg, YT, XT, [&](int m, int n) { return quad_of<TYPE>(tile.acc[m][n]); });
    }
}

__device__ __forceinline__ float gradient_unit(int type, float post, const float *weight_max)
{
    return type == DQ_F16 ? post * ((weight_max ? weight_max[0] : 1.0f) / kF16Unit) : post;
}

// (Matrix cores: 8192 x 47236 x 4096 in bfloat16 2.15 to 2.20 ms, 1440 to 1475 TFLOP/s.)
// da of a piece, one split of its classes per blockIdx.y: partial sums [split][n][ldp] in float32, added to what the pieces before left.
// Where one launch has it all (partial null) da itself.
template <int TYPE, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave, 2) void da_kernel(Operand w, Operand g, int64_t piece, int64_t per_split, int64_t n, int64_t d, int tiles_x,
                                                           int tiles_y, float *__restrict__ partial, int64_t ldp, int first, Targets targets, float post,
                                                           const float *__restrict__ weight_max, typename Num<TYPE>::Mem *__restrict__ da,
                                                           int64_t ldda, int vector)
{
    typedef TileProduct<typename Num<TYPE>::Mul, XT, YT, WX, WY, true, false, H, R, P> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, t0 = static_cast<int64_t>(ty) * YT, k0 = blockIdx.y * per_split;
    const int64_t k1 = lesser(k0 + per_split, piece);
    if (k0 >= k1 && !first) return;
    Tile tile;
    tile.run(w, g, i0, t0, k0, k0 < k1 ? k1 : k0);
    float *const out = partial + blockIdx.y * n * ldp;
    const float unit = gradient_unit(TYPE, post, weight_max);
#pragma unroll
    for (int y = 0; y < Tile::SY; ++y) {
        const int64_t t = t0 + Tile::at_y(y);
        if (t >= n) continue;
        const bool live = partial || targets.used(t);
#pragma unroll
        for (int m = 0; m < Tile::SX; ++m) {
            const int64_t i = i0 + Tile::at_x(m);
            if (i >= d) continue;
            if (partial) {
                f32x4 *const to = reinterpret_cast<f32x4 *>(out + t * ldp + i);
                *to = first ? tile.acc[m][y] : *to + tile.acc[m][y];
            } else {
                store_four<TYPE>(da + t * ldda + i, live ? tile.acc[m][y] * unit : f32x4{0.f, 0.f, 0.f, 0.f}, static_cast<int>(lesser(4, d - i)), vector);
            }
        }
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void da_finish_kernel(const float *__restrict__ partial, int splits, int64_t n, int64_t d, int64_t ldp, Targets targets,
                                                        float post, const float *__restrict__ weight_max, typename Num<TYPE>::Mem *__restrict__ da,
                                                        int64_t ldda, int vector)
{
    const int64_t quads = (d + 3) / 4, total = n * quads;
    const float unit = gradient_unit(TYPE, post, weight_max);
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < total; at += gridDim.x * 256ll) {
        const int64_t t = at / quads, i = (at - t * quads) * 4;
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        if (targets.used(t)) {
#pragma unroll 4
            for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4 *>(partial + (s * n + t) * ldp + i);
            v *= unit;
        }
        store_four<TYPE>(da + t * ldda + i, v, static_cast<int>(lesser(4, d - i)), vector);
    }
}

// dw of a piece.  Both operands are stored across k: no LDS bank is met twice, and half tiles, two blocks to a compute unit, are the
// faster ones (8192 x 47236 x 4096 in bfloat16 2.29, 256 x 256 2.46 ms; on other cards 2.33 to 2.50, 1270 to 1360 TFLOP/s).  16-bit half tiles need two
// registers more than there are and keep them in scratch memory (12 bytes a lane).
template <int TYPE, int XT, int YT, int WX, int WY, int H, int R, int P>
__global__ __launch_bounds__(WX *WY *kWave, 2) void dw_kernel(Operand a, Operand g, int64_t k, int64_t piece, int64_t d, int tiles_x, int tiles_y,
                                                           float post, const float *__restrict__ weight_max,
                                                           typename Num<TYPE>::Mem *__restrict__ dw, int64_t lddw)
{
    typedef TileProduct<typename Num<TYPE>::Mul, XT, YT, WX, WY, true, true, H, R, P> Tile;
    int tx, ty;
    tile_of_block(blockIdx.x, tiles_x, tiles_y, tx, ty);
    const int64_t i0 = static_cast<int64_t>(tx) * XT, j0 = static_cast<int64_t>(ty) * YT;
    Tile tile;
    tile.run(a, g, i0, j0, 0, k);
    const float unit = gradient_unit(TYPE, post, weight_max);
    tile.store(dw + j0 * lddw + i0, lddw, piece - j0, d - i0, [&](int m, int n) { return quad_of<TYPE>(tile.acc[m][n] * unit); });
}

// ---- host ----------------------------------------------------------------------
static inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
static inline int64_t room(int64_t &at, int64_t bytes)
{
    const int64_t here = at;
    at = up(at + bytes, 256);
    return here;
}

// Sizes and places of everything a call passes through its workspace.
struct ClassPlan {
    int32_t type, planes, wide;         // wide: bytes of a number in memory
    int64_t n, c, d, k, dp;             // dp: columns of packed rows
    bool direct_a, direct_w;
    TileSize tile, tile_da, tile_dw;
    TileDims td, td_da, td_dw;
    int64_t tiles_x, tiles_y;           // of scores
    int64_t piece, pieces, ldg, rows_g, rows_z, planes_g, splits, per_split;
    bool da_at_once;
    int64_t cls, q, entropy, weight_max, lse, target_z, sums, hits, a, w, az, g, partial, bytes;
};

static int32_t class_plan(const dq_classes *p, int64_t k, bool grad, ClassPlan &s)
{
    if (!p || p->n <= 0 || p->c <= 0 || p->d <= 0 || k < 0 || !p->a || !p->w || p->lda < p->d || p->ldw < p->d) return DQ_ERR_INVALID_ARG;
    if (p->type != DQ_F32 && p->type != DQ_F16 && p->type != DQ_BF16) return DQ_ERR_INVALID_ARG;
    s = ClassPlan{};
    s.type = p->type;
    s.planes = p->type == DQ_F32 ? 3 : 1;
    s.wide = p->type == DQ_F32 ? 4 : 2;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(p->a), pw = reinterpret_cast<uintptr_t>(p->w);
    if (pa % s.wide || pw % s.wide) return DQ_ERR_INVALID_ARG;
    constexpr int64_t kMost = 1ll << 30;
    if (p->n > kMost || p->c > kMost || p->d > (1 << 20) || p->lda > (1 << 22) || p->ldw > (1 << 22)) return DQ_ERR_UNSUPPORTED;
    if (k > DQ_MAX_TEACHER) return DQ_ERR_UNSUPPORTED;
    s.n = p->n;
    s.c = p->c;
    s.d = p->d;
    s.k = k ? k : 1;
    s.dp = up(s.d, 64);
    // Read in place where rows are whole 16-byte chunks, also if they end inside of a step of 32 columns.
    s.direct_a = s.planes == 1 && s.d % 8 == 0 && p->lda % 8 == 0 && pa % 16 == 0;
    s.direct_w = s.planes == 1 && s.d % 8 == 0 && p->ldw % 8 == 0 && pw % 16 == 0;
    const bool parts = s.planes > 1;
    s.tile = tile_for_rows(s.c, s.n, parts, true);
    s.td = dims_of(s.tile, parts, false);
    s.tiles_x = (s.c + s.td.x - 1) / s.td.x;
    s.tiles_y = (s.n + s.td.y - 1) / s.td.y;
    if (!launchable(s.tiles_x * s.tiles_y, threads_of(s.tile)) || !launchable(finish_blocks(s.n), 256) || (k && !launchable(s.n, kTeacherThreads)))
        return DQ_ERR_UNSUPPORTED;
    int64_t at = 0;
    s.cls = room(at, k ? 4 * s.n * s.k : 0);
    s.q = room(at, k ? 4 * s.n * s.k : 0);
    s.entropy = room(at, k ? 4 * s.n : 0);
    s.weight_max = room(at, 4);
    s.lse = room(at, 4 * s.n);
    s.sums = room(at, 8 * s.tiles_x * s.n);
    s.hits = room(at, 4 * s.tiles_x * s.n);
    s.a = room(at, s.direct_a ? 0 : 2 * s.planes * s.n * s.dp);
    s.w = room(at, s.direct_w ? 0 : 2 * s.planes * s.c * s.dp);
    if (grad) {
        s.rows_z = up(s.n, 32);
        s.rows_g = s.tiles_y * s.td.y;
        s.planes_g = planes_of_g(parts, s.td.x);
        s.piece = piece_of(s.c, s.rows_g, s.planes_g);
        s.pieces = ceil_div(s.c, s.piece);
        s.ldg = s.piece;
        s.tile_dw = tile_for_dw(s.n, s.c, s.d, s.piece, parts);
        s.td_dw = dims_of(s.tile_dw, parts, true);
        s.tile_da = tile_for_da(s.n, s.d);
        s.td_da = dims_of(s.tile_da, parts, true);
        if (!launchable(tiles_of(s.d, std::min(s.c, s.piece), s.td_dw), threads_of(s.tile_dw)) || !launchable(tiles_of(s.d, s.n, s.td_da), threads_of(s.tile_da)))
            return DQ_ERR_UNSUPPORTED;
        s.per_split = da_split(s.n, s.d, s.piece, parts);
        s.splits = ceil_div(s.piece, s.per_split);
        s.da_at_once = s.splits == 1 && s.pieces == 1;
        s.az = room(at, 2 * s.planes * s.rows_z * s.dp);
        s.target_z = room(at, 4 * s.n * s.k);
        s.g = room(at, 2 * s.planes_g * s.rows_g * s.ldg);
        s.partial = room(at, s.da_at_once ? 0 : 4 * s.splits * s.n * s.dp);
    }
    s.bytes = up(at, 16);
    return DQ_OK;
}

struct ClassCall {
    const dq_classes *prob;
    const int32_t *label;
    const dq_teacher *teacher;
    const float *weight;
    float scale;
    float *loss, *lse;
    void *da;
    int64_t ldda;
    void *dw;
    int64_t lddw;
    bool grad;
    uint32_t *status;
    char *ws;
    hipStream_t st;
};

template <int TYPE>
static int32_t class_run(const ClassCall &q, const ClassPlan &s)
{
    typedef typename Num<TYPE>::Mem Mem;
    const dq_classes &p = *q.prob;
    char *const ws = q.ws;
    const hipStream_t st = q.st;
    const int64_t n = s.n, c = s.c, wide = s.wide;
    const float tau = q.teacher ? q.teacher->tau : 1.0f;
    Targets targets{q.label, nullptr, static_cast<int32_t>(s.k), static_cast<uint32_t>(c)};
    const float *entropy = nullptr;
    if (q.teacher) {
        int pow2 = 1;
        while (pow2 < s.k) pow2 *= 2;
        int32_t *const cls = reinterpret_cast<int32_t *>(ws + s.cls);
        float *const tq = reinterpret_cast<float *>(ws + s.q), *const ent = reinterpret_cast<float *>(ws + s.entropy);
        teacher_kernel<<<static_cast<unsigned>(n), kTeacherThreads, 0, st>>>(q.teacher->cls, q.teacher->logit, q.teacher->ld, targets.k, pow2, c,
                                                                             1.0f / tau, cls, tq, ent, q.status);
        DQ_LAUNCH_CHECK();
        targets.cls = cls;
        targets.q = tq;
        entropy = ent;
    }

    // operands: in place, or packed
    const bool want_dw = q.grad && q.dw;
    const int32_t dp = static_cast<int32_t>(s.dp);
    Operand a{static_cast<const char *>(p.a), p.lda * 2, n, static_cast<int32_t>(s.d), 0}, w{static_cast<const char *>(p.w), p.ldw * 2, c, static_cast<int32_t>(s.d), 0};
    if (!s.direct_a) a = Operand{ws + s.a, s.dp * 2, n, dp, n * s.dp * 2};
    if (!s.direct_w) w = Operand{ws + s.w, s.dp * 2, c, dp, c * s.dp * 2};
    const Operand az{ws + s.az, s.dp * 2, s.rows_z, dp, s.rows_z * s.dp * 2};
    const int64_t of_a = s.direct_a && !want_dw ? 0 : (want_dw ? s.rows_z : n) * s.dp / 8, of_w = s.direct_w ? 0 : c * s.dp / 8;
    if (of_a + of_w) {
        const Packed pa{p.a, p.lda, n, s.d, s.direct_a ? nullptr : reinterpret_cast<u16 *>(ws + s.a), want_dw ? reinterpret_cast<u16 *>(ws + s.az) : nullptr,
                        n, s.rows_z};
        const Packed pw{p.w, p.ldw, c, s.d, reinterpret_cast<u16 *>(ws + s.w), nullptr, c, 0};
        const int64_t blocks = std::min<int64_t>((of_a + of_w + 255) / 256, 1 << 16);
        pack_kernel<TYPE><<<static_cast<unsigned>(blocks), 256, 0, st>>>(pa, pw, s.dp, of_a, of_a + of_w, targets);
        DQ_LAUNCH_CHECK();
    }
    const int64_t kd = up(s.d, 32);
    float2 *const sums = reinterpret_cast<float2 *>(ws + s.sums);
    float *const hits = reinterpret_cast<float *>(ws + s.hits), *const lse = reinterpret_cast<float *>(ws + s.lse);
    const int tiles_x = static_cast<int>(s.tiles_x), tiles_y = static_cast<int>(s.tiles_y);
    constexpr bool kInParts = TYPE == DQ_F32;
    dim3 grid(static_cast<unsigned>(tiles_x * tiles_y));
    // gradients: kept of the first piece
    const bool products = q.grad && (q.da || q.dw);
    const int64_t plane = s.rows_g * s.ldg;
    u16 *const g = reinterpret_cast<u16 *>(ws + s.g);
    const Kept kept = products ? Kept{g, s.ldg, plane, std::min(s.piece, c), reinterpret_cast<float *>(ws + s.target_z)} : Kept{};
    // (Rows that end inside of a step: the smaller tiles' stages are two steps, and look in any case.  float32 has no half tiles.)
    constexpr int kEdged = kInParts ? TYPE : TYPE | kEdge;
    const bool edge = (s.direct_a || s.direct_w) && s.d % 32;
#define DQ_EDGE(kernel, size, ...) edge ? DQ_TILE_LAUNCH(kernel, kEdged, size, __VA_ARGS__) : DQ_TILE_LAUNCH(kernel, TYPE, size, __VA_ARGS__)
#define DQ_SCORES w, a, kd, n, c, 1.0f / tau, targets, tiles_x, tiles_y, sums, hits, kept
    switch (s.tile) {
    case kTileLarge: DQ_EDGE(scores_kernel, Large, DQ_SCORES); break;
    case kTileHalf:
        if constexpr (kInParts) return DQ_ERR_UNSUPPORTED;
        else DQ_EDGE(scores_kernel, Half, DQ_SCORES);
        break;
    case kTileMiddle: DQ_EDGE(scores_kernel, Middle, DQ_SCORES); break;
    case kTileFew: DQ_TILE_LAUNCH(scores_kernel, TYPE, Few, DQ_SCORES); break;
    case kTileFewest: DQ_TILE_LAUNCH(scores_kernel, TYPE, Fewest, DQ_SCORES); break;
    }
#undef DQ_SCORES
    DQ_LAUNCH_CHECK();
    const Finish finish{sums, hits, tiles_x, entropy, tau * tau, q.loss, q.lse, q.status};
    const bool finish_later = products && s.pieces == 1 && n <= 256 && c <= 4096 && s.td.x < 256;      // (by the gradients' first kernel)
    if (!finish_later) {
        const unsigned blocks = static_cast<unsigned>(finish_blocks(n));
        if (n <= kFinishFew) finish_kernel<1><<<blocks, 256, 0, st>>>(finish, n, targets, q.grad ? lse : nullptr);
        else finish_kernel<kFinishRows><<<blocks, 256, 0, st>>>(finish, n, targets, q.grad ? lse : nullptr);
        DQ_LAUNCH_CHECK();
    }
    if (!products) return DQ_OK;

    const float post = q.scale * tau;
    float *weight_max = nullptr;
    if (TYPE == DQ_F16 && q.weight) {
        weight_max = reinterpret_cast<float *>(ws + s.weight_max);
        weight_max_kernel<<<1, 1024, 0, st>>>(q.weight, n, targets, weight_max);
        DQ_LAUNCH_CHECK();
    }
    float *const partial = s.da_at_once ? nullptr : reinterpret_cast<float *>(ws + s.partial);
    const int64_t rows_k = std::min(s.rows_g, s.rows_z);           // of g: nothing else of it is read
    const Operand go{reinterpret_cast<const char *>(g), s.ldg * 2, rows_k, static_cast<int32_t>(s.ldg), plane * 2};
    const int vector_da = four_at_once(q.da, q.ldda, static_cast<int>(wide));
    Mem *const da = static_cast<Mem *>(q.da);
    for (int64_t at = 0; at < c; at += s.piece) {
        const int64_t have = std::min(s.piece, c - at);
        if (at == 0) {
            const int64_t cols = up(have, 32);
            const dim3 spans(static_cast<unsigned>((cols + 2047) / 2048), static_cast<unsigned>(std::min<int64_t>(rows_k, 65535)));
#define DQ_KEPT(x, later) kept_kernel<TYPE, x, later><<<spans, 256, 0, st>>>(kept, cols, rows_k, n, finish, targets, lse, q.weight, weight_max)
            if (kept_whole(kInParts, s.td.x)) {
                finish_later ? DQ_KEPT(64, true) : DQ_KEPT(64, false);
            } else if constexpr (!kInParts) {
                if (s.td.x == 256) DQ_KEPT(256, false);          // (too many classes or rows to finish later)
                else finish_later ? DQ_KEPT(128, true) : DQ_KEPT(128, false);
            }
#undef DQ_KEPT
        } else {
            const int tiles_p = static_cast<int>((have + s.td.x - 1) / s.td.x);
            grid = dim3(static_cast<unsigned>(tiles_p * tiles_y));
            // (Several pieces are 21 turns of large tiles or more: middle ones, 1.05 times as long at best, are not taken.)
#define DQ_GRAD w, a, kd, n, c, at, have, 1.0f / tau, targets, lse, q.weight, weight_max, tiles_p, tiles_y, g, s.ldg, plane
            switch (s.tile) {
            case kTileLarge: DQ_EDGE(grad_kernel, Large, DQ_GRAD); break;
            case kTileHalf:
                if constexpr (kInParts) return DQ_ERR_UNSUPPORTED;
                else DQ_EDGE(grad_kernel, Half, DQ_GRAD);
                break;
            case kTileMiddle: return DQ_ERR_UNSUPPORTED;
            case kTileFew: DQ_TILE_LAUNCH(grad_kernel, TYPE, Few, DQ_GRAD); break;
            case kTileFewest: DQ_TILE_LAUNCH(grad_kernel, TYPE, Fewest, DQ_GRAD); break;
            }
#undef DQ_GRAD
        }
        DQ_LAUNCH_CHECK();
        if (q.da) {
            const Operand piece{w.p + at * w.ld, w.ld, c - at, w.cols, w.plane};
            const int tx = static_cast<int>((s.d + s.td_da.x - 1) / s.td_da.x), ty = static_cast<int>((n + s.td_da.y - 1) / s.td_da.y);
            grid = dim3(static_cast<unsigned>(tx * ty), static_cast<unsigned>(s.splits));
#define DQ_DA piece, go, up(have, 32), s.per_split, n, s.d, tx, ty, partial, s.dp, at == 0, targets, post, weight_max, da, q.ldda, vector_da
            switch (s.tile_da) {
            case kTileLarge: DQ_TILE_LAUNCH(da_kernel, TYPE, Large, DQ_DA); break;
            case kTileMiddle: DQ_TILE_LAUNCH(da_kernel, TYPE, Middle, DQ_DA); break;
            case kTileFew: DQ_TILE_LAUNCH(da_kernel, TYPE, Few, DQ_DA); break;
            case kTileFewest: DQ_TILE_LAUNCH(da_kernel, TYPE, FewestAcross, DQ_DA); break;
            case kTileHalf: return DQ_ERR_UNSUPPORTED;           // (never: tile_for_da)
            }
#undef DQ_DA
            DQ_LAUNCH_CHECK();
        }
        if (q.dw) {
            const int tx = static_cast<int>((s.d + s.td_dw.x - 1) / s.td_dw.x), ty = static_cast<int>((have + s.td_dw.y - 1) / s.td_dw.y);
            grid = dim3(static_cast<unsigned>(tx * ty));
#define DQ_DW az, go, s.rows_z, have, s.d, tx, ty, post, weight_max, static_cast<Mem *>(q.dw) + at * q.lddw, q.lddw
            switch (s.tile_dw) {                                 // (half ones are through before large ones wherever there are any)
            case kTileLarge:
                if constexpr (kInParts) DQ_TILE_LAUNCH(dw_kernel, TYPE, Large, DQ_DW);
                else return DQ_ERR_UNSUPPORTED;
                break;
            case kTileHalf:
                if constexpr (kInParts) return DQ_ERR_UNSUPPORTED;
                else DQ_TILE_LAUNCH(dw_kernel, TYPE, Half, DQ_DW);
                break;
            case kTileMiddle: DQ_TILE_LAUNCH(dw_kernel, TYPE, Middle, DQ_DW); break;
            case kTileFew: DQ_TILE_LAUNCH(dw_kernel, TYPE, Few, DQ_DW); break;
            case kTileFewest: return DQ_ERR_UNSUPPORTED;         // (never: tile_for_dw)
            }
#undef DQ_DW
            DQ_LAUNCH_CHECK();
        }
    }
#undef DQ_EDGE
    if (q.da && partial) {
        const int64_t blocks = std::min<int64_t>((n * ((s.d + 3) / 4) + 255) / 256, 1 << 16);
        da_finish_kernel<TYPE><<<static_cast<unsigned>(blocks), 256, 0, st>>>(partial, static_cast<int>(s.splits), n, s.d, s.dp, targets, post, weight_max, da,
                                                                              q.ldda, vector_da);
        DQ_LAUNCH_CHECK();
    }
    return DQ_OK;
}

static int32_t class_call(ClassCall &q, void *ws, int64_t ws_bytes)
{
    ClassPlan s;
    const int64_t k = q.teacher ? q.teacher->k : 0;
    if (q.teacher && (k <= 0 || !q.teacher->cls || !q.teacher->logit || q.teacher->ld < k || !(q.teacher->tau > 0.0f) ||
                      !__builtin_isfinite(q.teacher->tau) || !__builtin_isfinite(1.0f / q.teacher->tau)))
        return DQ_ERR_INVALID_ARG;
    if (!q.teacher && !q.label) return DQ_ERR_INVALID_ARG;
    if (const int32_t e = class_plan(q.prob, k, q.grad, s)) return e;
    const int32_t wide = s.wide;
    if ((q.da && (q.ldda < s.d || reinterpret_cast<uintptr_t>(q.da) % wide)) || (q.dw && (q.lddw < s.d || reinterpret_cast<uintptr_t>(q.dw) % wide)))
        return DQ_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws)) return DQ_ERR_INVALID_ARG;
    if (ws_bytes < s.bytes) return DQ_ERR_WORKSPACE;
    q.ws = static_cast<char *>(ws);
    switch (s.type) {
    case DQ_F32: return class_run<DQ_F32>(q, s);
    case DQ_F16: return class_run<DQ_F16>(q, s);
    default: return class_run<DQ_BF16>(q, s);
    }
}

}  // namespace dq

extern "C" int64_t dq_class_workspace_bytes(int32_t op, const dq_classes *prob, int64_t k)
{
    if (op != DQ_OP_CLASS_LOSS && op != DQ_OP_CLASS_GRAD) return DQ_ERR_INVALID_ARG;
    dq::ClassPlan s;
    const int32_t e = dq::class_plan(prob, k, op == DQ_OP_CLASS_GRAD, s);
    return e ? e : s.bytes;
}

extern "C" int32_t dq_class_loss(const dq_classes *prob, const int32_t *label, float *loss_out, float *lse_out, uint32_t *status, void *ws,
                                 int64_t ws_bytes, void *stream)
{
    if (!loss_out) return DQ_ERR_INVALID_ARG;
    dq::ClassCall q{prob, label, nullptr, nullptr, 1.0f, loss_out, lse_out, nullptr, 0, nullptr, 0, false, status, nullptr, static_cast<hipStream_t>(stream)};
    return dq::class_call(q, ws, ws_bytes);
}

extern "C" int32_t dq_class_grad(const dq_classes *prob, const int32_t *label, const float *weight, float scale, float *loss_out, float *lse_out,
                                 void *da_out, int64_t ldda, void *dw_out, int64_t lddw, uint32_t *status, void *ws, int64_t ws_bytes, void *stream)
{
    dq::ClassCall q{prob, label, nullptr, weight, scale, loss_out, lse_out, da_out, ldda, dw_out, lddw, true, status, nullptr, static_cast<hipStream_t>(stream)};
    return dq::class_call(q, ws, ws_bytes);
}

extern "C" int32_t dq_distill_loss(const dq_classes *prob, const dq_teacher *teacher, float *loss_out, float *lse_out, uint32_t *status, void *ws,
                                   int64_t ws_bytes, void *stream)
{
    if (!loss_out || !teacher) return DQ_ERR_INVALID_ARG;
    dq::ClassCall q{prob, nullptr, teacher, nullptr, 1.0f, loss_out, lse_out, nullptr, 0, nullptr, 0, false, status, nullptr, static_cast<hipStream_t>(stream)};
    return dq::class_call(q, ws, ws_bytes);
}

extern "C" int32_t dq_distill_grad(const dq_classes *prob, const dq_teacher *teacher, const float *weight, float scale, float *loss_out,
                                   float *lse_out, void *da_out, int64_t ldda, void *dw_out, int64_t lddw, uint32_t *status, void *ws, int64_t ws_bytes,
                                   void *stream)
{
    if (!teacher) return DQ_ERR_INVALID_ARG;
    dq::ClassCall q{prob, nullptr, teacher, weight, scale, loss_out, lse_out, da_out, ldda, dw_out, lddw, true, status, nullptr, static_cast<hipStream_t>(stream)};
    return dq::class_call(q, ws, ws_bytes);
}
