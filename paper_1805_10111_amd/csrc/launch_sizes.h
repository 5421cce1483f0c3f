// Sizes that the host works out for a launch: plain C++, no HIP, so that they can be checked over their whole range
// without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace dq {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t packed_words(int64_t d, int b) { return (d * b + 31) / 32; }
inline int64_t pad4(int64_t d) { return (d + 3) / 4 * 4; }
// A dimension of a launch has fewer than 2^32 threads.
inline bool launchable(int64_t blocks, int threads) { return blocks <= 0xffffffffll / threads; }

// ------------------------------------------------------------------ full gradient on dense features (grad_dense.hip)
// Threads per block and float4 columns per thread on rows of more than 1024 floats: of 256 to 512 threads in whole
// wavefronts, as few as cover the row with 1, 2, 4 or 8 columns each.
struct FullShape {
    int threads, cols;
};

inline FullShape full_shape(int64_t d)
{
    const int64_t quads = ceil_div(d, 4);
    const int cols = quads <= 512 ? 1 : quads <= 1024 ? 2 : quads <= 2048 ? 4 : 8;
    const int64_t threads = ceil_div(ceil_div(quads, cols), 64) * 64;
    return FullShape{static_cast<int>(threads < 256 ? 256 : threads), cols};
}

// Of a thread's `cols` columns the first so many lie inside the row for every thread and need no mask, in any shape that
// full_shape gives: threads * full_whole_cols(cols) <= d / 4.  Rounding up to whole wavefronts adds up to 63 quads per
// column; with eight columns those can pass the end by more than the last column (8197 floats: 320 threads, seven
// columns of them 2240 quads of 2050).
constexpr int full_whole_cols(int cols) { return cols >= 8 ? cols - 2 : cols - 1; }

// ------------------------------------------------------------------ worker step on CSR features (grad_csr.hip)
constexpr int kColBits = 20;                     // staged entries carry column | row << kColBits
constexpr int kCsrMaxRows = 256;                 // rows a block handles per pass (LDS metadata)
constexpr int kMaxStage = 8192;                  // most entries the staging buffer is given
constexpr int64_t kMinStage = 4096;              // least entries it is given beside one of several windows
constexpr int64_t kLdsBudget = 152 * 1024;       // of the 160 KB per compute unit
constexpr int64_t kCsrFixedLds = 10 * 1024;      // static arrays, rounded up

// LDS plan for a d-vector plus the staging buffer.  When both fit, the vector is one window; otherwise it is built
// in several equal windows (multiples of 4 columns) that leave room for at least kMinStage staged entries.
// Columns carry the row number in the bits above kColBits while staged, hence the limit on d.
struct CsrPlan {
    int win;        // columns per window
    int cap;        // staged (column, value) entries
    int nwin;
    size_t lds;     // bytes of dynamic LDS: window + staging
};

// A staged entry takes 12 bytes of LDS, 16 when the caller needs two sums per row (no cached margins).
inline bool csr_plan(int64_t d, bool second, CsrPlan &p)
{
    if (d >= (1ll << kColBits)) return false;
    const int64_t budget = kLdsBudget - kCsrFixedLds;                     // bytes for window + staging
    const int64_t each = second ? 16 : 12;
    int64_t nwin = 1;
    if (pad4(d) * 4 + each * 512 > budget) nwin = ceil_div(pad4(d) * 4, budget - each * kMinStage);
    const int64_t win = pad4(ceil_div(pad4(d), nwin));
    int64_t cap = (budget - win * 4) / each;
    if (cap > kMaxStage) cap = kMaxStage;
    p.lds = static_cast<size_t>(win * 4 + cap * each);
    p.win = static_cast<int>(win);
    p.cap = static_cast<int>(cap);
    p.nwin = static_cast<int>(ceil_div(pad4(d), win));
    return true;
}

// A mini-batch prepared ahead of its round: layout in 32-bit words (see grad_csr.hip) of its tables for B rows, for `cap`
// entries.  The kernels with cached margins lay it out for the rows of the batch, those without for kCsrMaxRows; the master,
// which does not know which of them reads next, writes one word of it, so that word lies in the same place in every
// layout: the row starts come first, as many as a block takes, and it is the last behind them.
struct PrepLayout {
    int pre, dev_max;  // (see WorkerArgs::dev_max)
    int row, len, y, z, entries;
    constexpr explicit PrepLayout(int B)
        : pre(4), dev_max(pre + kCsrMaxRows + 3), row(dev_max + 1), len(row + (B + 3) / 4 * 4), y(len + (B + 3) / 4 * 4),
          z(y + (B + 3) / 4 * 4), entries(z + (B + 3) / 4 * 4) {}
};
constexpr int kPrepEntries = PrepLayout(kCsrMaxRows).entries;
constexpr int64_t kPrepInts(int64_t cap) { return kPrepEntries + (2 * cap + 3) / 4 * 4; }

// Words per worker that the workspace holds for one: room for what the plan for one sum per row stages.
inline int64_t csr_prep_stride(int64_t d)
{
    CsrPlan one_sum;
    return csr_plan(d, false, one_sum) ? kPrepInts(one_sum.cap) : 0;
}

// Most entries of a mini-batch that is prepared ahead for a step with this plan.  Not the plan's capacity: without cached
// margins the vector may take more windows than with them, narrower ones, which leave MORE entries for staging than the
// workspace has room for (47,236 columns: 5151 against 4244; 34,400: 4788 against 650).
inline int csr_prep_cap(int64_t d, const CsrPlan &plan)
{
    CsrPlan one_sum;
    if (!csr_plan(d, false, one_sum)) return 0;
    return plan.cap < one_sum.cap ? plan.cap : one_sum.cap;
}

// A step's workspace: M rows of the gradient, then kMaxSlices maxima and as many counts per worker.  A run's has its own behind
// them: pad4(d) words and twice M times csr_prep_stride(d).
constexpr int kMaxSlices = 8;                    // blocks that share a worker's step
inline int64_t csr_run_offset(int64_t d, int64_t M) { return M * pad4(d) * 4 + M * kMaxSlices * 8; }
inline int64_t csr_run_bytes(int64_t d, int64_t M) { return csr_run_offset(d, M) + pad4(d) * 4 + 2 * M * csr_prep_stride(d) * 4; }

// What a run's workspace holds behind its M rows and slice results.
// Either the difference of model and snapshot, a word per column, and the two sets of prepared mini-batches; or, where the
// worker kernel quantizes the model and has no use for that row, two sets of mini-batches in all of it, whose entries
// can have the snapshot at their column beside them.
struct PrepRoom {
    int64_t stride;     // words per worker
    int cap;            // most entries of a mini-batch
    int snap_cap;       // most entries that have the snapshot value beside them
};

inline PrepRoom csr_prep_room(int64_t d, int64_t M, int64_t B, const CsrPlan &plan, bool snaps)
{
    if (!snaps) return PrepRoom{csr_prep_stride(d), csr_prep_cap(d, plan), 0};
    PrepRoom r{};
    r.stride = (pad4(d) + 2 * M * csr_prep_stride(d)) / (2 * M) / 4 * 4;
    const int64_t room = r.stride - PrepLayout(static_cast<int>(B)).entries;
    r.cap = static_cast<int>(room / 2 < plan.cap ? room / 2 : plan.cap);
    r.snap_cap = static_cast<int>(room / 3 < r.cap ? room / 3 : r.cap);
    return r;
}

// Whether mini-batches of B of the n rows are light enough for what the worker kernel does entry by entry instead of column by
// column elsewhere: quantizing the model, in every block, instead of a launch of its own; and, in Alg. 2, finding ||alpha||_inf
// (see csr_run_layout): on average little more entries than a block keeps in its registers
// (`in_flight`), and no more than it can prepare ahead (`cap`, with an eighth to spare for batches above the average).
// `entries` is what the caller says the matrix holds; unknown (0), rows of 100 are assumed.
// Measured, Alg. 1, eight workers, us a round with a launch for the model and without: 4200 columns, 485 entries 11.7 and 9.7,
// 4757 entries 13.3 and 13.0, 6627 entries 15.1 and 15.8, 9515 (not prepared) 24.5 and 27.2; 20,958 columns, 1656 entries 13.0 and
// 11.5, 9518 (not prepared) 27.6 and 31.8; 32,000 columns, 1656 (not prepared) 19.9 and 21.0, 12,693 (not prepared) 60.2 and 74.0.
// 25 workers: 4200 columns, 4757 entries 16.4 both; 14,000 columns, 4759 entries 17.9 and 18.1, 3838 entries 17.4 and 17.0.
inline bool csr_light_batches(int64_t B, int64_t n, int64_t entries, int in_flight, int cap)
{
    const double mean = static_cast<double>(B) * (entries > 0 ? static_cast<double>(entries) / static_cast<double>(n) : 100.0);
    return mean <= 1.2 * in_flight && mean * 1.125 <= cap;
}

// ------------------------------------------------------------------ blocks that work together on one die (die.h)
constexpr uint32_t kDies = 16;                   // (numbers that a die may have; the part has eight)

// The die where a launch has most blocks (count_of a number), `own` where it has none; of several with as many the first from number
// lot % 8 on: launches that hold equal parts of all dies pick different ones, seven times of eight.
template <typename CountOf>
constexpr uint32_t die_pick(CountOf count_of, uint32_t own, uint32_t lot)
{
    uint32_t best = own, most = 0;
    for (uint32_t i = 0; i < kDies; ++i) {
        const uint32_t at = (i + lot % 8) % kDies, c = count_of(at);
        if (c > most) {
            most = c;
            best = at;
        }
    }
    return best;
}

// ------------------------------------------------------------------ rounds on one die, CSR features (csr_rounds.hip)
constexpr int kDieUnits = 32;                    // compute units of a die
constexpr int kRoundsRows = 128;                 // rows of a mini-batch: two a lane of the wavefront that lays them out
constexpr int kBusyWaves = 15, kBusy = kBusyWaves * 64;       // all but the wavefront that waits at exchanges
constexpr int kUnitWaves = kBusyWaves - 1;       // (not the one that lays out mini-batches)
constexpr int kEntriesEach = 8;                  // entries a thread holds; with more of them the rows are read in the round
constexpr int kChunk = 256;                      // columns of a chunk: a quad a lane
constexpr int kMostChunks = 7, kColumns = 2;     // of a member, and columns a thread
constexpr int kPasses = 2;                       // chunks of all workers that a wavefront takes in turn
constexpr int64_t kFewRounds = 8;                // calls of fewer are not for one die
constexpr int64_t kRoundsFixedLds = 13360;       // static arrays
constexpr int64_t kRoundsLds = 160 * 1024 - kRoundsFixedLds;  // for the dynamic part
constexpr int64_t kRoundsControl = 848;          // bytes of a run's workspace, from csr_run_offset on, for what the members share

static_assert(kMostChunks * kChunk <= kColumns * kBusy, "every column has a thread");

struct CsrRoundsShape {
    int S, win;                                  // slices of a worker, columns of one
    int want, chunks;                            // members, chunks of one
    int cap;                                     // entries of a group of rows (CsrPlan::cap)
    int room;                                    // entries that LDS has room for
    int64_t lds;                                 // bytes of dynamic LDS
};

// false: these rounds are not for one die.  They are where measured faster than launches (us a round, 30 rounds a call unless
// said; launches, then this):
//  - the snapshot has room in LDS: d 26,323, M 12, read from L2 instead: 13.1, 18.2; d 38,834, M 8: 16.1, 19.1.
//  - no wavefront has more than two chunks of gradients to quantize, which stay in registers: M 8, d 20,958 (24 chunks a
//    member) 11.4, 9.9; M 4, d 28,409 12.6, 11.3; M 28, d 5000 12.7, 10.7; M 21, d 4340 12.2, 10.1; M 1, d 300 9.0, 7.7; M 8,
//    d 20,000, b_x 12 16.4, 11.5; M 20, d 6385, batches of 128 17.2, 14.5.  With four: M 10, d 20,958 12.0, 12.7; M 16, d
//    12,000 11.6, 12.7; M 32, d 6400 13.3, 14.0.
//  - calls of eight rounds or more: the launches around it, and finding together, are 10 us a call.  M 8, d 20,958: two rounds
//    12.5, 15.2; five 11.8, 12.0; eight 11.6, 11.2.
//  - mini-batches that the busy threads hold in registers, as far as the caller's count of entries can tell.  It cannot tell uneven
//    rows, nor any where it is not given; larger batches are read in the round.  M 8, d 20,958, 64 rows of 50 entries in the mean,
//    lognormal with sigma 1, 1.5 and 2: 14.8, 12.4; 20.7, 15.6; 29.5, 20.2; no count, 32 rows of 200 and of 1000: 26.6, 18.1; 87, 51.
inline bool csr_rounds_shape(int64_t d, int64_t n, int64_t entries, int64_t M, int64_t B, int b_x, int64_t rounds, CsrRoundsShape &s)
{
    const auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    const auto most = [](int64_t a, int64_t b) { return a > b ? a : b; };
    CsrPlan plan;
    if (b_x < 2 || b_x > 16 || B > kRoundsRows || M > kDieUnits || rounds < kFewRounds || !csr_plan(d, false, plan)) return false;
    const int64_t S = least(least(kDieUnits / M, 16), ceil_div(d, 256));
    s.win = static_cast<int>(ceil_div(ceil_div(d, S), 256) * 256);
    s.S = static_cast<int>(ceil_div(d, s.win));
    s.want = static_cast<int>(most(M * s.S, least(kDieUnits, ceil_div(d, kChunk))));
    const int64_t chunks = ceil_div(ceil_div(d, kChunk), s.want);
    if (chunks > kMostChunks || M * chunks > kPasses * kUnitWaves) return false;
    s.chunks = static_cast<int>(chunks);
    const double mean = static_cast<double>(B) * (entries > 0 ? static_cast<double>(entries) / static_cast<double>(n) : 100.0);
    s.cap = plan.cap;
    const int64_t held = least(plan.cap, kEntriesEach * kBusy);
    if (mean * 1.25 > static_cast<double>(held)) return false;
    const int64_t room = most(M * chunks * (kChunk / 4), least(held, static_cast<int64_t>(1.5 * mean) + 256));
    s.room = static_cast<int>(ceil_div(room, 64) * 64);
    const int64_t message = pad4((d * b_x + 31) / 32 + 1);
    int64_t bytes = (s.win + message + s.room + pad4(d)) * 4;
    if (bytes > kRoundsLds) return false;
    // (what is left is for larger mini-batches than the mean's, as far as the threads hold them)
    const int64_t more = least((kRoundsLds - bytes) / 256 * 64, most(0, held / 64 * 64 - s.room));
    s.room += static_cast<int>(more);
    bytes += more * 4;
    // (what makes up more than half of a compute unit's LDS: no two blocks on one)
    s.lds = most(bytes, 72 * 1024);
    return true;
}

// ------------------------------------------------------------------ products of many-class models (matrix_tile.h, classes.hip, mx4.hip)
// Tiles of the products, and how many of their blocks a compute unit has at a time.
enum TileSize { kTileLarge, kTileHalf, kTileMiddle, kTileFew, kTileFewest };
struct TileDims {
    int x, y;
};
// x by y results a tile.  float32 in parts takes three times the room in LDS, and tiles half as high (and no half ones).  The last: 64 by
// 16 rows, of 128 columns where x is stored across k.
constexpr TileDims dims_of(TileSize s, bool parts, bool across)
{
    return s == kTileLarge ? TileDims{256, parts ? 128 : 256} : s == kTileHalf ? TileDims{256, 128} : s == kTileMiddle ? TileDims{128, parts ? 64 : 128} :
           s == kTileFew ? TileDims{64, 64} : TileDims{across ? 128 : 64, 16};
}
inline int64_t tiles_of(int64_t x, int64_t y, TileDims t) { return (x + t.x - 1) / t.x * ((y + t.y - 1) / t.y); }
constexpr int threads_of(TileSize s) { return s == kTileLarge ? 512 : 256; }

// The tile that is through first, of large ones (one block to a compute unit, 256 of which take 1), half ones and middle ones (two; where 256
// or fewer are left over, each has a compute unit to itself and takes 0.6 as long).  Measured on large products in bfloat16: 512 half ones take
// 1.1 (operands along k: 8192 x 47236 x 4096 in 2.81 and 3.10 ms), both operands across k 0.93 (47236 x 4096 x 8192 in 2.46 and 2.29 ms),
// 512 middle ones 0.7 for their half of the work.
inline TileSize tile_for(int64_t x, int64_t y, bool parts, bool half, bool across)
{
    auto pairs = [](int64_t tiles, double each) { return each * (static_cast<double>(tiles / 512) + (tiles % 512 > 256 ? 1.0 : tiles % 512 ? 0.6 : 0.0)); };
    const double large = static_cast<double>((tiles_of(x, y, dims_of(kTileLarge, parts, across)) + 255) / 256);
    const double halves = half && !parts ? pairs(tiles_of(x, y, dims_of(kTileHalf, parts, across)), across ? 0.93 : 1.1) : large;
    const double middle = pairs(tiles_of(x, y, dims_of(kTileMiddle, parts, across)), 0.7);
    return middle < large && middle < halves ? kTileMiddle : halves < large ? kTileHalf : kTileLarge;
}
// ... of products over `rows` rows.
inline TileSize tile_for_rows(int64_t x, int64_t rows, bool parts, bool half)
{
    return rows <= 16 ? kTileFewest : rows <= 64 ? kTileFew : tile_for(x, rows, parts, half, false);
}
// ... of dW, c classes (a piece at a time) of d columns.  Few rows of few classes: small tiles, of which there are more.
inline TileSize tile_for_dw(int64_t n, int64_t c, int64_t d, int64_t piece, bool parts)
{
    return n <= 64 && c * d <= (1 << 20) ? kTileFew : tile_for(d, c < piece ? c : piece, parts, true, true);
}
// ... of da, n rows of d columns.
inline TileSize tile_for_da(int64_t n, int64_t d) { return n <= 16 ? kTileFewest : n <= 64 ? kTileFew : n * d <= 256 * 1024 ? kTileMiddle : kTileLarge; }

// Whether 32 bits of each score are kept for the gradients, in tiles of x classes (up to 64 rows), and 16-bit planes of scores or gradients.
constexpr bool kept_whole(bool parts, int x) { return parts || x <= 64; }
constexpr int planes_of_g(bool parts, int x) { return parts ? 3 : kept_whole(parts, x) ? 2 : 1; }

// Bytes of g.  What is kept of the first piece need not be multiplied again: 8192 rows of 47236 classes (774 MB) in pieces of 512 MB 9.0 ms,
// in one 8.1; the workspace is a three-hundredth of the card's memory.
constexpr int64_t kPieceBytes = 1024ll << 20;
// Classes of a piece of c: all (in whole tiles), or as many as there is room for, as the first one's scores are kept.
inline int64_t piece_of(int64_t c, int64_t rows, int planes)
{
    const int64_t room = kPieceBytes / (2 * planes * rows) / 256, most = (room > 1 ? room : 1) * 256;
    return c > most ? most : ceil_div(c, 256) * 256;
}

// Classes of one split of da's piece.  da has few tiles: its classes are split until the chip is full (a block per compute unit, smaller
// tiles two or more), though not below four steps each.  (Few rows of few classes in 16 bits are not split at all: one launch less, 64 x 1000 x
// 4096 41 -> 35 us and 16 x 1000 x 256 34 -> 31 us a pass; in float32, whose steps are six products, the same takes 34.5 -> 38 us.)
inline int64_t da_split(int64_t n, int64_t d, int64_t piece, bool parts)
{
    const TileSize tile = tile_for_da(n, d);
    const int64_t tiles = tiles_of(d, n, dims_of(tile, parts, true)), blocks = tile == kTileLarge ? 256 : 512;
    const auto between = [](int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; };
    const int64_t most = !parts && n <= 64 && piece <= 1024 ? 1 : between(piece / 128, 1, between(blocks / tiles, 1, blocks));
    int64_t splits = 1;
    double best = 1e30;
    for (int64_t i = 1; i <= most; ++i) {                // fewest rounds for the work of one split, and something for its sums
        const double cost = static_cast<double>((tiles * i + blocks - 1) / blocks) / static_cast<double>(i) * (1.0 + 0.01 * static_cast<double>(i));
        if (cost < best) {
            best = cost;
            splits = i;
        }
    }
    return ceil_div(ceil_div(piece, splits), 32) * 32;
}

// ------------------------------------------------------------------ orthogonalized updates (orthogonal.hip)
#if defined(__HIPCC__)
#define DQ_HOST_DEVICE __host__ __device__
#else
#define DQ_HOST_DEVICE
#endif
// A symmetric product of `side` rows over k (or `jobs` of them): only tiles that reach to the diagonal or below it are made, and k is split until the chip is full;
// the tiles' sums of every split are added up by a second launch.  Row ty of tiles begins with tile ty.
// (All tiles' stages dealt out evenly, so that a block begins and ends anywhere in a tile: blocks that share rows then read them at different times, and
// 136 tiles over 47236 took 1070 us instead of 685, over 4096 in two parts 380 instead of 215.)
struct GramPlan {
    TileSize size;
    TileDims dims;
    int tiles_x, tiles, splits;
    int64_t per_split;
    bool at_once;             // small squares: tiles of 64 x 64 over all of k, each of which ends what it began, and no second launch
    int64_t floats() const { return static_cast<int64_t>(tiles) * splits * dims.x * dims.y; }
};
DQ_HOST_DEVICE constexpr int gram_before(int ty) { return ty * (ty - 1) / 2; }      // tiles that rows 0 .. ty - 1 leave out
// products: of the matrix cores for one of two numbers (1, 3).  Times in us: a stage of 32 of k takes, for each of them, 0.74 where a compute unit has one large
// tile, 0.5 where it has two middle ones (0.3 one of them), whatever they are 0.4 of a small one; a unit of work begins and ends in about 8 stages, and its sums are
// written and read by a launch that takes 7 and half of one a split.  (Small tiles split, float32: 10000 x 128 249 -> 186 us a pass, 20000 x 64 294 -> 213.)
constexpr int64_t kGramAtOnce = 1408;           // (253 tiles of 64 x 64 at the diagonal and below it)
inline GramPlan gram_plan(int64_t side, int64_t k, int products, int jobs)
{
    GramPlan best{};
    double least = 1e300;
    for (int i = 0; i < (side <= kGramAtOnce ? 4 : 2); ++i) {
        if (i == 2 && products == 1) continue;                    // (middle tiles were never slower)
        GramPlan p{};
        p.at_once = i == 3;
        p.size = i == 0 ? kTileLarge : i == 1 ? kTileMiddle : kTileFew;
        p.dims = dims_of(p.size, false, false);
        p.tiles_x = static_cast<int>(ceil_div(side, p.dims.x));
        p.tiles = p.tiles_x * p.tiles_x - gram_before(p.tiles_x);
        const int64_t stages = ceil_div(k, 32);
        for (int splits = 1; splits <= (p.at_once ? 1 : 64) && splits <= stages; ++splits) {
            p.per_split = ceil_div(stages, splits) * 32;
            p.splits = static_cast<int>(ceil_div(k, p.per_split));
            if (p.splits != splits) continue;
            const int64_t units = static_cast<int64_t>(p.tiles) * splits * jobs, full = units / 512, left = units % 512;
            const double each = (static_cast<double>(p.per_split / 32) + 8.0) * products;
            const double rounds = p.size == kTileLarge ? 0.74 * static_cast<double>(ceil_div(units, 256)) : p.size == kTileFew ? 0.4 / products * static_cast<double>(ceil_div(units, 256)) :
                                  0.5 * static_cast<double>(full) + (left > 256 ? 0.5 : left ? 0.3 : 0.0);
            const double cost = each * rounds + (p.at_once ? 0.0 : 7.0 + 0.5 * splits + static_cast<double>(p.floats() * jobs) * 8.0 / 4.5e6);
            if (cost < least) {
                least = cost;
                best = p;
            }
        }
    }
    return best;
}
// Whether two products go together, in one launch: where one leaves much of the chip idle.  Five steps in float16, one after the other and together: 256 x 256 157 and
// 134 us, 1000 x 1000 328 and 299, 1500 x 1500 589 and 545, 2500 x 2500 1736 and 1564; of large tiles 3000 x 3000 2123 and 2168, 4096 x 4096 4885 and 4967.  (2048 x
// 2048, 408 middle tiles, stays apart, 1019, where together it took 947.)
inline bool gram_together(const GramPlan &p) { return static_cast<int64_t>(p.tiles) * p.splits <= (p.size == kTileLarge ? 64 : 256); }
// Whether 16-bit updates of `side` by `deep` go through the small matrices: float16 always, bfloat16 where that is faster than step by step (about 2.5 side^2 deep and
// 32 side^3 against 20 and 9): us for five steps of 1000 x 1000 299 and 262, x 1250 312 and 325, x 2000 319 and 392; 2500 x 3000 1581 and 1535; 4096 x 4096
// 4917 and 3977, x 5000 5099 and 5425, x 8192 5245 and 6731; 100 x 4000 125 and 161.  (Small ones near the border are 5 us, of 150 to 220, off it either way.)
inline bool small_matrices(int64_t side, int64_t deep, bool f16) { return f16 || 5 * deep > 6 * side; }
// Tiles of X's next value, rows x cols numbers.
inline TileSize update_tile(int64_t cols, int64_t rows)
{
    return tiles_of(cols, rows, dims_of(kTileMiddle, false, false)) <= 128 ? kTileFew : tile_for(cols, rows, false, false, false);
}

// ------------------------------------------------------------------ products of 8-bit matrices (fp8.hip)
// n rows by c results over `groups` blocks of 128: one row or two in strips of 16 results, few rows in strips of 64 results by 64 rows, else in tiles; where that
// leaves the chip idle the blocks are split, an even number of them a split, and a second launch adds the splits' sums up.
// Strips are right up to 64 rows, with float32 results (whose tiles need both matrices in bfloat16 first) up to 128: 128 x 47236 x 4096 132 us, in tiles
// 216; with 16-bit results of more than 16 rows only where there are few tiles (17 x 4096 x 4096 13.2 us, in
// tiles 17.0; 64 x 8192 x 4096 19.7 and 15.8).
constexpr int64_t kFewestRows8 = 2, kFewRows8 = 64;
constexpr bool in_strips(int64_t n, int64_t c, bool f32) { return n <= 16 || (f32 ? n <= 2 * kFewRows8 : n <= kFewRows8 && c <= 4096); }
struct ProductPlan {
    bool few;
    TileSize size;
    int64_t tiles_x, tiles_y, splits, per_split;
    int64_t sums_bytes(int64_t n, int64_t c) const { return splits > 1 ? ceil_div(4 * splits * n * c, 16) * 16 : 0; }
};
// Times in us: of a block of 128, 0.9 where a compute unit has one large tile, 0.6 where it has up to two middle ones, 0.7 of a strip of 64
// (three to a compute unit), 0.25 a wavefront of a strip of 16 (four to a strip, eight strips to a compute unit); begin and end as long as
// eight; the second launch 6, and what it reads and writes.
inline ProductPlan product_plan(int64_t n, int64_t c, int64_t groups, bool f32)
{
    ProductPlan best{};
    best.few = in_strips(n, c, f32);
    best.size = best.few ? kTileFewest : tile_for(c, n, false, false, false);
    const bool fewest = n <= kFewestRows8;
    const TileDims t = fewest ? TileDims{16, static_cast<int>(kFewestRows8)} : best.few ? TileDims{64, static_cast<int>(kFewRows8)} : dims_of(best.size, false, false);
    best.tiles_x = ceil_div(c, t.x);
    best.tiles_y = ceil_div(n, t.y);
    const int64_t tiles = best.tiles_x * best.tiles_y, room = fewest ? 2048 : best.few ? 768 : best.size == kTileLarge ? 256 : 512;
    double least = 1e300;
    for (int64_t splits = 1; splits <= 64; ++splits) {
        const int64_t per = ceil_div(ceil_div(groups, splits), 2) * 2;
        if (ceil_div(groups, per) != splits) continue;
        const double each = fewest ? 0.25 * (static_cast<double>(per) / 4.0 + 8.0) : best.few ? 0.7 * (static_cast<double>(per) + 8.0) : (best.size == kTileLarge ? 0.9 : 0.6) * (static_cast<double>(per) + 8.0);
        const double cost = each * static_cast<double>(ceil_div(tiles * splits, room)) + (splits > 1 ? 6.0 + static_cast<double>(n * c) * (4.0 + 8.0 * static_cast<double>(splits)) / 4.5e6 : 0.0);
        if (cost < least) {
            least = cost;
            best.splits = splits;
            best.per_split = per;
        }
    }
    return best;
}

}  // namespace dq
