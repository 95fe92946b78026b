// The head's operators: entry points, shapes and workspaces (kernels: head_kernels.h, products: head_tile.h).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "head_kernels.h"

namespace svip {

static bool dtype_ok(int d) { return d == SVIP_F32 || d == SVIP_BF16 || d == SVIP_F16; }
static int size_of(int d) { return d == SVIP_F32 ? 4 : 2; }
static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
static int up(int n, int to) { return (n + to - 1) / to * to; }
static int ceil_div(long long n, long long d) { return (int)((n + d - 1) / d); }

constexpr int HEAD_MAX_ROWS = 1 << 20;                 // of hidden states
constexpr int HEAD_MAX_VOCAB = 1 << 22;
constexpr int HEAD_MAX_WIDTH = 1 << 17;                // hidden channels
constexpr long long HEAD_MAX_STRIDE = 1 << 23;         // elements: 256 rows of a tile lie within 32 bits of bytes

constexpr long long MOST_THREADS = 0xffffffffLL;       // of a launch

// A matrix of rows x cols of dtype: stride of a row in whole 16 bytes, within reach of a tile's 32-bit offsets.
static svip_status check_matrix(const void *p, int dtype, int cols, long long stride)
{
    if (stride < cols || stride > HEAD_MAX_STRIDE) return SVIP_ERR_SHAPE;
    return aligned16(p) && stride * size_of(dtype) % 16 == 0 ? SVIP_OK : SVIP_ERR_ALIGN;
}

template <typename A>
static bool launch(void (*kernel)(A), long long grid, unsigned block, hipStream_t st, const A &args)
{
    if (grid <= 0 || grid * block > MOST_THREADS) return false;
    A copy = args;
    void *argv[] = {&copy};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)grid), dim3(block), argv, 0, st) == hipSuccess;
}

template <typename F>
static bool by_dtype(int d, F f)
{
    if (d == SVIP_F32) return f(std::integral_constant<int, SVIP_F32>{});
    if (d == SVIP_BF16) return f(std::integral_constant<int, SVIP_BF16>{});
    return f(std::integral_constant<int, SVIP_F16>{});
}

// ---- shapes of the tiles -------------------------------------------------------------------------------------------------------------------

// m x n of a workgroup's tile, its waves along either, buffers in LDS.
using Large = TileShape<256, 256, 2, 4, 2>;            // one workgroup a CU
using Middle = TileShape<128, 128, 2, 2, 2>;           // two
using Small = TileShape<128, 64, 4, 1, 3>;             // two: up to 64 rows wait for the weight's bytes, and a tile has them all
using Few = TileShape<128, 32, 4, 1, 4>;               // two: up to 32 rows; both also for more rows of a small vocabulary
using Narrow = TileShape<64, 32, 4, 1, 4>;             // three: 8-bit and fp32 logits of a vocabulary too small to fill the chip with tiles of 128
// of 8-bit matrices (16-bit logits of many rows: Large and Middle)
using Middle8 = TileShape<128, 128, 2, 2, 3>;          // fp32 logits (the tile's bf16 fragments need the registers)
enum ShapeId { LARGE, MIDDLE, SMALL, FEW, NARROW };

constexpr int FEW_ROWS = 64, FEWER_ROWS = 32;
constexpr int CUS = 256;
constexpr int MOST_TILE = 256;                         // tokens of a tile

// What the products are made of.
enum Kind { HALVES, SINGLES, CODES };                  // 16-bit values, fp32 as it is, 8-bit codes

static int tile_rows(ShapeId id) { return id == LARGE ? Large::BM : id == NARROW ? Narrow::BM : Middle::BM; }
// Time of a product of m x n over `steps` steps, in units of 1 us or so: 5 us, and for each step of a round of tiles what one takes alone on a
// CU or next to a second one.  16-bit values in large tiles, of which a CU holds one: 1.4 us a step; in smaller ones less for the tile, but more for
// the product.  So many tiles go faster as large ones (loss of 8192 x 151936 x 2048: 3690 us against 4820), and where large ones would leave CUs
// without work as smaller ones.  Measured, large / middle / small / few: loss of 129 x 32000 x 1024: 27 / 23 us; 300 x 32000 x 1024: 32.7 / 33.7 / 41.2 /
// 44.7; 128 x 32000 x 4096: 88 / 65 / 59 / 72; 200 x 8000 x 2048: 44.7 / 28.2 / 18.5 / 21.7; 360 x 1533 x 4064: 82 / 54 / 31 / 27; gradients of 1000 x 5000 x
// 1024: 125 / 91.  The fp32 instruction keeps a CU busy with one tile, two take twice as long: loss of 128 x 32000 x 1024: middle 70, small 69, few 73 us;
// 200 x 20000 x 1024: 124 / 99 / 89; 337 x 1164 x 3504: 211 / 115 / 66, narrow 41; loss and gradients of 700 x 1200 x 1024 with the weight's in middle / small /
// few: 130 / 108 / 106, of 128 x 32000 x 1024: 299 / 304 / 319.  8-bit tiles, whose steps are twice as many values, take 1.65 us and 8 us, middle
// ones 1.08 us and 3.8 us (logits of 1088 x 128256 x 4096: 610 us against 691; 325 x 50257 x 5120: 149 against 135; 100 x 32000 x 1024:
// 20 against 13).
static double tiles_cost(Kind kind, ShapeId id, long long m, long long n, int splits, double steps)
{
    static constexpr int BN[] = {Large::BN, Middle::BN, Small::BN, Few::BN, Narrow::BN};
    static constexpr double ALONE[] = {1.4, 0.7, 0.35, 0.25}, PAIR[] = {1.4, 0.85, 0.5, 0.4}, SINGLE[] = {0.0, 1.85, 0.97, 0.53, 0.29};
    const int rows = tile_rows(id);
    const long long tiles = ((m + rows - 1) / rows) * ((n + BN[id] - 1) / BN[id]) * splits, at_once = id == LARGE ? CUS : 2 * CUS;
    const double rounds = (double)((tiles + at_once - 1) / at_once);
    if (kind == SINGLES) return 5.0 + (double)((tiles + CUS - 1) / CUS) * SINGLE[id] * steps;
    if (kind == CODES) return rounds * (id == LARGE ? 8.0 + 1.65 * steps : 3.8 + 1.08 * steps);
    return rounds * (5.0 + (tiles <= CUS ? ALONE : PAIR)[id] * steps);
}
static ShapeId fastest(Kind kind, ShapeId first, ShapeId last, long long m, long long n, double steps)
{
    ShapeId best = first;
    for (int id = first + 1; id <= last; ++id)
        if (tiles_cost(kind, (ShapeId)id, m, n, 1, steps) < tiles_cost(kind, best, m, n, 1, steps)) best = (ShapeId)id;
    return best;
}
// f with the shape of that number, of those from FIRST to LAST.
template <ShapeId FIRST, ShapeId LAST, typename F>
static bool by_shape(ShapeId id, F f)
{
    if constexpr (FIRST <= LARGE)
        if (id == LARGE) return f(Large{});
    if (id == MIDDLE) return f(Middle{});
    if constexpr (LAST >= SMALL)
        if (id == SMALL) return f(Small{});
    if constexpr (LAST >= FEW)
        if (id == FEW) return f(Few{});
    if constexpr (LAST >= NARROW)
        if (id == NARROW) return f(Narrow{});
    return false;
}

// fp32 values go as two fp16 parts, at a third of the rate of 16-bit values and nearly three times that of fp32 products, where that gains more than
// laying out the parts costs: in us, a few launches and 12 bytes (gradients: 16) for each value of the weight.  The line is drawn on the side of the
// values as they are, which lose nothing.  Measured, in parts / as they are (with the loss as it is, where it differs), 32000 x 1024: loss of 128 rows
// 118 / 69, 200 rows 120 / 125, 300 rows 149 / 160, 512 rows 150 / 242; loss and gradients of 128 rows 360 / 298, 200 rows 425 / 514, 300 rows
// 510 / 682 (517), 512 rows 569 / 1001; 128256 x 2048: loss of 200 rows 1002 / 942, 300 rows 1195 / 1209; loss and gradients of 128
// rows 2737 / 2091, 200 rows 3058 / 3821 (2951), 300 rows 3757 / 5164.
static bool in_parts(int dtype, int call, int rows, int vocab, int width)
{
    const double weight = (double)vocab * width, product = 2.0 * rows * weight;
    if (dtype != SVIP_F32 || rows <= FEW_ROWS) return false;
    return call == SVIP_HEAD_LOSS_GRAD ? 100.0 + weight * 16 / 4.2e6 + 9.0 * product / 0.9e9 < 3.0 * product / 115e6
                                       : 60.0 + weight * 12 / 4.2e6 + 3.0 * product / 1e9 < product / 115e6;
}

// f with what the products are made of, their terms and the dtype.
template <typename F>
static bool by_product(int dtype, bool parts, F f)
{
    constexpr std::integral_constant<int, 1> one{};
    if (dtype == SVIP_BF16) return f(Bf16{}, one, std::integral_constant<int, SVIP_BF16>{});
    if (dtype == SVIP_F16) return f(F16{}, one, std::integral_constant<int, SVIP_F16>{});
    if (parts) return f(F16{}, std::integral_constant<int, 3>{}, std::integral_constant<int, SVIP_F32>{});
    return f(F32{}, one, std::integral_constant<int, SVIP_F32>{});
}
// The shapes that products of these come in: fp32 as it is in no large ones, in parts in no small ones.
template <typename T, int TERMS>
constexpr ShapeId first_shape() { return std::is_same<T, F32>::value ? MIDDLE : LARGE; }
template <typename T, int TERMS>
constexpr ShapeId last_shape() { return TERMS == 3 ? MIDDLE : std::is_same<T, F32>::value ? NARROW : FEW; }

// ---- workspace ---------------------------------------------------------------------------------------------------------------------------------

constexpr size_t HEAD_HEADER = 512;                    // flag word (256 bytes), HeadScalars
constexpr size_t PIECE_BYTES = (size_t)256 << 20;      // of a piece's softmax: what the memory-side cache holds
constexpr int LEAST_PIECE = 2048;                      // tokens
constexpr int MOST_SPLITS = 128;
constexpr size_t SPLIT_BYTES = (size_t)128 << 20;

struct HeadPlan {
    bool parts;                // fp32 as two fp16 parts
    bool fine;                 // 16-bit G' in two parts, with the rows' weights, for the gradient of the weight
    int planes, size, width;   // planes and bytes of what the products are made of; channels of its rows
    int piece;                 // tokens of a piece of the vocabulary, a multiple of MOST_TILE (of a loss without parts: nearly always all)
    ShapeId logits, hidden_grad, weight_grad;
    int splits, per_split;     // of a piece's tokens in the gradient of the hidden states
    size_t part, target, rows, maxima, hidden_parts, weighted, weight, grad, sum, bytes;     // offsets
    long long grad_stride;
};

// Splits of K in 8-bit logits of few rows whose tiles would leave CUs without work: as many as there are places for, of at least 8 steps each (2 rows x 5000
// x 4096: 15.5 us in one, 9.4 us in four with the join).  *per_split: of K.
static bool narrow_logits(int N, int V) { return N <= FEWER_ROWS && ceil_div(V, Small::BM) < 2 * CUS; }
static int logits_splits(int N, int V, int K, int *per_split)
{
    const int steps = ceil_div(K, QBLOCK);
    const long long tiles = narrow_logits(N, V) ? ceil_div(V, Narrow::BM) : ceil_div(V, Small::BM), places = narrow_logits(N, V) ? 3 * CUS : 2 * CUS;
    long long splits = N <= FEW_ROWS ? places / tiles : 1;
    if (splits > steps / 8) splits = steps / 8;
    if (splits < 1) splits = 1;
    *per_split = ceil_div(steps, splits) * QBLOCK;
    return ceil_div(steps * QBLOCK, *per_split);
}

static HeadPlan plan(int call, int dtype, int N, int V, int D)
{
    HeadPlan p = {};
    const bool grad = call == SVIP_HEAD_LOSS_GRAD;
    p.parts = in_parts(dtype, call, N, V, D);
    p.planes = p.parts ? 2 : 1;
    p.size = dtype == SVIP_F32 && !p.parts ? 4 : 2;
    p.width = p.parts ? up(D, 8) : D;
    p.fine = grad && p.size == 2 && !p.parts && N <= FEW_ROWS;
    const int grad_planes = p.fine ? 3 : p.parts ? 2 : 1;      // (fine: G', high and low parts of the weighted one)
    const double terms = p.parts ? 3.0 : 1.0;
    // pieces: of the softmax in the gradient, of the weight's parts in fp32, of what a launch has the threads for (at most four for a token and 32 rows,
    // whatever the tiles); equal, so that none is a sliver
    long long most = V, threads = MOST_THREADS / (4LL * ceil_div(N, 32)) / MOST_TILE * MOST_TILE;
    if (most > threads) most = threads;
    if (grad) most = (long long)(PIECE_BYTES / ((size_t)N * p.size * grad_planes));
    if (p.parts) most = most < (long long)(PIECE_BYTES / ((size_t)p.width * 4)) ? most : (long long)(PIECE_BYTES / ((size_t)p.width * 4));
    if (most < LEAST_PIECE) most = LEAST_PIECE;
    p.piece = up(ceil_div(V, ceil_div(V, most)), MOST_TILE);
    if (p.piece > up(V, MOST_TILE)) p.piece = up(V, MOST_TILE);
    p.grad_stride = p.piece;
    size_t at = HEAD_HEADER;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    if (call == SVIP_HEAD_LOGITS) {
        p.splits = logits_splits(N, V, D, &p.per_split);
        if (p.splits > 1) p.sum = take((size_t)p.splits * N * up(V, 4) * sizeof(float));
        p.bytes = at;
        return p;
    }
    const int step = STEP_BYTES / p.size;
    const bool few = N <= FEW_ROWS;
    const Kind kind = p.size == 2 ? HALVES : SINGLES;
    const ShapeId first = kind == HALVES ? LARGE : MIDDLE, last = p.parts ? MIDDLE : kind == HALVES ? FEW : NARROW;
    p.logits = N <= FEWER_ROWS ? FEW : few ? SMALL : fastest(kind, first, last, grad || p.parts ? p.piece : V, N, terms * ceil_div(D, step));
    const size_t packed = (size_t)p.planes * N * up(p.width, 8) * p.size;
    // (a loss and its gradient may use one workspace of either's size or more, one after the other: nothing is kept between them)
    p.part = take((size_t)ceil_div(V, tile_rows(p.logits)) * N * sizeof(float2));
    p.target = take((size_t)N * sizeof(float));
    if (p.parts) {
        p.rows = take((size_t)N * sizeof(float));
        p.hidden_parts = take(packed);
        p.weight = take((size_t)2 * p.piece * p.width * 2);
    }
    if (grad) {
        p.weighted = take(packed);
        p.grad = take((size_t)grad_planes * N * p.grad_stride * p.size);
        p.weight_grad = few ? MIDDLE : fastest(kind, first, kind == HALVES ? MIDDLE : FEW, D, p.piece, terms * ceil_div(N, step));
        // The gradient of the hidden states has few tiles and many steps, which are split where that fills the chip better.
        const int steps = p.piece / step;
        double best = 0.0;
        for (int splits = 1; splits <= MOST_SPLITS && (splits == 1 || steps / splits >= 8); ++splits) {
            if (splits > 1 && (size_t)splits * N * p.width * sizeof(float) > SPLIT_BYTES) break;
            for (ShapeId id : {LARGE, MIDDLE}) {
                if (id < (few ? MIDDLE : first)) continue;
                // few rows: tiles of 128 x all rows, whatever the rows' number and type, which wait for the weight's bytes; the sums of the splits are
                // read once more in the end
                const double cost = tiles_cost(few ? HALVES : kind, id, p.width, few ? 1 : N, splits, terms * ceil_div(steps, splits)) + 4.0 * N * p.width * splits / 3e6;
                if (best == 0.0 || cost < best) {
                    best = cost;
                    p.hidden_grad = few ? p.logits : id;
                    p.per_split = ceil_div(steps, splits) * step;
                }
            }
        }
        p.splits = ceil_div(p.piece, p.per_split);
        p.sum = take((size_t)p.splits * N * p.width * sizeof(float));
    }
    if (p.parts || (grad && dtype == SVIP_F16)) p.maxima = take((size_t)2 * MAX_GROUPS * sizeof(int));
    if (grad) {
        const size_t loss = plan(SVIP_HEAD_LOSS, dtype, N, V, D).bytes;          // (one workspace serves both)
        if (at < loss) at = loss;
    }
    p.bytes = at;
    return p;
}

static svip_status check_sizes(int N, int V, int D)
{
    return N <= 0 || N > HEAD_MAX_ROWS || V <= 0 || V > HEAD_MAX_VOCAB || D <= 0 || D > HEAD_MAX_WIDTH ? SVIP_ERR_SHAPE : SVIP_OK;
}
// The join of the hidden states' gradient, four values of a row a thread, has more threads than other launches whose size is N x D.
static svip_status check_grad_sizes(int N, int D)
{
    return (long long)ceil_div(N, JOIN_SLICES) * ceil_div(D, 4 * JOIN_COLUMNS) * (JOIN_COLUMNS * JOIN_SLICES) > MOST_THREADS ? SVIP_ERR_SHAPE : SVIP_OK;
}
static svip_status check_workspace(const void *ws, size_t bytes, size_t need)
{
    return !ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || bytes < need ? SVIP_ERR_WORKSPACE : SVIP_OK;
}

// ---- loss and gradient -----------------------------------------------------------------------------------------------------------------------------

struct LossCall {
    const void *hidden, *weight;
    int dtype, N, V, D;
    long long hidden_stride, weight_stride;
    float temperature;
    const int *targets;
    char *ws;
    hipStream_t st;
};

static svip_status check_loss(const LossCall &c, const void *out, int call, size_t ws_bytes)
{
    if (!c.hidden || !c.weight || !c.targets || !out) return SVIP_ERR_NULL;
    if (!dtype_ok(c.dtype)) return SVIP_ERR_DTYPE;
    if (svip_status s = check_sizes(c.N, c.V, c.D)) return s;
    if (call == SVIP_HEAD_LOSS_GRAD)
        if (svip_status s = check_grad_sizes(c.N, c.D)) return s;
    if (svip_status s = check_matrix(c.hidden, c.dtype, c.D, c.hidden_stride)) return s;
    if (svip_status s = check_matrix(c.weight, c.dtype, c.D, c.weight_stride)) return s;
    if (c.D * size_of(c.dtype) % 16 != 0) return SVIP_ERR_ALIGN;
    if (!(c.temperature > 0.f) || !isfinite(c.temperature)) return SVIP_ERR_PARAM;
    return check_workspace(c.ws, ws_bytes, plan(call, c.dtype, c.N, c.V, c.D).bytes);
}

// Workgroups of k_head_pack; sets the threads to a row.
static long long pack_grid(HeadPackArgs &a)
{
    a.row_threads = 1;
    while (a.row_threads < 256 && a.row_threads * 8 < a.cols_p) a.row_threads *= 2;
    return (long long)ceil_div(a.rows, 256 / a.row_threads) * ceil_div(a.cols_p, 8 * a.row_threads);
}

static HeadScalars *scalars(const LossCall &c) { return reinterpret_cast<HeadScalars *>(c.ws + 256); }

// The scalars that the tiles use, and in fp32 the parts of the hidden states.  weight_grad: the gradient of the weight is asked for.
static bool prepare(const LossCall &c, const HeadPlan &p, const float *grad_loss, float grad_scale, bool weight_grad)
{
    if (!p.parts && !grad_loss) return true;
    HeadScalarsArgs a = {};
    a.sc = scalars(c);
    a.fine = p.fine;
    a.N = c.N;
    a.vocab = c.V;
    a.temperature = c.temperature;
    a.targets = c.targets;
    a.grad_loss = grad_loss;
    a.grad_scale = grad_scale;
    a.flags = reinterpret_cast<unsigned *>(c.ws);
    int *const maxima = reinterpret_cast<int *>(c.ws + p.maxima);
    auto largest = [&](const void *x, long long stride, int rows, const int *targets, int *out, int *groups) {
        *groups = rows < 4 * MAX_GROUPS ? ceil_div(rows, 4) : MAX_GROUPS;
        const HeadMaxArgs m = {x, stride, rows, c.D, targets, grad_loss, c.V, out};
        return c.dtype == SVIP_F16 ? launch(k_head_max<SVIP_F16>, *groups, 256, c.st, m) : launch(k_head_max<SVIP_F32>, *groups, 256, c.st, m);
    };
    if (p.parts) {
        a.weight_max = maxima;
        if (!largest(c.weight, c.weight_stride, c.V, nullptr, maxima, &a.weight_groups)) return false;
    }
    if (weight_grad && (p.parts || c.dtype == SVIP_F16)) {
        a.hidden_max = maxima + MAX_GROUPS;
        if (!largest(c.hidden, c.hidden_stride, c.N, c.targets, maxima + MAX_GROUPS, &a.hidden_groups)) return false;
    }
    if (!launch(k_head_scalars, 1, SCALARS_WG, c.st, a)) return false;
    if (!p.parts) return true;
    HeadPackArgs h = {};
    h.x = c.hidden;
    h.stride = c.hidden_stride;
    h.rows = c.N;
    h.cols = c.D;
    h.cols_p = p.width;
    h.out = c.ws + p.hidden_parts;
    h.plane = (long long)c.N * p.width * 2;
    h.row_inv = reinterpret_cast<float *>(c.ws + p.rows);
    return launch(k_head_pack_rows, ceil_div(c.N, 4), 256, c.st, h);
}

// The arguments of a piece's tiles of logits; fp32: after the piece's parts have been laid out.
static bool piece_args(const LossCall &c, const HeadPlan &p, int v0, int count, HeadArgs *out)
{
    HeadArgs a = {};
    const int size = size_of(c.dtype);
    const char *rows = static_cast<const char *>(c.weight) + (long long)v0 * c.weight_stride * size;
    if (p.parts) {
        HeadPackArgs w = {};
        w.x = rows;
        w.stride = c.weight_stride;
        w.rows = count;
        w.cols = c.D;
        w.cols_p = p.width;
        w.out = c.ws + p.weight;
        w.plane = (long long)p.piece * p.width * 2;
        w.sc = scalars(c);
        if (!launch(k_head_pack<SVIP_F32>, pack_grid(w), 256, c.st, w)) return false;
        a.weight = {w.out, (long long)p.width * 2, w.plane};
        a.hidden = {c.ws + p.hidden_parts, (long long)p.width * 2, (long long)c.N * p.width * 2};
        a.row_inv = reinterpret_cast<const float *>(c.ws + p.rows);
    } else {
        a.weight = {rows, c.weight_stride * size, 0};
        a.hidden = {static_cast<const char *>(c.hidden), c.hidden_stride * size, 0};
    }
    a.N = c.N;
    a.V = count;
    a.D = p.width;
    a.v0 = v0;
    a.sc = scalars(c);
    a.to_log2 = (float)(1.4426950408889634 / (double)c.temperature);
    a.targets = c.targets;
    a.part = reinterpret_cast<float2 *>(c.ws + p.part);
    a.target_logit = reinterpret_cast<float *>(c.ws + p.target);
    a.vocab = c.V;
    a.flags = reinterpret_cast<unsigned *>(c.ws);
    *out = a;
    return true;
}

static bool run_loss(const LossCall &c, const HeadPlan &p, float *loss, float *lse)
{
    if (!prepare(c, p, nullptr, 1.f, false)) return false;
    int records = 0;
    for (int v0 = 0; v0 < c.V; v0 += p.piece) {
        const int count = c.V - v0 < p.piece ? c.V - v0 : p.piece;
        HeadArgs a;
        if (!piece_args(c, p, v0, count, &a)) return false;
        const bool ok = by_product(c.dtype, p.parts, [&](auto type, auto terms, auto) {
            using T = decltype(type);
            constexpr int TERMS = decltype(terms)::value;
            return by_shape<first_shape<T, TERMS>(), last_shape<T, TERMS>()>(p.logits, [&](auto shape) {
                using S = decltype(shape);
                a.tiles = {ceil_div(count, S::BM), ceil_div(c.N, S::BN)};
                records = v0 / S::BM + a.tiles.m;
                return launch(k_head_stats<T, S, TERMS>, (long long)a.tiles.m * a.tiles.n, S::THREADS, c.st, a);
            });
        });
        if (!ok) return false;
    }
    HeadFinishArgs f = {reinterpret_cast<const float2 *>(c.ws + p.part), records, c.N, c.V, reinterpret_cast<const float *>(c.ws + p.target), c.targets,
                        loss, lse, reinterpret_cast<unsigned *>(c.ws)};
    return launch(k_head_finish, ceil_div(c.N, FINISH_ROWS), FINISH_WG, c.st, f);
}

struct GradOut {
    void *hidden, *weight;
    long long hidden_stride, weight_stride;
};

static bool run_grad(const LossCall &c, const HeadPlan &p, const float *lse, const float *grad_loss, const GradOut &out)
{
    const float scale = c.dtype == SVIP_F16 || p.parts ? GRAD_SCALE_F16 : 1.f;
    if (!prepare(c, p, grad_loss, scale, out.weight != nullptr)) return false;
    const int size = size_of(c.dtype);
    const int wide = up(p.width, 8);                       // of the weighted hidden states' rows
    const long long packed_plane = (long long)c.N * wide * p.size, grad_plane = (long long)c.N * p.grad_stride * p.size;
    if (out.weight) {
        HeadPackArgs h = {};
        h.x = c.hidden;
        h.stride = c.hidden_stride;
        h.rows = c.N;
        h.cols = c.D;
        h.cols_p = wide;
        h.whole = p.size == 4;
        h.out = c.ws + p.weighted;
        h.plane = packed_plane;
        h.sc = scalars(c);
        h.targets = c.targets;
        h.grad_loss = grad_loss;
        h.fine = p.fine;
        h.vocab = c.V;
        if (!by_dtype(c.dtype, [&](auto dt) {
                return launch(k_head_pack<decltype(dt)::value>, pack_grid(h), 256, c.st, h);
            }))
            return false;
    }
    for (int v0 = 0; v0 < c.V; v0 += p.piece) {
        const int count = c.V - v0 < p.piece ? c.V - v0 : p.piece;
        HeadArgs a;
        if (!piece_args(c, p, v0, count, &a)) return false;
        a.lse = lse;
        a.grad_loss = grad_loss;
        a.grad = p.fine && !out.hidden ? nullptr : c.ws + p.grad;
        a.weighted = p.fine && out.weight ? c.ws + p.grad + grad_plane : nullptr;
        a.grad_stride = p.grad_stride;
        a.grad_plane = grad_plane;
        a.low_plane = p.parts;
        const Operand grad = {c.ws + p.grad, p.grad_stride * p.size, grad_plane};
        const bool ok = by_product(c.dtype, p.parts, [&](auto type, auto terms, auto dt) {
            using T = decltype(type);
            constexpr int TERMS = decltype(terms)::value, DT = decltype(dt)::value;
            constexpr ShapeId FIRST = first_shape<T, TERMS>(), LAST = last_shape<T, TERMS>();
            // launches a kernel in a shape, `tiles` its tiles along m and n
            const auto softmax = [&](auto shape) {
                using S = decltype(shape);
                a.tiles = {ceil_div(count, S::BM), ceil_div(c.N, S::BN)};
                return launch(k_head_softmax<T, S, TERMS>, (long long)a.tiles.m * a.tiles.n, S::THREADS, c.st, a);
            };
            const auto grad_hidden = [&](auto shape) {
                using S = decltype(shape);
                HeadHiddenArgs g = {};
                g.weight = a.weight;
                g.grad = grad;
                g.N = c.N;
                g.D = p.width;
                g.V = count;
                g.tiles = {ceil_div(p.width, S::BM), ceil_div(c.N, S::BN)};
                g.splits = ceil_div(count, p.per_split);
                g.per_split = p.per_split;
                g.first = v0 == 0;
                g.sum = reinterpret_cast<float *>(c.ws + p.sum);
                return launch(k_head_grad_hidden<T, S, TERMS>, (long long)g.tiles.m * g.tiles.n * g.splits, S::THREADS, c.st, g);
            };
            const auto grad_weight = [&](auto shape) {
                using S = decltype(shape);
                HeadWeightArgs g = {};
                g.hidden = {c.ws + p.weighted, (long long)wide * p.size, packed_plane};
                g.grad = grad;
                if (p.fine) g.grad.base = a.weighted;
                g.N = c.N;
                g.D = c.D;
                g.Dp = p.width;
                g.V = count;
                g.tiles = {ceil_div(p.width, S::BM), ceil_div(count, S::BN)};
                g.sc = scalars(c);
                g.out = static_cast<char *>(out.weight) + (long long)v0 * out.weight_stride * size;
                g.out_stride = out.weight_stride;
                const long long grid = (long long)g.tiles.m * g.tiles.n;
                if constexpr (DT != SVIP_F32 && std::is_same<S, Middle>::value)
                    if (p.fine) return launch(k_head_grad_weight<T, S, 2, DT>, grid, S::THREADS, c.st, g);
                return launch(k_head_grad_weight<T, S, TERMS, DT>, grid, S::THREADS, c.st, g);
            };
            return by_shape<FIRST, LAST>(p.logits, softmax) && (!out.hidden || by_shape<FIRST, LAST == NARROW ? FEW : LAST>(p.hidden_grad, grad_hidden)) &&
                   (!out.weight || by_shape<FIRST, std::is_same<T, F32>::value ? FEW : MIDDLE>(p.weight_grad, grad_weight));
        });
        if (!ok) return false;
    }
    if (!out.hidden) return true;
    const int splits = ceil_div(c.V < p.piece ? c.V : p.piece, p.per_split);           // (of the first piece: those that were written)
    const int slices = splits < JOIN_SLICES ? 1 : JOIN_SLICES;
    HeadHiddenFinishArgs f = {reinterpret_cast<const float *>(c.ws + p.sum), splits, slices, c.N, c.D, p.width, scalars(c), c.targets, grad_loss, c.V, out.hidden,
                              out.hidden_stride};
    return by_dtype(c.dtype, [&](auto dt) {
        return launch(k_head_hidden_finish<decltype(dt)::value>, (long long)ceil_div(c.N, JOIN_SLICES / slices) * ceil_div(c.D, 4 * JOIN_COLUMNS), JOIN_COLUMNS * JOIN_SLICES, c.st, f);
    });
}

}  // namespace svip

// ---- C ABI -------------------------------------------------------------------------------------------------------------------------------------------

using namespace svip;

size_t svip_head_workspace_bytes(int call, int dtype, int N, int V, int D)
{
    if (call < SVIP_HEAD_LOGITS || call > SVIP_HEAD_LOSS_GRAD || !dtype_ok(dtype) || check_sizes(N, V, D)) return 0;
    if (call == SVIP_HEAD_LOSS_GRAD && check_grad_sizes(N, D)) return 0;
    return plan(call, dtype, N, V, D).bytes;
}

svip_status svip_quantize_blocks(const void *x, int dtype, int rows, int cols, long long row_stride, int block_rows, void *q_out,
                                 long long q_stride, void *scale_out, long long scale_stride, void *hip_stream)
{
    if (!x || !q_out || !scale_out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype)) return SVIP_ERR_DTYPE;
    if (rows <= 0 || rows > HEAD_MAX_VOCAB || cols <= 0 || cols > HEAD_MAX_WIDTH || row_stride < cols) return SVIP_ERR_SHAPE;
    const int kb = ceil_div(cols, QBLOCK);
    if (q_stride < (long long)kb * QBLOCK || scale_stride < kb || (long long)rows * kb >= 1LL << 27) return SVIP_ERR_SHAPE;
    // (fp32 in blocks of one row, 32 lanes a block: whole workgroups of 2^27 - 7 and more would be 2^32 threads)
    if (dtype == SVIP_F32 && block_rows == 1 && (long long)rows * kb > (1LL << 27) - QUANT_WG * Stored<SVIP_F32>::VEC / QBLOCK) return SVIP_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(x) % size_of(dtype) != 0 || !aligned16(q_out) || q_stride % 16 != 0) return SVIP_ERR_ALIGN;
    if (block_rows != 1 && block_rows != QBLOCK) return SVIP_ERR_PARAM;
    QuantizeArgs a = {x, row_stride, rows, cols, kb, static_cast<unsigned char *>(q_out), q_stride, static_cast<unsigned char *>(scale_out), scale_stride};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool ok = by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (block_rows == 1) return launch(k_quantize_rows<DT>, ceil_div((long long)rows * kb, QUANT_WG * Stored<DT>::VEC / QBLOCK), QUANT_WG, st, a);
        return launch(k_quantize_blocks<DT>, (long long)ceil_div(rows, QBLOCK) * kb, QUANT_WG, st, a);
    });
    return ok ? SVIP_OK : SVIP_ERR_HIP;
}

svip_status svip_head_logits(const void *hidden_q, const void *hidden_scale, const void *weight_q, const void *weight_scale, int N, int V, int K,
                             long long hidden_stride, long long hidden_scale_stride, long long weight_stride, long long weight_scale_stride,
                             void *logits_out, int dtype, long long row_stride, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!hidden_q || !hidden_scale || !weight_q || !weight_scale || !logits_out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype)) return SVIP_ERR_DTYPE;
    if (svip_status s = check_sizes(N, V, K)) return s;
    if (K % QBLOCK != 0 || hidden_scale_stride < K / QBLOCK || weight_scale_stride < K / QBLOCK || row_stride < V) return SVIP_ERR_SHAPE;
    if (hidden_stride < K || hidden_stride > 2 * HEAD_MAX_STRIDE || weight_stride < K || weight_stride > 2 * HEAD_MAX_STRIDE) return SVIP_ERR_SHAPE;
    if (!aligned16(hidden_q) || !aligned16(weight_q) || !aligned16(logits_out) || hidden_stride % 16 != 0 || weight_stride % 16 != 0 ||
        row_stride * size_of(dtype) % 16 != 0)
        return SVIP_ERR_ALIGN;
    const HeadPlan p = plan(SVIP_HEAD_LOGITS, dtype, N, V, K);
    if (svip_status s = check_workspace(workspace, workspace_bytes, p.bytes)) return s;
    HeadLogitsArgs a = {};
    a.weight = {static_cast<const char *>(weight_q), weight_stride, 0};
    a.hidden = {static_cast<const char *>(hidden_q), hidden_stride, 0};
    a.weight_scale = static_cast<const unsigned char *>(weight_scale);
    a.hidden_scale = static_cast<const unsigned char *>(hidden_scale);
    a.weight_scale_stride = weight_scale_stride;
    a.hidden_scale_stride = hidden_scale_stride;
    a.N = N;
    a.V = V;
    a.K = K;
    a.out = logits_out;
    a.out_stride = row_stride;
    a.per_split = p.per_split;
    a.part = p.splits > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + p.sum) : nullptr;
    a.part_stride = up(V, 4);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool ok = by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto in = [&](auto shape) {
            using S = decltype(shape);
            a.tiles = {ceil_div(V, S::BM), ceil_div(N, S::BN)};
            return launch(k_head_logits<S, DT>, (long long)a.tiles.m * a.tiles.n * p.splits, S::THREADS, st, a);
        };
        if (narrow_logits(N, V)) return in(Narrow{});
        if (N <= FEW_ROWS) return in(Small{});
        if constexpr (DT == SVIP_F32)
            return in(Middle8{});
        else
            return fastest(CODES, LARGE, MIDDLE, V, N, K / QBLOCK) == LARGE ? in(Large{}) : in(Middle{});
    });
    if (!ok) return SVIP_ERR_HIP;
    if (p.splits == 1) return SVIP_OK;
    const HeadLogitsJoinArgs j = {a.part, a.part_stride, p.splits, N, V, logits_out, row_stride};
    const bool joined = by_dtype(dtype, [&](auto dt) { return launch(k_head_logits_join<decltype(dt)::value>, (long long)N * ceil_div(up(V, 4), 1024), 256, st, j); });
    return joined ? SVIP_OK : SVIP_ERR_HIP;
}

svip_status svip_head_loss(const void *hidden, const void *weight, int dtype, int N, int V, int D, long long hidden_stride, long long weight_stride,
                           float temperature, const int *targets, float *loss_out, float *lse_out, void *workspace, size_t workspace_bytes,
                           void *hip_stream)
{
    const LossCall c = {hidden, weight, dtype, N, V, D, hidden_stride, weight_stride, temperature, targets, static_cast<char *>(workspace),
                        static_cast<hipStream_t>(hip_stream)};
    if (!lse_out) return SVIP_ERR_NULL;
    if (svip_status s = check_loss(c, loss_out, SVIP_HEAD_LOSS, workspace_bytes)) return s;
    return run_loss(c, plan(SVIP_HEAD_LOSS, dtype, N, V, D), loss_out, lse_out) ? SVIP_OK : SVIP_ERR_HIP;
}

svip_status svip_head_loss_grad(const void *hidden, const void *weight, int dtype, int N, int V, int D, long long hidden_stride,
                                long long weight_stride, float temperature, const int *targets, const float *lse, const float *grad_loss,
                                void *grad_hidden_out, long long grad_hidden_stride, void *grad_weight_out, long long grad_weight_stride,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const LossCall c = {hidden, weight, dtype, N, V, D, hidden_stride, weight_stride, temperature, targets, static_cast<char *>(workspace),
                        static_cast<hipStream_t>(hip_stream)};
    if (!lse || !grad_loss) return SVIP_ERR_NULL;
    if (svip_status s = check_loss(c, grad_hidden_out ? grad_hidden_out : grad_weight_out, SVIP_HEAD_LOSS_GRAD, workspace_bytes)) return s;
    if (grad_hidden_out)
        if (svip_status s = check_matrix(grad_hidden_out, dtype, D, grad_hidden_stride)) return s;
    if (grad_weight_out)
        if (svip_status s = check_matrix(grad_weight_out, dtype, D, grad_weight_stride)) return s;
    const GradOut out = {grad_hidden_out, grad_weight_out, grad_hidden_stride, grad_weight_stride};
    return run_grad(c, plan(SVIP_HEAD_LOSS_GRAD, dtype, N, V, D), lse, grad_loss, out) ? SVIP_OK : SVIP_ERR_HIP;
}
