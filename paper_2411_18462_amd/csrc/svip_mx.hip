// The head in 4 bits: entry points, shapes and workspaces (kernels: mx_kernels.h, tiles: head_tile.h).
#include "mx_kernels.h"

#include "host_calls.h"

namespace svip {

template <int BITS> struct MxShapes;
template <> struct MxShapes<4> {
    using Large = TileShape<256, 256, 4, 4, 2>;        // one workgroup a CU
    using Middle = TileShape<128, 128, 2, 2, 2>;       // two
    using Few = TileShape<128, 64, 4, 1, 3>;           // up to 64 rows, which wait for the weight's bytes: two
    using Fewer = TileShape<128, 32, 4, 1, 3>;         // up to 32: two
    using Narrow = TileShape<64, 32, 4, 1, 3>;         // and of a small vocabulary: three
};
template <> struct MxShapes<8> {
    using Large = TileShape<256, 128, 2, 2, 2>;        // two
    using Middle = TileShape<128, 128, 2, 2, 3>;
    using Few = TileShape<128, 64, 4, 1, 4>;
    using Fewer = TileShape<128, 32, 4, 1, 4>;
    using Narrow = TileShape<64, 32, 4, 1, 5>;
};

constexpr int MX_UNIT = 512;                           // values: a split of K has a multiple of it: its scales begin on 16 bytes where a row's do
constexpr int MX_FEW_ROWS = 64, MX_FEWER_ROWS = 32, MX_CUS = 256;

struct MxPlan {
    int splits, per_split;
    size_t part, bytes;
};
// Up to 32 rows and fewer tiles of 128 than CUs: tiles of 64 (8 rows of 8 bits, 32000 x 4096: 15.6 us, with tiles of 128 18.8; 50257 x 5120, 32 rows: 44.8
// against 37.9)
static bool mx_narrow(int N, int V) { return N <= MX_FEWER_ROWS && ceil_div(V, 128) < MX_CUS; }
static MxPlan mx_plan(int N, int V, int K)
{
    MxPlan p = {};
    const int units = ceil_div(K, MX_UNIT);
    const long long tiles = N > MX_FEW_ROWS ? (long long)ceil_div(V, 128) * ceil_div(N, 128) : ceil_div(V, mx_narrow(N, V) ? 64 : 128);
    // Splits of K that fill the chip; of more than 64 rows where a quarter of it would have work (8 bits, 512 x 2000 x 4096: 64 tiles, 27 us, in splits 18; 4 bits,
    // 168 x 8481 x 2560: 134 tiles, 13.4 us, in splits 15.2; 100 x 32000 x 4096: 250 tiles, 21 us, in splits 30).
    long long splits = N > MX_FEW_ROWS && tiles > MX_CUS / 2 ? 1 : (mx_narrow(N, V) ? 3 : 2) * MX_CUS / tiles;
    if (splits > units / 2) splits = units / 2;
    if (splits < 1) splits = 1;
    p.per_split = ceil_div(units, splits) * MX_UNIT;
    p.splits = ceil_div(K, p.per_split);
    p.part = 512;
    p.bytes = p.part + (p.splits > 1 ? up256((size_t)p.splits * N * up(V, 4) * sizeof(float)) : 0);
    return p;
}
size_t mx_logits_workspace(int N, int V, int K) { return mx_plan(N, V, K).bytes; }

// rows of 4-bit codes and their scales
static svip_status check_mx(const void *q, long long q_stride, const void *scale, long long scale_stride, int K)
{
    if (q_stride < K / 2 || q_stride > 2 * HEAD_MAX_STRIDE || scale_stride < K / MX_BLOCK || scale_stride > 2 * HEAD_MAX_STRIDE) return SVIP_ERR_SHAPE;
    return aligned16(q) && q_stride % 16 == 0 && reinterpret_cast<uintptr_t>(scale) % 4 == 0 && scale_stride % 4 == 0 ? SVIP_OK : SVIP_ERR_ALIGN;
}

}  // namespace svip

using namespace svip;

svip_status svip_quantize_mx(const void *x, int dtype, int rows, int cols, long long row_stride, void *q_out, long long q_stride,
                              void *scale_out, long long scale_stride, void *hip_stream)
{
    if (!x || !q_out || !scale_out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype)) return SVIP_ERR_DTYPE;
    if (rows <= 0 || rows > HEAD_MAX_VOCAB || cols <= 0 || cols > HEAD_MAX_WIDTH || row_stride < cols) return SVIP_ERR_SHAPE;
    const int runs = ceil_div(cols, MX_RUN);
    if ((long long)rows * runs >= 1LL << 27) return SVIP_ERR_SHAPE;
    // (fp32, 32 lanes a run: whole workgroups of 2^27 - 7 runs and more would be 2^32 threads)
    if (dtype == SVIP_F32 && (long long)rows * runs > (1LL << 27) - MX_WG * Stored<SVIP_F32>::VEC / MX_RUN) return SVIP_ERR_SHAPE;
    if (svip_status s = check_mx(q_out, q_stride, scale_out, scale_stride, runs * MX_RUN)) return s;
    if (reinterpret_cast<uintptr_t>(x) % size_of(dtype) != 0) return SVIP_ERR_ALIGN;
    const MxQuantizeArgs a = {x, row_stride, rows, cols, runs, static_cast<unsigned char *>(q_out), q_stride, static_cast<unsigned char *>(scale_out), scale_stride};
    const bool ok = by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        return launch(k_mx_quantize<DT>, ceil_div((long long)rows * runs, MX_WG * Stored<DT>::VEC / MX_RUN), MX_WG, static_cast<hipStream_t>(hip_stream), a);
    });
    return ok ? SVIP_OK : SVIP_ERR_HIP;
}

svip_status svip_mx_rows(const void *q, const void *scale, int rows, int cols, long long q_stride, long long scale_stride, const int *ids, int n,
                          void *out, int dtype, long long out_stride, void *hip_stream)
{
    if (!q || !scale || !out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype)) return SVIP_ERR_DTYPE;
    if (rows <= 0 || rows > HEAD_MAX_VOCAB || cols <= 0 || cols > HEAD_MAX_WIDTH || n <= 0 || n > HEAD_MAX_VOCAB || out_stride < cols) return SVIP_ERR_SHAPE;
    if (!ids && n > rows) return SVIP_ERR_SHAPE;
    const int chunks = ceil_div(cols, 8);
    if ((long long)n * chunks > MOST_THREADS - MX_WG) return SVIP_ERR_SHAPE;
    if (svip_status s = check_mx(q, q_stride, scale, scale_stride, up(cols, MX_RUN))) return s;
    if (reinterpret_cast<uintptr_t>(out) % size_of(dtype) != 0) return SVIP_ERR_ALIGN;
    const MxRowsArgs a = {static_cast<const unsigned char *>(q), q_stride, static_cast<const unsigned char *>(scale), scale_stride, rows, cols, chunks, ids, n, out, out_stride};
    const bool ok = by_dtype(dtype, [&](auto dt) {
        return launch(k_mx_rows<decltype(dt)::value>, ceil_div((long long)n * chunks, MX_WG), MX_WG, static_cast<hipStream_t>(hip_stream), a);
    });
    return ok ? SVIP_OK : SVIP_ERR_HIP;
}

svip_status svip_head_logits_mx(const void *hidden_q, const void *hidden_scale, int hidden_bits, const void *weight_q, const void *weight_scale, int N,
                                 int V, int K, long long hidden_stride, long long hidden_scale_stride, long long weight_stride,
                                 long long weight_scale_stride, void *logits_out, int dtype, long long row_stride, void *workspace,
                                 size_t workspace_bytes, void *hip_stream)
{
    if (!hidden_q || !hidden_scale || !weight_q || !weight_scale || !logits_out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype) || (hidden_bits == 8 && dtype == SVIP_F32)) return SVIP_ERR_DTYPE;
    if (hidden_bits != 4 && hidden_bits != 8) return SVIP_ERR_PARAM;
    if (svip_status s = check_sizes(N, V, K)) return s;
    if (K % MX_RUN != 0 || row_stride < V) return SVIP_ERR_SHAPE;
    if (svip_status s = check_mx(weight_q, weight_stride, weight_scale, weight_scale_stride, K)) return s;
    if (hidden_bits == 4) {
        if (svip_status s = check_mx(hidden_q, hidden_stride, hidden_scale, hidden_scale_stride, K)) return s;
    } else {
        if (hidden_stride < K || hidden_stride > 2 * HEAD_MAX_STRIDE || hidden_scale_stride < K / MX_RUN) return SVIP_ERR_SHAPE;
        if (!aligned16(hidden_q) || hidden_stride % 16 != 0) return SVIP_ERR_ALIGN;
    }
    if (!aligned16(logits_out) || row_stride * size_of(dtype) % 16 != 0) return SVIP_ERR_ALIGN;
    const MxPlan p = mx_plan(N, V, K);
    if (svip_status s = check_workspace(workspace, workspace_bytes, p.bytes)) return s;
    MxLogitsArgs a = {};
    a.weight = {static_cast<const char *>(weight_q), weight_stride, 0};
    a.hidden = {static_cast<const char *>(hidden_q), hidden_stride, 0};
    a.weight_scale = {static_cast<const char *>(weight_scale), weight_scale_stride, 0};
    a.hidden_scale = {static_cast<const char *>(hidden_scale), hidden_scale_stride, 0};
    a.N = N;
    a.V = V;
    a.K = K;
    a.out = logits_out;
    a.out_stride = row_stride;
    a.per_split = p.per_split;
    a.part = p.splits > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part) : nullptr;
    a.part_stride = up(V, 4);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const auto with = [&](auto bits, auto dt) {
        constexpr int BITS = decltype(bits)::value, DT = decltype(dt)::value;
        const auto in = [&](auto shape) {
            using S = decltype(shape);
            a.tiles = {ceil_div(V, S::BM), ceil_div(N, S::BN)};
            return launch(k_mx_logits<S, BITS, DT>, (long long)a.tiles.m * a.tiles.n * p.splits, S::THREADS, st, a);
        };
        using Shapes = MxShapes<BITS>;
        if (mx_narrow(N, V)) return in(typename Shapes::Narrow{});
        if (N <= MX_FEWER_ROWS) return in(typename Shapes::Fewer{});
        if (N <= MX_FEW_ROWS) return in(typename Shapes::Few{});
        // rounds over the card, of which one of Large tiles takes 1.75 times as long as one of Middle tiles (4 bits, 128256 x 4096, 192 rows: 94 against 115 us,
        // 65 rows: 89 against 67; 32000 x 4096, 600 rows: 83 against 73; 8 bits, 128256 x 4096, 128 rows: 78 against 92; 32000 x 4096, 100 rows: 38 against 29)
        const auto rounds = [&](auto shape, int places) { return ceil_div((long long)ceil_div(V, decltype(shape)::BM) * ceil_div(N, decltype(shape)::BN), places); };
        const auto large = rounds(typename Shapes::Large{}, (BITS == 4 ? 1 : 2) * MX_CUS), middle = rounds(typename Shapes::Middle{}, 2 * MX_CUS);
        return 7 * large <= 4 * middle ? in(typename Shapes::Large{}) : in(typename Shapes::Middle{});
    };
    constexpr std::integral_constant<int, 4> four{};
    constexpr std::integral_constant<int, 8> eight{};
    const bool ok = by_dtype(dtype, [&](auto dt) {
        if constexpr (decltype(dt)::value == SVIP_F32)
            return with(four, dt);
        else
            return hidden_bits == 4 ? with(four, dt) : with(eight, dt);
    });
    if (!ok) return SVIP_ERR_HIP;
    if (p.splits == 1) return SVIP_OK;
    const MxJoinArgs j = {a.part, a.part_stride, p.splits, N, V, logits_out, row_stride};
    const bool joined = by_dtype(dtype, [&](auto dt) { return launch(k_mx_join<decltype(dt)::value>, (long long)N * ceil_div(up(V, 4), 1024), 256, st, j); });
    return joined ? SVIP_OK : SVIP_ERR_HIP;
}
