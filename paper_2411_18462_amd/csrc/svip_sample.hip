// svip_sample: entry point and workspace (kernels: sample_kernels.h).
#include "sample_kernels.h"

#include "host_calls.h"

namespace svip {

constexpr int SAMPLE_MAX_ROWS = 1 << 20, SAMPLE_MAX_VOCAB = 1 << 22;

constexpr long long MANY_GROUPS = 1024;                  // of tiles, for the border (see k_sample_border)

static int sample_tiles(int V) { return ceil_div(V, SAMPLE_TILE); }
static svip_status check_sample_sizes(int N, int V)
{
    if (N <= 0 || N > SAMPLE_MAX_ROWS || V <= 0 || V > SAMPLE_MAX_VOCAB) return SVIP_ERR_SHAPE;
    return (long long)N * ceil_div(sample_tiles(V), TILES_WAVES) * TILES_WG > MOST_THREADS ? SVIP_ERR_SHAPE : SVIP_OK;
}
}  // namespace svip

using namespace svip;

size_t svip_sample_workspace_bytes(int dtype, int N, int V)
{
    if (!dtype_ok(dtype) || check_sample_sizes(N, V)) return 0;
    return 512 + up256((size_t)N * row_bytes(sample_tiles(V)));          // flag word, rows
}

svip_status svip_sample(const void *logits, int dtype, int N, int V, long long row_stride, const float *temperature, const int *top_k,
                        const float *top_p, const float *min_p, const float *u, int *token_out, float *prob_out, int *kept_out, void *workspace,
                        size_t workspace_bytes, void *hip_stream)
{
    if (!logits || !u || !token_out) return SVIP_ERR_NULL;
    if (!dtype_ok(dtype)) return SVIP_ERR_DTYPE;
    if (svip_status s = check_sample_sizes(N, V)) return s;
    if (row_stride < V) return SVIP_ERR_SHAPE;
    if (!aligned16(logits) || row_stride * size_of(dtype) % 16 != 0) return SVIP_ERR_ALIGN;
    if (svip_status s = check_workspace(workspace, workspace_bytes, svip_sample_workspace_bytes(dtype, N, V))) return s;
    SampleArgs a = {logits, row_stride, V, temperature, top_k, top_p, min_p, u, token_out, prob_out, kept_out, static_cast<unsigned *>(workspace)};
    int log2_v = 0;
    while ((1 << log2_v) < V) ++log2_v;
    a.unit_bits = 62 - log2_v < 51 ? 62 - log2_v : 51;
    a.tiles = sample_tiles(V);
    a.groups = ceil_div(a.tiles, TILES_WAVES);
    a.data = static_cast<char *>(workspace) + 512;
    const bool ok = by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        using X = std::conditional_t<DT == SVIP_F32, float, std::conditional_t<DT == SVIP_BF16, bf16, f16>>;
        const hipStream_t st = static_cast<hipStream_t>(hip_stream);
        const long long grid = (long long)N * a.groups;
        if (!launch(k_sample_tiles<X>, grid, TILES_WG, st, a)) return false;
        if (top_p || min_p) {
            if (grid <= MANY_GROUPS) {
                if (!launch(k_sample_border<X, BORDER_BOTH>, grid, TILES_WG, st, a)) return false;
            } else if (!launch(k_sample_border<X, BORDER_FIND>, N, TILES_WG, st, a) || !launch(k_sample_border<X, BORDER_MARK>, grid, TILES_WG, st, a)) {
                return false;
            }
        }
        return launch(k_sample_rows<X>, N, SAMPLE_WG, st, a);
    });
    return ok ? SVIP_OK : SVIP_ERR_HIP;
}
