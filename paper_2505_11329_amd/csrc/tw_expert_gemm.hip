// The experts' products: the entry points, and which tiles a product's rows are cut into.
#include <algorithm>
#include <cmath>

#include "tw_internal.h"

namespace tw {

static tw_status expert_sizes(int64_t rows, int64_t N, int64_t K, int n_experts, int b_layout)
{
    if (rows < 0 || N < 0 || K < 0 || n_experts < 1 || (b_layout != TW_B_NK && b_layout != TW_B_KN)) return TW_ERR_SHAPE;
    if (rows > INT32_MAX || N % 8 != 0 || K % 8 != 0 || N > TW_MAX_EXPERT_WIDTH || K > TW_MAX_EXPERT_WIDTH || n_experts > TW_MAX_EXPERTS)
        return TW_ERR_UNSUPPORTED;
    return TW_OK;
}

static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The three tensors of a call: `out` written, the others read.
static tw_status expert_tensors(const void *a, uint64_t a_bytes, const void *b, uint64_t b_bytes, const void *out, uint64_t out_bytes,
                                const int32_t *offsets, int n_experts)
{
    if ((a_bytes && !a) || (b_bytes && !b) || !out || !offsets) return TW_ERR_NULL;
    if (!aligned16(a) || !aligned16(b) || !aligned16(out) || !aligned4(offsets)) return TW_ERR_ALIGN;
    if (ranges_overlap(out, out_bytes, a, a_bytes) || ranges_overlap(out, out_bytes, b, b_bytes) ||
        ranges_overlap(out, out_bytes, offsets, (n_experts + 1) * 4u))
        return TW_ERR_ALIAS;
    return TW_OK;
}

// The tile shapes: their size, and for weights stored [N x K] and [K x N] what a 64-deep K step of an almost empty tile takes with every
// compute unit busy, how much of that more a full one, what a tile takes besides (us), the share of the time that goes by whole turns where tiles are few, the
// rate at which the weights come in (TB/s) and what passes until they do (us). Fitted to 3200 products of 1 to 32768 rows, 8 to 160 experts, N and K of 256 to
// 8192, with every shape timed: the choice is 2.3 % off the best of them on average, 2.6 % for [K x N]. (Without one of the shapes 3 to 7 %; 64 x 128 besides:
// 0.4 % less.)
struct GroupShape {
    int rows, cols;
    struct {
        double step, fuller, tile, uneven, rate, start;
    } us[2];
};
static const GroupShape kGroupShapes[] = {
    {32, 32, {{0.122, 0.04, 1.33, 0.13, 7.07, 3.42}, {0.162, 0.05, 1.09, 0.82, 6.73, 3.74}}},
    {16, 64, {{0.186, 0.00, 1.08, 0.29, 9.00, 4.44}, {0.252, 0.00, 0.94, 1.00, 8.62, 4.39}}},
    {32, 128, {{0.397, 0.00, 1.16, 0.74, 7.78, 5.29}, {0.451, 0.00, 0.82, 0.67, 9.00, 4.61}}},
    {128, 128, {{0.392, 0.47, 4.69, 0.32, 7.59, 5.06}, {0.476, 0.25, 4.57, 0.28, 7.79, 5.54}}},
    {192, 128, {{0.549, 0.39, 4.08, 0.39, 5.78, 3.31}, {0.564, 0.28, 4.92, 0.57, 6.39, 5.45}}},
    {256, 256, {{1.020, 0.28, 9.07, 0.84, 5.43, 10.00}, {1.360, 0.24, 5.80, 0.64, 5.69, 8.86}}},
};

// The shape of the least estimated time: of its tiles' and of the weights' the longer, nearly. The host knows only how many rows there are: they
// meet as many experts as choices at random do, and an expert has the tiles of a number of rows that is spread like waiting times, 1 / (1 - exp(-tile / mean)).
static const GroupShape &choose_shape(const GroupGemm &g, int cus)
{
    const double rows = static_cast<double>(g.rows), experts = -std::expm1(-rows / g.groups) * g.groups, each = rows / experts;
    const double weights = experts * static_cast<double>(g.N) * static_cast<double>(g.K) * 2e-6;  // MB
    const GroupShape *best = nullptr;
    double least = 0.0;
    for (const GroupShape &s : kGroupShapes) {
        const auto &us = s.us[g.kn];
        const double tiles = -experts / std::expm1(-s.rows / each) * static_cast<double>((g.N + s.cols - 1) / s.cols);
        double turns = tiles / cus;
        if (turns < 8.0) turns = (1.0 - us.uneven) * std::max(1.0, turns) + us.uneven * std::ceil(turns);
        const double step = us.step * (1.0 + us.fuller * std::min(1.0, each / s.rows));
        const double tiles_us = turns * (static_cast<double>((g.K + 63) / 64) * step + us.tile), weights_us = weights / us.rate + us.start;
        const double time = std::pow(std::pow(tiles_us, 4.0) + std::pow(weights_us, 4.0), 0.25);
        if (!best || time < least) {
            best = &s;
            least = time;
        }
    }
    return *best;
}

static tw_status launch_products(const GroupGemm &g, hipStream_t stream)
{
    int cus = 0;
    TW_TRY(current_cu_count(&cus));
    const GroupShape &s = choose_shape(g, cus);
    // every expert has one tile more than its rows fill, at most
    const int64_t tiles = (g.rows / s.rows + std::min<int64_t>(g.groups, g.rows)) * ((g.N + s.cols - 1) / s.cols);
    if (tiles > (1 << 23)) return TW_ERR_UNSUPPORTED;
    return s.rows == 256 ? launch_group_gemm(g, tiles, cus, stream) : launch_group_tile(g, s.rows, s.cols, tiles, stream);
}

}  // namespace tw

using namespace tw;

extern "C" {

tw_status tw_expert_gemm(const void *A, const void *B, void *C, const int32_t *offsets, int64_t rows, int64_t N, int64_t K,
                         int n_experts, int b_layout, void *stream)
{
    TW_TRY(expert_sizes(rows, N, K, n_experts, b_layout));
    if (rows == 0 || N == 0) return TW_OK;
    TW_TRY(expert_tensors(A, uint64_t(rows) * K * 2, B, uint64_t(n_experts) * N * K * 2, C, uint64_t(rows) * N * 2, offsets, n_experts));
    return launch_products({A, B, C, offsets, rows, N, K, n_experts, b_layout == TW_B_KN}, static_cast<hipStream_t>(stream));
}

tw_status tw_expert_gemm_backward(const void *A, const void *dC, void *dB, const int32_t *offsets, int64_t rows, int64_t N,
                                  int64_t K, int n_experts, int b_layout, void *stream)
{
    TW_TRY(expert_sizes(rows, N, K, n_experts, b_layout));
    if (N == 0 || K == 0) return TW_OK;
    TW_TRY(expert_tensors(A, uint64_t(rows) * K * 2, dC, uint64_t(rows) * N * 2, dB, uint64_t(n_experts) * N * K * 2, offsets, n_experts));
    const bool nk = b_layout == TW_B_NK;
    return launch_expert_gradient(nk ? dC : A, nk ? A : dC, dB, offsets, rows, nk ? N : K, nk ? K : N, n_experts,
                                  static_cast<hipStream_t>(stream));
}

}  // extern "C"
