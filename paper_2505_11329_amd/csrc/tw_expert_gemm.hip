// The experts' products: the entry points, and which tiles a product's rows are cut into.
#include <algorithm>
#include <cmath>

#include "tw_internal.h"
#include "tw_mfma.h"

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
// rate at which the weights come in (TB/s) and what passes until they do (us). Fitted to 3000 products of 1 to 32768 rows, 8 to 160 experts, N and K of 256 to
// 8192, with every shape timed: the choice is 2.4 % off the best of them on average, 2.7 % for [K x N]. (The best without 16 x 32 is 4.3 and 3.4 % slower on average, without 16 x 64 5.0
// and 3.5, 32 x 128 1.5 and 3.4, 128 x 128 1.0 and 0.9, 192 x 128 0.5 and 0.7, 256 x 256 0.8 and 0.4; 64 x 128, 64 x 64 and 32 x 32 besides gain less than 0.5 % each.)
struct GroupShape {
    int rows, cols;
    struct {
        double step, fuller, tile, uneven, rate, start;
    } us[2];
};
static const GroupShape kGroupShapes[] = {
    {16, 32, {{0.079, 0.16, 2.87, 0.65, 6.56, 2.52}, {0.126, 0.25, 2.34, 0.76, 5.14, 2.67}}},
    {16, 64, {{0.186, 0.00, 1.06, 0.48, 9.00, 4.17}, {0.247, 0.00, 0.93, 0.94, 7.49, 4.23}}},
    {32, 128, {{0.410, 0.00, 1.09, 0.45, 7.70, 4.81}, {0.441, 0.00, 0.67, 0.52, 9.00, 5.01}}},
    {128, 128, {{0.422, 0.31, 4.35, 0.50, 7.47, 3.37}, {0.488, 0.18, 4.15, 0.27, 7.77, 4.60}}},
    {192, 128, {{0.527, 0.47, 4.30, 0.20, 6.17, 5.73}, {0.564, 0.21, 4.83, 0.52, 6.02, 2.43}}},
    {256, 256, {{1.080, 0.25, 6.87, 0.92, 4.83, 8.67}, {1.190, 0.32, 6.92, 0.81, 5.05, 13.70}}},
};

// As many tiles as there may be: every expert has one more than its rows fill, at most.
static int64_t most_tiles(const GroupGemm &g, const GroupShape &s)
{
    return (g.rows / s.rows + std::min<int64_t>(g.groups, g.rows)) * ((g.N + s.cols - 1) / s.cols);
}
// Of a workgroup each but for the largest, whose workgroups stay.
static bool launches(const GroupGemm &g, const GroupShape &s) { return most_tiles(g, s) <= (s.rows == 256 ? 1 << 30 : 1 << 22); }

// The shape of the least estimated time: of its tiles' and of the weights' the longer, nearly. The host knows only how many rows there are: they
// meet as many experts as choices at random do, and an expert has the tiles of a number of rows that is spread like waiting times, 1 / (1 - exp(-tile / mean)).
static const GroupShape *choose_shape(const GroupGemm &g, int cus)
{
    const double rows = static_cast<double>(g.rows), experts = -std::expm1(-rows / g.groups) * g.groups, each = rows / experts;
    const double weights = experts * static_cast<double>(g.N) * static_cast<double>(g.K) * 2e-6;  // MB
    const GroupShape *best = nullptr;
    double least = 0.0;
    for (const GroupShape &s : kGroupShapes) {
        if (!launches(g, s)) continue;
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
    return best;
}

static tw_status plan_products(const GroupGemm &g, int cus, GroupLaunch *l)
{
    const GroupShape *const s = choose_shape(g, cus);
    if (!s) return TW_ERR_UNSUPPORTED;
    const int64_t tiles = most_tiles(g, *s), slots = (tiles + kXcds - 1) / kXcds * kXcds;
    *l = {s->rows, s->cols, tiles, s->rows == 256 ? std::min<int64_t>(slots, cus) : slots};
    return TW_OK;
}

static tw_status launch_products(const GroupGemm &g, hipStream_t stream)
{
    int cus = 0;
    TW_TRY(current_cu_count(&cus));
    GroupLaunch l;
    TW_TRY(plan_products(g, cus, &l));
    return l.tile_rows == 256 ? launch_group_gemm(g, l, cus, stream) : launch_group_tile(g, l, stream);
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

tw_status tw_expert_gemm_plan(int64_t rows, int64_t N, int64_t K, int n_experts, int b_layout, int backward, int cus,
                              tw_expert_gemm_launch *launch)
{
    if (!launch) return TW_ERR_NULL;
    TW_TRY(expert_sizes(rows, N, K, n_experts, b_layout));
    if (cus < 1) return TW_ERR_SHAPE;
    *launch = {};
    if (N == 0 || (backward ? K : rows) == 0) return TW_OK;
    const bool nk = b_layout == TW_B_NK;
    if (!backward) return plan_products({nullptr, nullptr, nullptr, nullptr, rows, N, K, n_experts, !nk}, cus, launch);
    *launch = plan_expert_gradient(rows, nk ? N : K, nk ? K : N, n_experts, cus);
    return TW_OK;
}

}  // extern "C"
