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

// The tile shapes: their size, how many workgroups of them a compute unit holds, and for weights stored [N x K] and [K x N] what a 64-deep
// K step of a tile takes with every compute unit busy, what a tile takes besides (us), and how much of a tile an expert has more than its
// rows fill, of which the host knows only the average. Fitted to 8127 products of 1 to 65536 rows, 8 to 128 experts, N and K of 512 to 8192, with
// every shape timed: the choice is 3.0 % off the best of them on average, 2.2 % for [K x N]. Without 32 x 32 it would be 19 % and 13 %, without 64 x 128
// 2.5 and 4.1 %, without 256 x 256 2.7 and 1.8 %, without the other two 0.5 to 1 % each.
struct GroupShape {
    int rows, cols, at_once;
    struct {
        double step, tile, more;
    } us[2];
};
static const GroupShape kGroupShapes[] = {
    {32, 32, 2, {{0.166, 2.0, 0.89}, {0.302, 2.7, 1.0}}},   {64, 128, 2, {{0.843, 4.6, 0.32}, {0.716, 2.1, 0.69}}},
    {128, 128, 1, {{0.554, 4.3, 0.55}, {0.540, 5.9, 0.32}}}, {192, 128, 1, {{0.810, 5.2, 0.38}, {0.794, 3.7, 0.38}}},
    {256, 256, 1, {{1.372, 7.9, 0.54}, {1.566, 5.5, 0.55}}},
};

// The shape of the least estimated time.
static const GroupShape &choose_shape(const GroupGemm &g, int cus)
{
    const double experts = static_cast<double>(std::min<int64_t>(g.groups, g.rows)), each = static_cast<double>(g.rows) / experts;
    const GroupShape *best = nullptr;
    double least = 0.0;
    for (const GroupShape &s : kGroupShapes) {
        const auto &us = s.us[g.kn];
        const double tiles = experts * std::max(1.0, each / s.rows + us.more) * static_cast<double>((g.N + s.cols - 1) / s.cols);
        double turns = std::max(1.0, tiles / (double(cus) * s.at_once));
        if (turns < 4.0) turns = 0.5 * (turns + std::ceil(turns));  // (few turns end in one that is not full)
        const double time = turns * (static_cast<double>((g.K + 63) / 64) * us.step + us.tile);
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
    return s.rows == 256 ? launch_group_gemm(g, tiles, cus, stream) : launch_group_tile(g, s.rows, tiles, stream);
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
