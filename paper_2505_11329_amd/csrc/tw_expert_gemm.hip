// The experts' products: the entry points, and which tiles a product's rows are cut into.
#include <algorithm>

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

// The tile shapes and what one 64-deep K step of a tile takes with every compute unit busy (us), of weights stored [N x K] and [K x N];
// `at_once`: workgroups of it on a compute unit.
struct GroupShape {
    int rows, cols_nk, cols_kn, at_once;
    double us_nk, us_kn;
};
static const GroupShape kGroupShapes[] = {
    {32, 32, 32, 2, 0.24, 0.28}, {64, 128, 64, 2, 0.58, 0.28}, {128, 128, 128, 1, 0.53, 0.55}, {192, 128, 128, 1, 0.70, 0.69}, {256, 256, 256, 1, 1.40, 1.45},
};

// The shape of the least estimated time, whatever the rows of each expert, of which the host knows the average only: an expert has
// half a tile more than its rows fill.
static const GroupShape *choose_shape(const GroupGemm &g, int cus)
{
    const double active = static_cast<double>(std::min<int64_t>(g.groups, g.rows)), each = static_cast<double>(g.rows) / active;
    const GroupShape *best = nullptr;
    double least = 0.0;
    for (const GroupShape &s : kGroupShapes) {
        const int cols = g.kn ? s.cols_kn : s.cols_nk;
        const double tiles = active * std::max(1.0, each / s.rows + 0.5) * static_cast<double>((g.N + cols - 1) / cols);
        const double turns = std::max(1.0, tiles / (cus * s.at_once)), steps = static_cast<double>((g.K + 63) / 64);
        const double us = turns * (steps * (g.kn ? s.us_kn : s.us_nk) + 4.0);
        if (!best || us < least) {
            best = &s;
            least = us;
        }
    }
    return best;
}

static tw_status launch_products(const GroupGemm &g, hipStream_t stream)
{
    int cus = 0;
    TW_TRY(current_cu_count(&cus));
    const GroupShape &s = *choose_shape(g, cus);
    const int cols = g.kn ? s.cols_kn : s.cols_nk;
    const int64_t tiles = (g.rows / s.rows + std::min<int64_t>(g.groups, g.rows)) * ((g.N + cols - 1) / cols);
    if (tiles > (1 << 23)) return TW_ERR_UNSUPPORTED;
    return s.rows == 256 ? launch_group_gemm(g, cols, tiles, cus, stream) : launch_group_tile(g, s.rows, tiles, stream);
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
