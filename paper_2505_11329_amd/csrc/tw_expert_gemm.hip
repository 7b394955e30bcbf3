// The experts' products: C[r] = A[r] B[e] for the rows r of each expert e, and the gradient of B, whose depth is the expert's
// rows. Both are one kernel: tiles of 64 x 64 results, operands staged in the LDS as rows of the depth, whichever way they lie in
// memory.
#include <algorithm>

#include "tw_group.h"
#include "tw_internal.h"
#include "tw_mfma.h"

namespace tw {

struct ExpertParams {
    const char *x, *y;  // x: a row of results (A, or what has the weights' rows); y: a column
    char *out;
    Groups groups;
    int64_t M, N, K;    // of one expert; of products M, of gradients K is the expert's
    int tiles_m, tiles_n;
};

static constexpr int kTile = 64, kDepth = 32, kPitch = kDepth + 8;

// 64 rows of an operand, 32 of its depth, to the LDS. ALONG: the depth lies along the rows in memory; else across them.
template <bool ALONG>
__device__ __forceinline__ void stage(uint16_t *to, const char *from, int64_t row0, int64_t rows, int64_t depth0, int64_t depth,
                                      int64_t pitch)
{
    const int t = threadIdx.x;
    u32x4 v = {0, 0, 0, 0};
    if constexpr (ALONG) {
        const int r = t / 4, c = t % 4 * 8;
        if (row0 + r < rows && depth0 + c < depth) v = *reinterpret_cast<const u32x4 *>(from + ((row0 + r) * pitch + depth0 + c) * 2);
        *reinterpret_cast<u32x4 *>(to + r * kPitch + c) = v;
    } else {
        const int d = t / 8, r = t % 8 * 8;
        if (row0 + r < rows && depth0 + d < depth) v = *reinterpret_cast<const u32x4 *>(from + ((depth0 + d) * pitch + row0 + r) * 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) to[(r + i) * kPitch + d] = static_cast<uint16_t>(v[i / 2] >> (i % 2 * 16));
    }
}

template <bool X_ALONG, bool Y_ALONG, bool GRADIENT>
__global__ __launch_bounds__(256) void expert_simple_kernel(ExpertParams p)
{
    __shared__ uint16_t lx[kTile * kPitch], ly[kTile * kPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, lgrp = lane >> 4;
    const char *x = p.x, *y = p.y;
    char *out = p.out;
    int64_t M = p.M, K = p.K;
    int tm, tn;
    if constexpr (GRADIENT) {
        const int e = blockIdx.x / (p.tiles_m * p.tiles_n), in = blockIdx.x % (p.tiles_m * p.tiles_n);
        int carry = first_group_row(p.groups);
        GroupRows r = {};
        for (int first = 0; first <= e; first += 64) r = group_rows(p.groups, first, lane, &carry);
        const int begin = __builtin_amdgcn_readlane(r.begin, e & 63), end = __builtin_amdgcn_readlane(r.end, e & 63);
        tm = in / p.tiles_n;
        tn = in % p.tiles_n;
        K = end - begin;
        x += int64_t(begin) * p.M * 2;
        y += int64_t(begin) * p.N * 2;
        out += int64_t(e) * p.M * p.N * 2;
    } else {
        const GroupTile t = find_group_tile(p.groups, 6, p.tiles_n, blockIdx.x);
        if (t.group < 0) return;
        tm = t.tile / p.tiles_n;
        tn = t.tile % p.tiles_n;
        M = t.rows;
        x += int64_t(t.begin) * K * 2;
        y += int64_t(t.group) * p.N * K * 2;
        out += int64_t(t.begin) * p.N * 2;
    }
    f32x4 acc[2][2] = {};
    const int wm = wave / 2 * 32, wn = wave % 2 * 32;
    for (int64_t k = 0; k < K; k += kDepth) {
        __syncthreads();
        stage<X_ALONG>(lx, x, int64_t(tm) * kTile, M, k, K, X_ALONG ? K : p.M);
        stage<Y_ALONG>(ly, y, int64_t(tn) * kTile, p.N, k, K, Y_ALONG ? K : p.N);
        __syncthreads();
        bf16x8 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = *reinterpret_cast<const bf16x8 *>(lx + (wm + i * 16 + l15) * kPitch + lgrp * 8);
            b[i] = *reinterpret_cast<const bf16x8 *>(ly + (wn + i * 16 + l15) * kPitch + lgrp * 8);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
    }
    // a lane has four columns of one row of each block
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t m = int64_t(tm) * kTile + wm + i * 16 + l15, n = int64_t(tn) * kTile + wn + j * 16 + lgrp * 4;
            if (m >= M || n >= p.N) continue;
            const u32x2 v = {pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3])};
            *reinterpret_cast<u32x2 *>(out + (m * p.N + n) * 2) = v;
        }
}

// ---- host ----

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

}  // namespace tw

using namespace tw;

extern "C" {

tw_status tw_expert_gemm(const void *A, const void *B, void *C, const int32_t *offsets, int64_t rows, int64_t N, int64_t K,
                         int n_experts, int b_layout, void *stream)
{
    TW_TRY(expert_sizes(rows, N, K, n_experts, b_layout));
    if (rows == 0 || N == 0) return TW_OK;
    TW_TRY(expert_tensors(A, uint64_t(rows) * K * 2, B, uint64_t(n_experts) * N * K * 2, C, uint64_t(rows) * N * 2, offsets, n_experts));
    ExpertParams p = {};
    p.x = static_cast<const char *>(A);
    p.y = static_cast<const char *>(B);
    p.out = static_cast<char *>(C);
    p.groups = {offsets, n_experts, static_cast<int>(rows)};
    p.N = N;
    p.K = K;
    p.tiles_n = static_cast<int>((N + kTile - 1) / kTile);
    const int64_t tiles = (rows / kTile + std::min<int64_t>(n_experts, rows)) * p.tiles_n;
    if (tiles > (1 << 23)) return TW_ERR_UNSUPPORTED;
    TW_HIP(launch_kernel(b_layout == TW_B_NK ? expert_simple_kernel<true, true, false> : expert_simple_kernel<true, false, false>,
                         dim3(static_cast<uint32_t>(tiles)), dim3(256), 0, static_cast<hipStream_t>(stream), p));
    return TW_OK;
}

tw_status tw_expert_gemm_backward(const void *A, const void *dC, void *dB, const int32_t *offsets, int64_t rows, int64_t N,
                                  int64_t K, int n_experts, int b_layout, void *stream)
{
    TW_TRY(expert_sizes(rows, N, K, n_experts, b_layout));
    if (N == 0 || K == 0) return TW_OK;
    TW_TRY(expert_tensors(A, uint64_t(rows) * K * 2, dC, uint64_t(rows) * N * 2, dB, uint64_t(n_experts) * N * K * 2, offsets, n_experts));
    ExpertParams p = {};
    const bool nk = b_layout == TW_B_NK;
    p.x = static_cast<const char *>(nk ? dC : A);
    p.y = static_cast<const char *>(nk ? A : dC);
    p.out = static_cast<char *>(dB);
    p.groups = {offsets, n_experts, static_cast<int>(rows)};
    p.M = nk ? N : K;
    p.N = nk ? K : N;
    p.tiles_m = static_cast<int>((p.M + kTile - 1) / kTile);
    p.tiles_n = static_cast<int>((p.N + kTile - 1) / kTile);
    const int64_t tiles = int64_t(p.tiles_m) * p.tiles_n * n_experts;
    if (tiles > (1 << 23)) return TW_ERR_UNSUPPORTED;
    TW_HIP(launch_kernel(expert_simple_kernel<false, false, true>, dim3(static_cast<uint32_t>(tiles)), dim3(256), 0,
                         static_cast<hipStream_t>(stream), p));
    return TW_OK;
}

}  // extern "C"
