// Tokens to their experts and back: the pairs of tokens and experts sorted by expert, rows copied to the sorted places,
// the weighted sum of a token's rows, and its gradient.
#include <algorithm>

#include "tw_device.h"
#include "tw_internal.h"

namespace tw {

// ---- sort ----
//
// A stable counting sort. A workgroup has a run of consecutive pairs and each of its waves a part of the run; the place of a
// pair is the number of pairs of lower experts, plus those of its expert in earlier runs, in earlier waves of its own, and
// earlier in its wave. Only counts meet between waves, so nothing depends on the order they run in.

// A workgroup's pairs where there is more than one of them, and the fewest pairs for that (128 experts: 131072 pairs in runs of
// 1024, 2048, 4096, 8192 take 11.7, 11.0, 13.1, 16.4 us; 4096 pairs take 7.2 us in one run and 9.9 in two, 8192 pairs 10.9 and 9.8 in four).
static constexpr int kRun = 2048, kManyPairs = 8192;
static constexpr int kMaxRuns = 256;
static constexpr int kFewExperts = 512;  // 16 waves' counts fit 64 KiB

struct SortParams {
    const void *ids;
    int32_t *order, *position, *offsets;
    int32_t *counts;  // [runs x (experts + 1)]
    int64_t pairs;
    int64_t run;      // pairs of a workgroup
    int experts;
};

// A pair's bucket: its expert, or the last one where it has none.
template <typename Id>
__device__ __forceinline__ int bucket_of(const SortParams &p, int64_t pair)
{
    const Id id = static_cast<const Id *>(p.ids)[pair];
    return id >= 0 && id < p.experts ? static_cast<int>(id) : p.experts;
}

template <typename Id>
__global__ __launch_bounds__(1024) void expert_count_kernel(SortParams p)
{
    extern __shared__ int32_t count[];
    for (int e = threadIdx.x; e <= p.experts; e += blockDim.x) count[e] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.run, end = min(begin + p.run, p.pairs);
    for (int64_t i = begin + threadIdx.x; i < end; i += blockDim.x) atomicAdd(&count[bucket_of<Id>(p, i)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= p.experts; e += blockDim.x)
        p.counts[static_cast<int64_t>(blockIdx.x) * (p.experts + 1) + e] = count[e];
}

// Lanes of the wave whose pair has the same bucket as this lane's; `bits` bits tell buckets apart.
__device__ __forceinline__ uint64_t same_bucket(int bucket, int bits, uint64_t active)
{
    uint64_t same = active;
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((bucket >> b) & 1);
        same &= (bucket >> b) & 1 ? set : ~set;
    }
    return same;
}

template <typename Id, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void expert_place_kernel(SortParams p)
{
    constexpr int kThreads = 64 * WAVES;
    const int buckets = p.experts + 1;
    extern __shared__ int32_t start[];             // [waves x buckets]: counts, then each wave's next places
    int32_t *const all = start + WAVES * buckets;  // pairs of a bucket in all runs
    int32_t *const ahead = all + buckets;          // and in the runs before this one
    __shared__ int32_t wave_total[WAVES];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    for (int i = threadIdx.x; i < (WAVES + 2) * buckets; i += kThreads) start[i] = 0;
    __syncthreads();

    const int64_t run_begin = blockIdx.x * p.run, run_end = min(run_begin + p.run, p.pairs);
    const int64_t part = (p.run / 64 + WAVES - 1) / WAVES * 64;
    const int64_t begin = min(run_begin + wave * part, run_end), end = min(begin + part, run_end);
    int32_t *const mine = start + wave * buckets;
    // (integer sums: the order of these atomics does not show)
    for (int64_t i = begin + lane; i < end; i += 64) {
        const int bucket = bucket_of<Id>(p, i);
        atomicAdd(&mine[bucket], 1);
        if (gridDim.x == 1) atomicAdd(&all[bucket], 1);
    }
    if (gridDim.x > 1) {
        // as many columns of runs side by side as there are threads for
        const int columns = max(1, kThreads / buckets), runs = gridDim.x, here = blockIdx.x;
        for (int i = threadIdx.x; i < columns * buckets; i += kThreads) {
            const int e = i % buckets;
            int32_t n_all = 0, n_ahead = 0;
#pragma unroll 8
            for (int r = i / buckets; r < runs; r += columns) {
                const int32_t n = p.counts[static_cast<int64_t>(r) * buckets + e];
                n_all += n;
                n_ahead += r < here ? n : 0;
            }
            atomicAdd(&all[e], n_all);
            atomicAdd(&ahead[e], n_ahead);
        }
    }
    __syncthreads();

    // each thread has a few neighbouring buckets
    const int each = (buckets + kThreads - 1) / kThreads, first = threadIdx.x * each;
    int32_t total = 0;
    for (int e = first; e < min(first + each, buckets); ++e) total += all[e];
    int32_t upto = total;
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) wave_total[wave] = upto;
    __syncthreads();
    int32_t base = upto - total;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) base += w < wave ? wave_total[w] : 0;
    for (int e = first; e < min(first + each, buckets); ++e) {
        if (blockIdx.x == 0) p.offsets[e] = base;
        int32_t at = base + ahead[e], n[WAVES];
        base += all[e];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) n[w] = start[w * buckets + e];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            start[w * buckets + e] = at;
            at += n[w];
        }
    }
    __syncthreads();

    const int bits = 32 - __builtin_clz(p.experts);
    for (int64_t i0 = begin; i0 < end; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool has = i < end;
        const int bucket = has ? bucket_of<Id>(p, i) : 0;
        const uint64_t same = same_bucket(bucket, bits, __ballot(has));
        if (has) {
            const int before = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
            const int32_t place = mine[bucket] + before;
            // all lanes of the wave have read before one adds, and it has before the next round reads
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (before == 0) mine[bucket] = place + __builtin_popcountll(same);
            p.order[place] = static_cast<int32_t>(i);
            p.position[i] = bucket == p.experts ? -1 : place;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ---- rows ----
//
// All of these are bound by memory: 16 bytes of a row to a thread, 2^row_log2 threads to a row of up to 2048 elements. Longer rows
// are cut into parts of 2048 for workgroups of their own (16 tokens of 8 rows of 7168 summed: 4.1 us, 8.6 by one workgroup each, 5.4
// by two; 16384 of 2 rows of 8192: 133, 143), but for the backward pass, whose dot products need whole rows.

struct RowsParams {
    const char *in;       // x | y | dout
    const char *y;        // backward
    char *out;            // dispatched rows | sums | dy
    const int32_t *position;
    const float *weights;
    float *dweights;
    int64_t tokens, rows;
    int64_t first;        // token of the launch
    int top_k, pieces;    // 16-byte pieces of a row
    int row_log2;
};

static constexpr int kMost = 8;  // most pairs of a token that are worked on at a time

// Experts' rows are read once and not kept in the caches (the gradient of a dispatch, 2531 tokens of 8 rows of 5120: 50 us with
// ordinary loads, 46 so). Results of more than half of what the last-level cache holds are not kept either (STREAMED; 8101 tokens
// to 6 places of 4096: 93 us with ordinary stores, 76 so); smaller ones stay for the products that read them next.
template <bool ONCE>
__device__ __forceinline__ u32x4 row_piece(const char *base, int64_t row, int pieces, int c)
{
    const u32x4 *const from = reinterpret_cast<const u32x4 *>(base + (row * pieces + c) * 16);
    return ONCE ? __builtin_nontemporal_load(from) : *from;
}
template <bool STREAMED>
__device__ __forceinline__ void put_piece(char *base, int64_t row, int pieces, int c, u32x4 v)
{
    u32x4 *const to = reinterpret_cast<u32x4 *>(base + (row * pieces + c) * 16);
    if constexpr (STREAMED) __builtin_nontemporal_store(v, to);
    else *to = v;
}

// The places of pairs [k0, k0 + N) of a token, -1 for none.
template <int N>
__device__ __forceinline__ void places(const RowsParams &p, int64_t token, int k0, int32_t (&at)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        at[k] = -1;
        if (k0 + k < p.top_k) {
            const int32_t s = p.position[token * p.top_k + k0 + k];
            if (s >= 0 && s < p.rows) at[k] = s;
        }
    }
}

// Their weights, those of pairs without a place among them, so that nothing waits for the places.
template <int N>
__device__ __forceinline__ void weights(const RowsParams &p, int64_t token, int k0, float (&w)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = k0 + k < p.top_k ? p.weights[token * p.top_k + k0 + k] : 0.0f;
}

// This thread's piece of its row, and the token that the row is of.
__device__ __forceinline__ int row_part(const RowsParams &p)
{
    return (blockIdx.y << p.row_log2) + (threadIdx.x & ((1 << p.row_log2) - 1));
}
__device__ __forceinline__ int64_t row_token(const RowsParams &p)
{
    return p.first + static_cast<int64_t>(blockIdx.x) * (256 >> p.row_log2) + (threadIdx.x >> p.row_log2);
}

template <bool STREAMED>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(RowsParams p)
{
    const int c = row_part(p);
    const int64_t token = row_token(p);
    if (token >= p.tokens || c >= p.pieces) return;
    const u32x4 x = row_piece<false>(p.in, token, p.pieces, c);
    for (int k0 = 0; k0 < p.top_k; k0 += kMost) {
        int32_t at[kMost];
        places(p, token, k0, at);
#pragma unroll
        for (int k = 0; k < kMost; ++k)
            if (at[k] >= 0) put_piece<STREAMED>(p.out, at[k], p.pieces, c, x);
    }
}

template <bool WEIGHTED, bool STREAMED>
__global__ __launch_bounds__(256) void expert_combine_kernel(RowsParams p)
{
    const int c = row_part(p);
    const int64_t token = row_token(p);
    if (token >= p.tokens || c >= p.pieces) return;
    float sum[8] = {};
    for (int k0 = 0; k0 < p.top_k; k0 += kMost) {
        int32_t at[kMost];
        float w[kMost];
        if constexpr (WEIGHTED) weights(p, token, k0, w);
        places(p, token, k0, at);
        u32x4 v[kMost] = {};
#pragma unroll
        for (int k = 0; k < kMost; ++k)
            if (at[k] >= 0) v[k] = row_piece<true>(p.in, at[k], p.pieces, c);
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
            if (at[k] < 0) continue;
            if constexpr (WEIGHTED) {
                float f[8];
                unpack8(v[k], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[k], f[i], sum[i]);
            } else {
                add8(v[k], sum);
            }
        }
    }
    put_piece<STREAMED>(p.out, token, p.pieces, c, pack8(sum));
}

template <bool STREAMED, int PAIRS>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(RowsParams p)
{
    __shared__ float wave_dot[4][PAIRS];
    const int threads = 1 << p.row_log2, in_row = threadIdx.x & (threads - 1);
    const int64_t token = row_token(p);
    const bool has = token < p.tokens;
    for (int k0 = blockIdx.y * PAIRS; k0 < p.top_k; k0 += gridDim.y * PAIRS) {
        int32_t at[PAIRS];
        float w[PAIRS] = {}, dot[PAIRS] = {};
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) at[k] = -1;
        if (has) {
            weights(p, token, k0, w);
            places(p, token, k0, at);
            for (int c = in_row; c < p.pieces; c += threads) {
                float d[8];
                unpack8(row_piece<false>(p.in, token, p.pieces, c), d);
                u32x4 v[PAIRS] = {};
#pragma unroll
                for (int k = 0; k < PAIRS; ++k)
                    if (at[k] >= 0) v[k] = row_piece<true>(p.y, at[k], p.pieces, c);
#pragma unroll
                for (int k = 0; k < PAIRS; ++k) {
                    if (at[k] < 0) continue;
                    float f[8];
                    unpack8(v[k], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dot[k] = fmaf(f[i], d[i], dot[k]);
                        f[i] = w[k] * d[i];
                    }
                    put_piece<STREAMED>(p.out, at[k], p.pieces, c, pack8(f));
                }
            }
        }
        // a row's dot products: over its lanes, then over its waves in order
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) dot[k] = group_sum(dot[k], min(p.row_log2, 6));
        if (p.row_log2 > 6) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < PAIRS; ++k) wave_dot[threadIdx.x >> 6][k] = dot[k];
            __syncthreads();
            const int first = (threadIdx.x >> p.row_log2) << (p.row_log2 - 6);
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) {
                dot[k] = wave_dot[first][k];
                for (int w2 = 1; w2 < threads / 64; ++w2) dot[k] += wave_dot[first + w2][k];
            }
            __syncthreads();
        }
        if (has)
#pragma unroll
            for (int k = 0; k < PAIRS; ++k)
                if (in_row == k && k0 + k < p.top_k) p.dweights[token * p.top_k + k0 + k] = dot[k];
    }
}

// ---- host ----

static tw_status pair_sizes(int64_t N, int top_k)
{
    if (N < 0 || top_k < 1) return TW_ERR_SHAPE;
    if (top_k > TW_MAX_TOP_K || N > INT32_MAX / top_k) return TW_ERR_UNSUPPORTED;
    return TW_OK;
}

static tw_status sort_sizes(int64_t N, int top_k, int n_experts)
{
    TW_TRY(pair_sizes(N, top_k));
    if (n_experts < 1) return TW_ERR_SHAPE;
    return n_experts > TW_MAX_EXPERTS ? TW_ERR_UNSUPPORTED : TW_OK;
}

static int64_t sort_runs(int64_t pairs) { return pairs < kManyPairs ? 1 : std::min<int64_t>(kMaxRuns, pairs / kRun); }

static tw_status row_sizes(int64_t N, int top_k, int64_t H, int64_t rows)
{
    TW_TRY(pair_sizes(N, top_k));
    if (H < 1 || rows < 0) return TW_ERR_SHAPE;
    if (H % 8 != 0 || H > TW_MAX_H || rows > INT32_MAX) return TW_ERR_UNSUPPORTED;
    return TW_OK;
}

static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

static bool streamed(uint64_t result_bytes) { return result_bytes > static_cast<uint64_t>(kLastLevelCacheBytes / 2); }

// What the pairs' rows come to, however many more rows there are.
static uint64_t placed_bytes(const RowsParams &p) { return static_cast<uint64_t>(std::min(p.rows, p.tokens * p.top_k)) * p.pieces * 16u; }

static void row_layout(int64_t H, RowsParams *p)
{
    p->pieces = static_cast<int>(H / 8);
    p->row_log2 = 0;
    while (p->row_log2 < 8 && (1 << p->row_log2) < p->pieces) ++p->row_log2;
    p->row_log2 = std::max(p->row_log2, 3);  // eight threads at least: one to each pair's gradient
}

// Workgroups of a launch: for groups of rows, and `parts` for the parts of each.
static int64_t row_groups(const RowsParams &p) { return (p.tokens + (256 >> p.row_log2) - 1) / (256 >> p.row_log2); }

static tw_status launch_rows(void (*kernel)(RowsParams), const RowsParams &p, int parts, void *stream)
{
    // a launch has fewer than 2^32 threads
    const int64_t most = (int64_t(1) << 23) / parts;
    RowsParams part = p;
    for (int64_t groups = row_groups(p); groups > 0; groups -= most) {
        const dim3 grid(static_cast<uint32_t>(std::min(groups, most)), static_cast<uint32_t>(parts));
        TW_HIP(launch_kernel(kernel, grid, dim3(256), 0, static_cast<hipStream_t>(stream), part));
        part.first += most * (256 >> p.row_log2);
    }
    return TW_OK;
}

// Parts of a row of up to 256 pieces.
static int row_parts(const RowsParams &p) { return (p.pieces + 255) / 256; }

template <typename Id>
static tw_status launch_sort(const SortParams &p, int64_t runs, hipStream_t stream)
{
    const unsigned buckets = static_cast<unsigned>(p.experts + 1);
    if (runs > 1)
        TW_HIP(launch_kernel(expert_count_kernel<Id>, dim3(static_cast<uint32_t>(runs)), dim3(1024), buckets * 4, stream, p));
    if (p.experts <= kFewExperts)
        TW_HIP(launch_kernel(expert_place_kernel<Id, 16>, dim3(static_cast<uint32_t>(runs)), dim3(1024), 18 * buckets * 4, stream, p));
    else
        TW_HIP(launch_kernel(expert_place_kernel<Id, 8>, dim3(static_cast<uint32_t>(runs)), dim3(512), 10 * buckets * 4, stream, p));
    return TW_OK;
}

}  // namespace tw

using namespace tw;

extern "C" {

int64_t tw_expert_sort_workspace_bytes(int64_t N, int top_k, int n_experts)
{
    if (sort_sizes(N, top_k, n_experts) != TW_OK) return -1;
    const int64_t runs = sort_runs(N * top_k);
    return runs == 1 ? 0 : runs * (n_experts + 1) * 4;
}

tw_status tw_expert_sort(const void *expert_ids, int id_bytes, int64_t N, int top_k, int n_experts, int32_t *order,
                         int32_t *position, int32_t *offsets, void *workspace, int64_t workspace_bytes, void *stream)
{
    TW_TRY(sort_sizes(N, top_k, n_experts));
    if (id_bytes != 4 && id_bytes != 8) return TW_ERR_UNSUPPORTED;
    const int64_t pairs = N * top_k, need = tw_expert_sort_workspace_bytes(N, top_k, n_experts);
    if (!offsets || (pairs > 0 && (!expert_ids || !order || !position)) || (need > 0 && !workspace)) return TW_ERR_NULL;
    if (!aligned4(offsets) || !aligned4(order) || !aligned4(position) || (need > 0 && !aligned4(workspace)) ||
        (reinterpret_cast<uintptr_t>(expert_ids) & (id_bytes - 1)))
        return TW_ERR_ALIGN;
    if (workspace_bytes < need) return TW_ERR_SHAPE;
    const uint64_t list = static_cast<uint64_t>(pairs) * 4u;
    const struct {
        const void *p;
        uint64_t bytes;
    } all[] = {{expert_ids, static_cast<uint64_t>(pairs) * id_bytes},
               {order, list},
               {position, list},
               {offsets, (n_experts + 1) * 4u},
               {workspace, static_cast<uint64_t>(need)}};
    for (int i = 1; i < 5; ++i)
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(all[i].p, all[i].bytes, all[j].p, all[j].bytes)) return TW_ERR_ALIAS;
    SortParams p;
    p.ids = expert_ids;
    p.order = order;
    p.position = position;
    p.offsets = offsets;
    p.counts = static_cast<int32_t *>(workspace);
    p.pairs = pairs;
    p.experts = n_experts;
    const int64_t runs = sort_runs(pairs);
    p.run = ((pairs + runs - 1) / runs + 63) / 64 * 64;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return id_bytes == 4 ? launch_sort<int32_t>(p, runs, s) : launch_sort<int64_t>(p, runs, s);
}

tw_status tw_expert_dispatch(const void *x, const int32_t *position, int64_t N, int top_k, int64_t H, void *out,
                             int64_t rows, void *stream)
{
    TW_TRY(row_sizes(N, top_k, H, rows));
    if (N == 0 || rows == 0) return TW_OK;
    if (!x || !position || !out) return TW_ERR_NULL;
    if (!aligned16(x) || !aligned16(out) || !aligned4(position)) return TW_ERR_ALIGN;
    const uint64_t tokens_b = static_cast<uint64_t>(N) * H * 2u, rows_b = static_cast<uint64_t>(rows) * H * 2u;
    const uint64_t pairs_b = static_cast<uint64_t>(N) * top_k * 4u;
    if (ranges_overlap(out, rows_b, x, tokens_b) || ranges_overlap(out, rows_b, position, pairs_b)) return TW_ERR_ALIAS;
    RowsParams p = {};
    p.in = static_cast<const char *>(x);
    p.out = static_cast<char *>(out);
    p.position = position;
    p.tokens = N;
    p.rows = rows;
    p.top_k = top_k;
    row_layout(H, &p);
    return launch_rows(streamed(placed_bytes(p)) ? expert_dispatch_kernel<true> : expert_dispatch_kernel<false>, p, row_parts(p), stream);
}

tw_status tw_expert_combine(const void *y, int64_t rows, const int32_t *position, const float *weights, int64_t N,
                            int top_k, int64_t H, void *out, void *stream)
{
    TW_TRY(row_sizes(N, top_k, H, rows));
    if (N == 0) return TW_OK;
    if ((rows > 0 && !y) || !position || !out) return TW_ERR_NULL;
    if (!aligned16(y) || !aligned16(out) || !aligned4(position) || !aligned4(weights)) return TW_ERR_ALIGN;
    const uint64_t tokens_b = static_cast<uint64_t>(N) * H * 2u, rows_b = static_cast<uint64_t>(rows) * H * 2u;
    const uint64_t pairs_b = static_cast<uint64_t>(N) * top_k * 4u;
    if (ranges_overlap(out, tokens_b, y, rows_b) || ranges_overlap(out, tokens_b, position, pairs_b) ||
        (weights && ranges_overlap(out, tokens_b, weights, pairs_b)))
        return TW_ERR_ALIAS;
    RowsParams p = {};
    p.in = static_cast<const char *>(y);
    p.out = static_cast<char *>(out);
    p.position = position;
    p.weights = weights;
    p.tokens = N;
    p.rows = rows;
    p.top_k = top_k;
    row_layout(H, &p);
    if (streamed(tokens_b))
        return launch_rows(weights ? expert_combine_kernel<true, true> : expert_combine_kernel<false, true>, p, row_parts(p), stream);
    return launch_rows(weights ? expert_combine_kernel<true, false> : expert_combine_kernel<false, false>, p, row_parts(p), stream);
}

tw_status tw_expert_combine_backward(const void *dout, const void *y, int64_t rows, const int32_t *position,
                                     const float *weights, int64_t N, int top_k, int64_t H, void *dy, float *dweights,
                                     void *stream)
{
    TW_TRY(row_sizes(N, top_k, H, rows));
    if (N == 0) return TW_OK;
    if (!dout || (rows > 0 && (!y || !dy)) || !position || !weights || !dweights) return TW_ERR_NULL;
    if (!aligned16(dout) || !aligned16(y) || !aligned16(dy) || !aligned4(position) || !aligned4(weights) || !aligned4(dweights))
        return TW_ERR_ALIGN;
    const uint64_t tokens_b = static_cast<uint64_t>(N) * H * 2u, rows_b = static_cast<uint64_t>(rows) * H * 2u;
    const uint64_t pairs_b = static_cast<uint64_t>(N) * top_k * 4u;
    const struct {
        const void *p;
        uint64_t bytes;
    } read[] = {{dout, tokens_b}, {position, pairs_b}, {weights, pairs_b}};
    for (const auto &r : read)
        if (ranges_overlap(dy, rows_b, r.p, r.bytes) || ranges_overlap(dweights, pairs_b, r.p, r.bytes)) return TW_ERR_ALIAS;
    if (ranges_overlap(dweights, pairs_b, y, rows_b) || ranges_overlap(dweights, pairs_b, dy, rows_b) ||
        (dy != y && ranges_overlap(dy, rows_b, y, rows_b)))
        return TW_ERR_ALIAS;
    RowsParams p = {};
    p.in = static_cast<const char *>(dout);
    p.y = static_cast<const char *>(y);
    p.out = static_cast<char *>(dy);
    p.position = position;
    p.weights = weights;
    p.dweights = dweights;
    p.tokens = N;
    p.rows = rows;
    p.top_k = top_k;
    row_layout(H, &p);
    // Results that stay in the caches: workgroups for one or two of a token's pairs, which all find dout there (64 tokens of 8 rows of
    // 4096: 4.7 us with one, 5.4 with two, 8.3 with eight; 1500 tokens 47, 45, 48; 8192, whose results do not stay, 223, 211, 211).
    if (streamed(placed_bytes(p))) return launch_rows(expert_combine_backward_kernel<true, kMost>, p, 1, stream);
    if (row_groups(p) * top_k <= 4096) return launch_rows(expert_combine_backward_kernel<false, 1>, p, top_k, stream);
    return launch_rows(expert_combine_backward_kernel<false, 2>, p, (top_k + 1) / 2, stream);
}

}  // extern "C"
