// What a layer does row by row beside its products: the gated activation and its gradient; norms and position rotation of
// queries and keys, and their gradient.
#include <algorithm>
#include <cmath>

#include "tw_device.h"
#include "tw_internal.h"

namespace tw {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

static constexpr float kLog2e = 1.44269504088896340736f;

// ---- gated activation ----
//
// Bound by memory: three (backward five) pieces of 16 bytes to a thread.

struct GateParams {
    const char *x, *dout;
    char *out;             // out | dx
    const int32_t *limit;
    int64_t first, end;    // rows of the launch
    uint32_t pieces;       // 16-byte pieces of F columns
};

// s = 1 / (1 + exp(-g)): r for g >= 0, a^3 r below, with a the cube root of exp(g). exp2 gives 0 where its result lies below 2^-126: for exp(g)
// from g = -87.4 on, where products with large factors are not 0 before -190; for a from -262 on. With one a to each factor no product
// overflows that the result does not (|g| a^2 < 1), and one that falls below 2^-126 meets no more than 1.1 behind it. (64080 rows of 1024,
// gradient: 102.6 us, 101.6 with one exp(g) for all.)
struct Gate {
    float a, s;   // s a^2 is the gate's
    float rest;   // 1 - s, without the difference
};
__device__ __forceinline__ Gate gate_of(float g)
{
    const float a = __builtin_amdgcn_exp2f(-fabsf(g) * (kLog2e / 3.0f)), e = a * a * a, r = __builtin_amdgcn_rcpf(1.0f + e);
    return g >= 0.0f ? Gate{1.0f, r, e * r} : Gate{a, a * r, r};
}

template <bool STREAMED>
__device__ __forceinline__ void put(char *to, int64_t piece, u32x4 v)
{
    u32x4 *const at = reinterpret_cast<u32x4 *>(to) + piece;
    if constexpr (STREAMED) __builtin_nontemporal_store(v, at);
    else *at = v;
}

template <bool BACKWARD, bool STREAMED>
__global__ __launch_bounds__(256) void gated_silu_kernel(GateParams p)
{
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, in_launch = i / p.pieces, c = i - in_launch * p.pieces;
    const int64_t row = p.first + in_launch;
    if (row >= (p.limit ? min(static_cast<int64_t>(*p.limit), p.end) : p.end)) return;
    const u32x4 *const x = reinterpret_cast<const u32x4 *>(p.x) + row * 2 * p.pieces + c;
    float g[8], u[8];
    const u32x4 vg = __builtin_nontemporal_load(x), vu = __builtin_nontemporal_load(x + p.pieces);
    unpack8(vg, g);
    unpack8(vu, u);
    if constexpr (!BACKWARD) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const Gate t = gate_of(g[k]);
            u[k] = (u[k] * t.a) * (g[k] * t.s) * t.a;
        }
        put<STREAMED>(p.out, row * p.pieces + c, pack8(u));
    } else {
        float d[8];
        unpack8(__builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p.dout) + row * p.pieces + c), d);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const Gate t = gate_of(g[k]);
            const float gs = g[k] * t.s, slope = fmaf(g[k], t.rest, 1.0f) * t.s;
            g[k] = (d[k] * u[k] * t.a) * slope * t.a;
            u[k] = (d[k] * t.a) * gs * t.a;
        }
        put<STREAMED>(p.out, row * 2 * p.pieces + c, pack8(g));
        put<STREAMED>(p.out, row * 2 * p.pieces + p.pieces + c, pack8(u));
    }
}

// ---- norms and rotation ----
//
// A head belongs to a group of up to 16 lanes, each of which has two chunks of V columns of it: of rotated halves the two whose
// columns are pairs, so that nothing but the norm's sums goes from lane to lane. 16384 tokens, 32 / 8 heads of 128 take 60 us, 5.6 TB/s of
// what is read and written, 8101 of 28 / 4 heads 25.5, where the activation's gradient has 6.4: a wave has one round of loads under way,
// between the position's and the angles', and its stores behind them. (The angles come from the caches
// for each head: two, four and eight heads of a token to a group, with their loads under way together, are 3 to 15 % slower.)

// Queries or keys.
struct RopeSide {
    const char *in, *dy;
    char *out;
    int64_t in_stride, dy_stride, out_stride;  // bytes
    const char *weight;
    int heads;
    int first, grid;  // workgroups of the launch
};

struct RopeParams {
    RopeSide side[2];
    const void *positions;
    const float *rotation;
    float *part;                 // gradient: each workgroup's sums, [grid x dim]
    int tokens;
    int64_t n_positions;
    int position_bytes, dim, rot;
    int lanes_log2;
    float eps, inv_dim;
};

template <int V>
struct Piece;
template <>
struct Piece<8> {
    using T = u32x4;
};
template <>
struct Piece<4> {
    using T = u32x2_t;
};

__device__ __forceinline__ void unpack(const u32x4 &v, float (&f)[8]) { unpack8(v, f); }
__device__ __forceinline__ void unpack(const u32x2_t &v, float (&f)[4])
{
    f[0] = bf16_lo(v.x);
    f[1] = bf16_hi(v.x);
    f[2] = bf16_lo(v.y);
    f[3] = bf16_hi(v.y);
}
__device__ __forceinline__ u32x4 pack(const float (&f)[8]) { return pack8(f); }
__device__ __forceinline__ u32x2_t pack(const float (&f)[4]) { return u32x2_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])}; }

// A lane's two chunks of a head, and whether their columns are rotated.
struct Columns {
    int c[2];       // first column
    bool has[2], turned[2];
};
template <int V, bool NEXT>
__device__ __forceinline__ Columns lane_columns(const RopeParams &p, int j)
{
    const int n = p.dim / V;
    Columns l;
    if constexpr (NEXT) {
        const int half = (n + 1) / 2;
        l.c[0] = j * V;
        l.c[1] = (j + half) * V;
        l.has[0] = j < half;
        l.has[1] = l.has[0] && j + half < n;
        l.turned[0] = l.c[0] < p.rot;
        l.turned[1] = l.c[1] < p.rot;
    } else {
        const int pairs = p.rot / 2 / V, rest = 2 * pairs + 2 * (j - pairs);
        const bool paired = j < pairs;
        l.c[0] = (paired ? j : rest) * V;
        l.c[1] = (paired ? j + pairs : rest + 1) * V;
        l.has[0] = l.c[0] < p.dim;
        l.has[1] = l.c[1] < p.dim;
        l.turned[0] = l.turned[1] = paired;
    }
    return l;
}

// cos and sin of a lane's pairs: V of them where its chunks are halves, V / 2 to each chunk where pairs are neighbours.
template <int V, bool NEXT>
__device__ __forceinline__ void load_angles(const RopeParams &p, const Columns &l, int64_t position, float (&cs)[V], float (&sn)[V])
{
    const float *const row = p.rotation + position * p.rot;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = NEXT ? l.c[h] / 2 : l.c[0] + h * (V / 2);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            cs[h * (V / 2) + i] = 1.0f;
            sn[h * (V / 2) + i] = 0.0f;
        }
        if (l.turned[h])
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                cs[h * (V / 2) + i] = row[at + i];
                sn[h * (V / 2) + i] = row[p.rot / 2 + at + i];
            }
    }
}

template <int V, bool NEXT, bool BACK>
__device__ __forceinline__ void turn(const Columns &l, const float (&cs)[V], const float (&sn)[V], float (&x)[2][V])
{
    if constexpr (!NEXT) {
        if (!l.turned[0]) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float s = BACK ? -sn[i] : sn[i], a = x[0][i], b = x[1][i];
            x[0][i] = a * cs[i] - b * s;
            x[1][i] = b * cs[i] + a * s;
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!l.turned[h]) continue;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float c = cs[h * (V / 2) + i], s = BACK ? -sn[h * (V / 2) + i] : sn[h * (V / 2) + i], a = x[h][2 * i], b = x[h][2 * i + 1];
                x[h][2 * i] = a * c - b * s;
                x[h][2 * i + 1] = b * c + a * s;
            }
        }
    }
}

// The token's position, -1 for padding.
__device__ __forceinline__ int64_t position_of(const RopeParams &p, int token)
{
    if (!p.positions) return 0;
    const int64_t at = p.position_bytes == 8 ? static_cast<const int64_t *>(p.positions)[token] : static_cast<const int32_t *>(p.positions)[token];
    return at >= 0 && at < p.n_positions ? at : -1;
}

// 1 / sqrt(x), also of numbers so small that the instruction takes them for 0.
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    return __builtin_amdgcn_rsqf(small ? x * 0x1p60f : x) * (small ? 0x1p30f : 1.0f);
}

// NEXT: pairs are neighbours (interleaved), not halves. STREAMED: results of more than half of what the last-level cache holds are
// written past it.
template <int V, bool NEXT, bool NORM, bool STREAMED>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeParams p)
{
    using P = typename Piece<V>::T;
    const RopeSide &s = p.side[static_cast<int>(blockIdx.x) >= p.side[1].first];
    const int j = threadIdx.x & ((1 << p.lanes_log2) - 1);
    const uint32_t item = ((blockIdx.x - s.first) * 256u + threadIdx.x) >> p.lanes_log2, heads = s.heads;
    const int token = static_cast<int>(item / heads), head = static_cast<int>(item - token * heads);
    if (token >= p.tokens) return;
    const Columns l = lane_columns<V, NEXT>(p, j);
    const char *const in = s.in + token * s.in_stride + head * p.dim * 2;
    char *const out = s.out + token * s.out_stride + head * p.dim * 2;
    P x[2] = {}, w[2] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (l.has[h]) x[h] = __builtin_nontemporal_load(reinterpret_cast<const P *>(in + l.c[h] * 2));
    const int64_t position = position_of(p, token);
    if constexpr (NORM)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (l.has[h]) w[h] = *reinterpret_cast<const P *>(s.weight + l.c[h] * 2);
    if (position < 0) return;
    float cs[V], sn[V], f[2][V];
    if (p.rotation) load_angles<V, NEXT>(p, l, position, cs, sn);
#pragma unroll
    for (int h = 0; h < 2; ++h) unpack(x[h], f[h]);
    if constexpr (NORM) {
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < V; ++i) sum = fmaf(f[h][i], f[h][i], sum);
        const float r = inverse_root(group_sum(sum, p.lanes_log2) * p.inv_dim + p.eps);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float wf[V];
            unpack(w[h], wf);
#pragma unroll
            for (int i = 0; i < V; ++i) f[h][i] = f[h][i] * r * wf[i];
        }
    }
    if (p.rotation) turn<V, NEXT, false>(l, cs, sn, f);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (l.has[h]) {
            P *const to = reinterpret_cast<P *>(out + l.c[h] * 2);
            if constexpr (STREAMED) __builtin_nontemporal_store(pack(f[h]), to);
            else *to = pack(f[h]);
        }
}

// The gradient. The sums over tokens of the weights' gradient stay in registers; the workgroup's groups are added in their order.
// 16384 tokens, 32 / 8 heads of 128: 98 us, 5.1 TB/s, 4.5 us of it the join: with norms 118 registers, four waves to a SIMD, each with one
// head's loads under way (the next head's ahead of this one's work: 101).
template <int V, bool NEXT, bool NORM, bool STREAMED>
__global__ __launch_bounds__(256) void qk_norm_rope_backward_kernel(RopeParams p)
{
    using P = typename Piece<V>::T;
    extern __shared__ float sums[];  // [groups x dim]
    const RopeSide &s = p.side[static_cast<int>(blockIdx.x) >= p.side[1].first];
    const int j = threadIdx.x & ((1 << p.lanes_log2) - 1), groups = 256 >> p.lanes_log2, group = threadIdx.x >> p.lanes_log2;
    const Columns l = lane_columns<V, NEXT>(p, j);
    P w[2] = {};
    float dw[2][V] = {};
    if constexpr (NORM)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (l.has[h]) w[h] = *reinterpret_cast<const P *>(s.weight + l.c[h] * 2);
    const uint32_t heads = s.heads;
    const int64_t items = static_cast<int64_t>(p.tokens) * s.heads, step = static_cast<int64_t>(s.grid) * groups;
    for (int64_t item = static_cast<int64_t>(blockIdx.x - s.first) * groups + group; item < items; item += step) {
        const int token = static_cast<int>(items >> 32 ? item / heads : static_cast<uint32_t>(item) / heads);
        const int head = static_cast<int>(item - static_cast<int64_t>(token) * heads);
        const char *const dy = s.dy + token * s.dy_stride + head * p.dim * 2, *const in = s.in + token * s.in_stride + head * p.dim * 2;
        char *const out = s.out + token * s.out_stride + head * p.dim * 2;
        P d[2] = {}, x[2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (l.has[h]) {
                d[h] = __builtin_nontemporal_load(reinterpret_cast<const P *>(dy + l.c[h] * 2));
                if constexpr (NORM) x[h] = __builtin_nontemporal_load(reinterpret_cast<const P *>(in + l.c[h] * 2));
            }
        const int64_t position = position_of(p, token);
        if (position < 0) continue;
        float cs[V], sn[V], g[2][V];
        if (p.rotation) load_angles<V, NEXT>(p, l, position, cs, sn);
#pragma unroll
        for (int h = 0; h < 2; ++h) unpack(d[h], g[h]);
        if (p.rotation) turn<V, NEXT, true>(l, cs, sn, g);
        if constexpr (NORM) {
            float f[2][V], square = 0.0f, along = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float wf[V];
                unpack(x[h], f[h]);
                unpack(w[h], wf);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    square = fmaf(f[h][i], f[h][i], square);
                    along = fmaf(g[h][i] * wf[i], f[h][i], along);
                }
            }
            const float r = inverse_root(group_sum(square, p.lanes_log2) * p.inv_dim + p.eps);
            const float back = group_sum(along, p.lanes_log2) * p.inv_dim * r * r;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float wf[V];
                unpack(w[h], wf);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dw[h][i] = fmaf(g[h][i] * r, f[h][i], dw[h][i]);
                    g[h][i] = r * (g[h][i] * wf[i] - f[h][i] * back);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (l.has[h]) {
                P *const to = reinterpret_cast<P *>(out + l.c[h] * 2);
                if constexpr (STREAMED) __builtin_nontemporal_store(pack(g[h]), to);
                else *to = pack(g[h]);
            }
    }
    if constexpr (NORM) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (l.has[h])
#pragma unroll
                for (int i = 0; i < V; ++i) sums[group * p.dim + l.c[h] + i] = dw[h][i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.dim; c += 256) {
            float sum = 0.0f;
            for (int g = 0; g < groups; ++g) sum += sums[g * p.dim + c];
            p.part[static_cast<int64_t>(blockIdx.x) * p.dim + c] = sum;
        }
    }
}

// The workgroups' sums of 16 columns, of the queries or the keys: 64 of each column's at a time, then those in order.
__global__ __launch_bounds__(1024) void qk_norm_rope_join_kernel(const float *part, int q_parts, int k_parts, int dim, float *dq_weight,
                                                                  float *dk_weight)
{
    __shared__ float sums[64][16];
    const int in = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + in;
    const float *const from = blockIdx.y ? part + static_cast<int64_t>(q_parts) * dim : part;
    const int parts = blockIdx.y ? k_parts : q_parts;
    float sum = 0.0f;
    if (c < dim)
#pragma unroll 8
        for (int g = row; g < parts; g += 64) sum += from[static_cast<int64_t>(g) * dim + c];
    sums[row][in] = sum;
    __syncthreads();
    if (row != 0 || c >= dim) return;
    for (int g = 1; g < 64; ++g) sum += sums[g][in];
    (blockIdx.y ? dk_weight : dq_weight)[c] = sum;
}

// ---- host ----

static bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

static tw_status gate_sizes(int64_t rows, int64_t F)
{
    if (rows < 0 || F < 1) return TW_ERR_SHAPE;
    return F % 8 != 0 || F > TW_MAX_H || rows > INT32_MAX ? TW_ERR_UNSUPPORTED : TW_OK;
}

static tw_status launch_gate(GateParams p, int64_t rows, int64_t F, bool backward, void *stream)
{
    p.pieces = static_cast<uint32_t>(F / 8);
    const bool streamed = rows * F * (backward ? 4 : 2) > kLastLevelCacheBytes / 2;
    auto *const kernel = backward ? (streamed ? gated_silu_kernel<true, true> : gated_silu_kernel<true, false>)
                                  : (streamed ? gated_silu_kernel<false, true> : gated_silu_kernel<false, false>);
    // a launch has fewer than 2^31 pieces
    const int64_t most = (int64_t(1) << 30) / p.pieces;
    for (; p.first < rows; p.first = p.end) {
        p.end = std::min(p.first + most, rows);
        const int64_t pieces = (p.end - p.first) * p.pieces;
        TW_HIP(launch_kernel(kernel, dim3(static_cast<uint32_t>((pieces + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), p));
    }
    return TW_OK;
}

// Rows of `width` bytes every `stride`: whether any byte belongs to both. Of rows with one stride, columns that are apart are apart.
struct RowSet {
    const void *p;
    int64_t stride, width;
};
static bool rows_overlap(const RowSet &a, const RowSet &b, int64_t rows)
{
    const uint64_t a_bytes = static_cast<uint64_t>((rows - 1) * a.stride + a.width), b_bytes = static_cast<uint64_t>((rows - 1) * b.stride + b.width);
    if (!ranges_overlap(a.p, a_bytes, b.p, b_bytes)) return false;
    if (a.stride != b.stride) return true;
    int64_t ahead = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % a.stride;
    if (ahead < 0) ahead += a.stride;
    return ahead < a.width || ahead + b.width > a.stride;
}

static tw_status rope_sizes(const tw_qk_norm_rope_args &a)
{
    if (a.tokens < 0 || a.q_heads < 1 || a.kv_heads < 1 || a.head_dim < 1 || !(a.eps >= 0.0f) || std::isinf(a.eps)) return TW_ERR_SHAPE;
    if (a.tokens > INT32_MAX || a.q_heads > TW_MAX_HEADS || a.kv_heads > TW_MAX_HEADS || a.head_dim % 8 != 0 || a.head_dim > TW_MAX_HEAD_DIM)
        return TW_ERR_UNSUPPORTED;
    if (a.rotation) {
        if (a.n_positions < 0 || a.rot_dim < 1 || a.rot_dim > a.head_dim) return TW_ERR_SHAPE;
        if (a.n_positions > INT32_MAX || a.rot_dim % 8 != 0 || (a.position_bytes != 4 && a.position_bytes != 8)) return TW_ERR_UNSUPPORTED;
    }
    return TW_OK;
}

static tw_status rope_stride(int64_t stride, int64_t width)
{
    if (stride < width) return TW_ERR_SHAPE;
    return stride % 8 != 0 || stride > TW_MAX_ROW_STRIDE ? TW_ERR_UNSUPPORTED : TW_OK;
}

struct RopeLayout {
    int v, lanes_log2;
    int64_t grid[2];
};
static RopeLayout rope_layout(const tw_qk_norm_rope_args &a, int rot, bool backward)
{
    RopeLayout l;
    l.v = !a.interleaved && rot % 16 != 0 ? 4 : 8;
    const int chunks = a.head_dim / l.v, pairs = a.interleaved ? 0 : rot / 2 / l.v;
    const int lanes = pairs + (chunks - 2 * pairs + 1) / 2;
    l.lanes_log2 = 0;
    while ((1 << l.lanes_log2) < lanes) ++l.lanes_log2;
    const int64_t groups = 256 >> l.lanes_log2;
    l.grid[0] = (a.tokens * a.q_heads + groups - 1) / groups;
    l.grid[1] = (a.tokens * a.kv_heads + groups - 1) / groups;
    if (backward) {
        // as many workgroups as 256 compute units hold, four each, shared out by the heads (16384 tokens, 32 / 8 heads: 98 us, with
        // three each 103, five 111, eight 97; 2000 tokens 20.0, 20.2, 22.3, 22.8)
        const int64_t most = 1024, k = std::max<int64_t>(1, most * a.kv_heads / (a.q_heads + a.kv_heads));
        l.grid[0] = std::min(l.grid[0], std::max<int64_t>(1, most - k));
        l.grid[1] = std::min(l.grid[1], k);
    }
    return l;
}

static RopeLayout rope_layout(const tw_qk_norm_rope_args &a, bool backward) { return rope_layout(a, a.rotation ? a.rot_dim : 0, backward); }

// The sums of the gradient's workgroups.
static int64_t rope_part_bytes(const tw_qk_norm_rope_args &a, const RopeLayout &l)
{
    return a.q_weight ? (l.grid[0] + l.grid[1]) * a.head_dim * 4 : 0;
}

static RopeParams rope_params(const tw_qk_norm_rope_args &a, const RopeLayout &l)
{
    RopeParams p = {};
    const char *const in[2] = {static_cast<const char *>(a.q), static_cast<const char *>(a.k)};
    const int64_t in_stride[2] = {a.q_stride, a.k_stride}, out_stride[2] = {a.q_out_stride, a.k_out_stride};
    void *const out[2] = {a.q_out, a.k_out};
    const void *const weight[2] = {a.q_weight, a.k_weight};
    for (int i = 0; i < 2; ++i) {
        RopeSide &s = p.side[i];
        s.in = in[i];
        s.out = static_cast<char *>(out[i]);
        s.in_stride = in_stride[i] * 2;
        s.out_stride = out_stride[i] * 2;
        s.weight = static_cast<const char *>(weight[i]);
        s.heads = i ? a.kv_heads : a.q_heads;
        s.first = i ? static_cast<int>(l.grid[0]) : 0;
        s.grid = static_cast<int>(l.grid[i]);
    }
    p.positions = a.positions;
    p.rotation = a.rotation;
    p.tokens = static_cast<int>(a.tokens);
    p.n_positions = a.n_positions;
    p.position_bytes = a.position_bytes;
    p.dim = a.head_dim;
    p.rot = a.rotation ? a.rot_dim : 0;
    p.lanes_log2 = l.lanes_log2;
    p.eps = a.eps;
    p.inv_dim = 1.0f / static_cast<float>(a.head_dim);
    return p;
}

static bool rope_streamed(const tw_qk_norm_rope_args &a)
{
    return a.tokens * (a.q_heads + a.kv_heads) * a.head_dim * 2 > kLastLevelCacheBytes / 2;
}

// What both directions ask of the arguments; `read` are the gradients' inputs besides.
static tw_status rope_tensors(const tw_qk_norm_rope_args &a, bool backward)
{
    const bool norm = a.q_weight != nullptr;
    if (norm != (a.k_weight != nullptr) || (a.rotation != nullptr) != (a.positions != nullptr) || (!norm && !a.rotation)) return TW_ERR_NULL;
    const bool reads_x = !backward || norm;
    if (!a.q_out || !a.k_out || (reads_x && (!a.q || !a.k)) || (backward && (!a.dq || !a.dk)) ||
        (backward && norm && (!a.dq_weight || !a.dk_weight)))
        return TW_ERR_NULL;
    const int64_t q_width = int64_t(a.q_heads) * a.head_dim, k_width = int64_t(a.kv_heads) * a.head_dim;
    TW_TRY(rope_stride(a.q_out_stride, q_width));
    TW_TRY(rope_stride(a.k_out_stride, k_width));
    if (reads_x) {
        TW_TRY(rope_stride(a.q_stride, q_width));
        TW_TRY(rope_stride(a.k_stride, k_width));
    }
    if (backward) {
        TW_TRY(rope_stride(a.dq_stride, q_width));
        TW_TRY(rope_stride(a.dk_stride, k_width));
    }
    if (!aligned16(a.q_out) || !aligned16(a.k_out) || (reads_x && (!aligned16(a.q) || !aligned16(a.k))) ||
        (backward && (!aligned16(a.dq) || !aligned16(a.dk))) || !aligned16(a.rotation) || !aligned16(a.q_weight) || !aligned16(a.k_weight) ||
        (a.positions && !aligned_to(a.positions, a.position_bytes)) ||
        (backward && norm && (!aligned_to(a.dq_weight, 4) || !aligned_to(a.dk_weight, 4))))
        return TW_ERR_ALIGN;
    const RowSet out[2] = {{a.q_out, a.q_out_stride * 2, q_width * 2}, {a.k_out, a.k_out_stride * 2, k_width * 2}};
    RowSet read[4];
    int n_read = 0, of[4];
    const auto reads = [&](const void *p, int64_t stride, int which) {
        read[n_read] = {p, stride * 2, out[which].width};
        of[n_read++] = which;
    };
    if (reads_x) {
        reads(a.q, a.q_stride, 0);
        reads(a.k, a.k_stride, 1);
    }
    if (backward) {
        reads(a.dq, a.dq_stride, 0);
        reads(a.dk, a.dk_stride, 1);
    }
    if (rows_overlap(out[0], out[1], a.tokens)) return TW_ERR_ALIAS;
    const struct {
        const void *p;
        uint64_t bytes;
    } flat[] = {{a.positions, static_cast<uint64_t>(a.positions ? a.tokens * a.position_bytes : 0)},
                {a.rotation, static_cast<uint64_t>(a.rotation ? a.n_positions * a.rot_dim * 4 : 0)},
                {a.q_weight, norm ? a.head_dim * 2u : 0u},
                {a.k_weight, norm ? a.head_dim * 2u : 0u},
                {a.dq_weight, backward && norm ? a.head_dim * 4u : 0u},
                {a.dk_weight, backward && norm ? a.head_dim * 4u : 0u}};
    for (int o = 0; o < 2; ++o) {
        for (int i = 0; i < n_read; ++i) {
            const bool in_place = of[i] == o && read[i].p == out[o].p && read[i].stride == out[o].stride;
            if (!in_place && rows_overlap(out[o], read[i], a.tokens)) return TW_ERR_ALIAS;
        }
        for (const auto &f : flat)
            if (ranges_overlap(out[o].p, static_cast<uint64_t>((a.tokens - 1) * out[o].stride + out[o].width), f.p, f.bytes)) return TW_ERR_ALIAS;
    }
    for (int w = 4; w < 6; ++w) {
        for (int i = 0; i < w; ++i)
            if (ranges_overlap(flat[w].p, flat[w].bytes, flat[i].p, flat[i].bytes)) return TW_ERR_ALIAS;
        for (int i = 0; i < n_read; ++i)
            if (ranges_overlap(flat[w].p, flat[w].bytes, read[i].p, static_cast<uint64_t>((a.tokens - 1) * read[i].stride + read[i].width)))
                return TW_ERR_ALIAS;
    }
    return TW_OK;
}

template <bool BACKWARD, int V, bool NEXT, bool NORM, bool STREAMED>
static constexpr auto rope_kernel()
{
    if constexpr (BACKWARD) return qk_norm_rope_backward_kernel<V, NEXT, NORM, STREAMED>;
    else return qk_norm_rope_kernel<V, NEXT, NORM, STREAMED>;
}

template <bool BACKWARD, int V, bool NEXT>
static tw_status launch_rope_t(const tw_qk_norm_rope_args &a, const RopeLayout &l, const RopeParams &p, hipStream_t stream)
{
    static void (*const kernels[])(RopeParams) = {rope_kernel<BACKWARD, V, NEXT, false, false>(), rope_kernel<BACKWARD, V, NEXT, false, true>(),
                                                  rope_kernel<BACKWARD, V, NEXT, true, false>(), rope_kernel<BACKWARD, V, NEXT, true, true>()};
    const bool norm = a.q_weight != nullptr;
    const unsigned lds = BACKWARD && norm ? (256u >> l.lanes_log2) * a.head_dim * 4 : 0;
    TW_HIP(launch_kernel(kernels[norm * 2 + rope_streamed(a)], dim3(static_cast<uint32_t>(l.grid[0] + l.grid[1])), dim3(256), lds, stream, p));
    return TW_OK;
}

template <bool BACKWARD>
static tw_status launch_rope(const tw_qk_norm_rope_args &a, const RopeLayout &l, const RopeParams &p, hipStream_t stream)
{
    if (a.interleaved) return launch_rope_t<BACKWARD, 8, true>(a, l, p, stream);
    return l.v == 8 ? launch_rope_t<BACKWARD, 8, false>(a, l, p, stream) : launch_rope_t<BACKWARD, 4, false>(a, l, p, stream);
}

// The workspace shares nothing with the call's tensors.
static tw_status rope_workspace(const tw_qk_norm_rope_args &a, const void *workspace, uint64_t need)
{
    const int64_t q = int64_t(a.q_heads) * a.head_dim, k = int64_t(a.kv_heads) * a.head_dim;
    const struct {
        const void *p;
        int64_t stride, width;
    } rows[] = {{a.q, a.q_stride, q},       {a.k, a.k_stride, k},   {a.q_out, a.q_out_stride, q}, {a.k_out, a.k_out_stride, k},
                {a.dq, a.dq_stride, q},     {a.dk, a.dk_stride, k}, {a.q_weight, 0, a.head_dim},  {a.k_weight, 0, a.head_dim},
                {a.dq_weight, 0, 2 * a.head_dim}, {a.dk_weight, 0, 2 * a.head_dim}};
    for (const auto &r : rows)
        if (ranges_overlap(workspace, need, r.p, static_cast<uint64_t>((a.tokens - 1) * r.stride + r.width) * 2)) return TW_ERR_ALIAS;
    if (ranges_overlap(workspace, need, a.positions, a.positions ? static_cast<uint64_t>(a.tokens) * a.position_bytes : 0) ||
        ranges_overlap(workspace, need, a.rotation, a.rotation ? static_cast<uint64_t>(a.n_positions) * a.rot_dim * 4 : 0))
        return TW_ERR_ALIAS;
    return TW_OK;
}

static tw_status launch_join(const tw_qk_norm_rope_args &a, const float *part, int q_parts, int k_parts, hipStream_t stream)
{
    TW_HIP(launch_kernel(qk_norm_rope_join_kernel, dim3(static_cast<uint32_t>((a.head_dim + 15) / 16), 2), dim3(1024), 0, stream, part, q_parts,
                         k_parts, a.head_dim, a.dq_weight, a.dk_weight));
    return TW_OK;
}

}  // namespace tw

using namespace tw;

extern "C" {

tw_status tw_gated_silu(const void *x, int64_t rows, int64_t F, const int32_t *limit, void *out, void *stream)
{
    TW_TRY(gate_sizes(rows, F));
    if (rows == 0) return TW_OK;
    if (!x || !out) return TW_ERR_NULL;
    if (!aligned16(x) || !aligned16(out) || !aligned_to(limit, 4)) return TW_ERR_ALIGN;
    const uint64_t half = static_cast<uint64_t>(rows) * F * 2u;
    if (ranges_overlap(out, half, x, 2 * half) || ranges_overlap(out, half, limit, limit ? 4 : 0)) return TW_ERR_ALIAS;
    GateParams p = {};
    p.x = static_cast<const char *>(x);
    p.out = static_cast<char *>(out);
    p.limit = limit;
    return launch_gate(p, rows, F, false, stream);
}

tw_status tw_gated_silu_backward(const void *dout, const void *x, int64_t rows, int64_t F, const int32_t *limit, void *dx, void *stream)
{
    TW_TRY(gate_sizes(rows, F));
    if (rows == 0) return TW_OK;
    if (!dout || !x || !dx) return TW_ERR_NULL;
    if (!aligned16(dout) || !aligned16(x) || !aligned16(dx) || !aligned_to(limit, 4)) return TW_ERR_ALIGN;
    const uint64_t half = static_cast<uint64_t>(rows) * F * 2u;
    if (ranges_overlap(dx, 2 * half, dout, half) || (dx != x && ranges_overlap(dx, 2 * half, x, 2 * half)) ||
        ranges_overlap(dx, 2 * half, limit, limit ? 4 : 0))
        return TW_ERR_ALIAS;
    GateParams p = {};
    p.x = static_cast<const char *>(x);
    p.dout = static_cast<const char *>(dout);
    p.out = static_cast<char *>(dx);
    p.limit = limit;
    return launch_gate(p, rows, F, true, stream);
}

tw_status tw_qk_norm_rope(const tw_qk_norm_rope_args *args, void *stream)
{
    if (!args) return TW_ERR_NULL;
    const tw_qk_norm_rope_args &a = *args;
    TW_TRY(rope_sizes(a));
    if (a.tokens == 0) return TW_OK;
    TW_TRY(rope_tensors(a, false));
    // a launch has at most 2^23 workgroups
    const int64_t most = (int64_t(1) << 22) * (256 >> rope_layout(a, false).lanes_log2) / std::max(a.q_heads, a.kv_heads);
    for (int64_t first = 0; first < a.tokens; first += most) {
        tw_qk_norm_rope_args part = a;
        part.tokens = std::min(most, a.tokens - first);
        part.q = static_cast<const char *>(a.q) + first * a.q_stride * 2;
        part.k = static_cast<const char *>(a.k) + first * a.k_stride * 2;
        part.q_out = static_cast<char *>(a.q_out) + first * a.q_out_stride * 2;
        part.k_out = static_cast<char *>(a.k_out) + first * a.k_out_stride * 2;
        if (a.positions) part.positions = static_cast<const char *>(a.positions) + first * a.position_bytes;
        const RopeLayout l = rope_layout(part, false);
        TW_TRY(launch_rope<false>(part, l, rope_params(part, l), static_cast<hipStream_t>(stream)));
    }
    return TW_OK;
}

int64_t tw_qk_norm_rope_backward_workspace_bytes(const tw_qk_norm_rope_args *args)
{
    if (!args || rope_sizes(*args) != TW_OK) return -1;
    if (args->tokens == 0) return 0;
    // (a rotation never makes the launch smaller: its chunks are of 4 columns or of 8)
    const bool rot = args->rot_dim >= 8 && args->rot_dim % 8 == 0 && args->rot_dim <= args->head_dim;
    return rope_part_bytes(*args, rope_layout(*args, rot ? args->rot_dim : 0, true));
}

tw_status tw_qk_norm_rope_backward(const tw_qk_norm_rope_args *args, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!args) return TW_ERR_NULL;
    const tw_qk_norm_rope_args &a = *args;
    TW_TRY(rope_sizes(a));
    const bool norm = a.q_weight != nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.tokens == 0) {
        if (!norm) return TW_OK;
        if (!a.dq_weight || !a.dk_weight) return TW_ERR_NULL;
        if (!aligned_to(a.dq_weight, 4) || !aligned_to(a.dk_weight, 4)) return TW_ERR_ALIGN;
        if (ranges_overlap(a.dq_weight, a.head_dim * 4u, a.dk_weight, a.head_dim * 4u)) return TW_ERR_ALIAS;
        return launch_join(a, nullptr, 0, 0, s);
    }
    TW_TRY(rope_tensors(a, true));
    const RopeLayout l = rope_layout(a, true);
    const int64_t need = rope_part_bytes(a, l);
    if (need > 0 && !workspace) return TW_ERR_NULL;
    if (workspace_bytes < need) return TW_ERR_SHAPE;
    if (need > 0 && !aligned16(workspace)) return TW_ERR_ALIGN;
    TW_TRY(rope_workspace(a, workspace, static_cast<uint64_t>(need)));
    RopeParams p = rope_params(a, l);
    p.side[0].dy = static_cast<const char *>(a.dq);
    p.side[1].dy = static_cast<const char *>(a.dk);
    p.side[0].dy_stride = a.dq_stride * 2;
    p.side[1].dy_stride = a.dk_stride * 2;
    p.part = static_cast<float *>(workspace);
    TW_TRY(launch_rope<true>(a, l, p, s));
    return norm ? launch_join(a, p.part, static_cast<int>(l.grid[0]), static_cast<int>(l.grid[1]), s) : TW_OK;
}

}  // extern "C"
