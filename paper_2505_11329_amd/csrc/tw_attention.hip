// Attention of a packed batch: out = softmax(scale * q k^T) v for each sequence, grouped heads, one pass over the keys.
//
// The rows of a sequence's query heads that share a key head are one list: row r of it is query row r / G, head r % G of
// the group (G = q_heads / kv_heads). So a tile of rows reads each key once for all heads of the group, and a single
// decode token still has G rows for the matrix cores.
//
// A wave owns 32 rows, one to a lane and its partner 32 lanes on. It computes S^T = K Q^T, whose column (a lane's 16
// values) belongs to one row: the running maximum and sum of the softmax are one register each, and O^T = V^T P^T is
// rescaled by a factor per lane. P^T needs no exchange between lanes: the order of the keys within a product's depth is
// free, and V's fragments are read in the order that S^T leaves them in (four keys of one column to a lane by the
// transposing LDS read).
//   p = 2^(s c - m), c = scale / ln 2, m the row's maximum of s c; l = sum p; out = (sum p v) / l; lse = (m + log2 l) ln 2
// p is rounded to bf16 for the product with v, as an operand of the matrix cores has to be (relative 2^-8 each, the
// sum over keys is in fp32); l sums the unrounded p in fp32.
#include <algorithm>

#include "tw_internal.h"
#include "tw_mfma.h"

namespace tw {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4_ptr_t;

struct AttentionParams {
    const char *q, *k, *v;
    char *out;
    float *lse;
    const int32_t *q_offsets, *k_offsets;
    float *part;      // partial sums, then their maxima and sums (one chunk of the keys each), where chunks > 1
    float *part_ml;
    int64_t q_rows, k_rows;
    int64_t q_stride, k_stride, v_stride, out_stride;  // bytes
    uint32_t group_magic;  // r / group = r * group_magic >> group_shift
    int group_shift;
    int n_seqs, q_heads, kv_heads, group, dim, causal;
    int chunks, min_chunk;
    float c, inv_c;
};

// The kernels' parts are lambdas: all of them belong into the loop they are called from.
#define TW_INLINE __attribute__((always_inline))

static constexpr float kMinusInf = -__builtin_inff();
static constexpr float kLag = 8.0f;
static constexpr float kLn2 = 0.693147180559945309f;

// The matrix instruction of M x M results, depth 512 / M: operands are 8 values of one row (or column) to a lane, lane l
// holding row l % M and the l / M-th eight of the depth; of the result's column l % M it holds rows
// U (i / 4) + 4 (l / M) + i % 4, U = 256 / M.
template <int M>
struct Mfma;
template <>
struct Mfma<32> {
    using acc = f32x16;
    static __device__ __forceinline__ acc run(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<16> {
    using acc = f32x4;
    static __device__ __forceinline__ acc run(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// Over the lanes of one row, 16 or 32 apart; all of them end with the same bits.
__device__ __forceinline__ float swap_max16(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, static_cast<unsigned>(r[0])), __builtin_bit_cast(float, static_cast<unsigned>(r[1])));
}
__device__ __forceinline__ float swap_max32(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, static_cast<unsigned>(r[0])), __builtin_bit_cast(float, static_cast<unsigned>(r[1])));
}
template <int M>
__device__ __forceinline__ float row_max(float v)
{
    return swap_max32(M == 16 ? swap_max16(v) : v);
}
template <int M>
__device__ __forceinline__ float row_sum(float v)
{
    return swap_add32(M == 16 ? swap_add16(v) : v);
}

// The query row, and the head of the group, of row r of a group's list.
__device__ __forceinline__ int list_pos(const AttentionParams &p, int r)
{
    return static_cast<int>(static_cast<uint64_t>(static_cast<uint32_t>(r)) * p.group_magic >> p.group_shift);
}

// Sequence b's rows, clamped to the tensors whatever the offsets say.
struct Sequence {
    int64_t q0, k0;
    int q_len, k_len;
};
__device__ __forceinline__ int clamp_row(int row, int from, int64_t rows)
{
    return min(max(row, from), static_cast<int>(rows));
}
__device__ __forceinline__ Sequence sequence(const AttentionParams &p, int b)
{
    // (b is the same in all lanes; what is loaded with it is made so for the compiler, too)
    const int q0 = clamp_row(__builtin_amdgcn_readfirstlane(p.q_offsets[b]), 0, p.q_rows);
    const int q1 = clamp_row(__builtin_amdgcn_readfirstlane(p.q_offsets[b + 1]), q0, p.q_rows);
    const int k0 = clamp_row(__builtin_amdgcn_readfirstlane(p.k_offsets[b]), 0, p.k_rows);
    const int k1 = clamp_row(__builtin_amdgcn_readfirstlane(p.k_offsets[b + 1]), k0, p.k_rows);
    return {q0, k0, q1 - q0, k1 - k0};
}

// The keys [begin, end) of chunk c of a sequence.
struct Keys {
    int begin, end;
};
__device__ __forceinline__ Keys chunk_keys(const AttentionParams &p, int k_len, int c)
{
    if (p.chunks == 1) return {0, k_len};
    const int each = max(p.min_chunk, (((k_len + p.chunks - 1) / p.chunks) + 127) & ~127);
    const int64_t b = static_cast<int64_t>(each) * c;
    if (b >= k_len) return {0, 0};
    return {static_cast<int>(b), static_cast<int>(min(b + each, static_cast<int64_t>(k_len)))};
}

// Where piece c of row r of a tile lies: at c XOR the row's swizzle. K's rows are read one piece of each of 16 rows at a
// time, V's by 8-byte halves, 32 or 64 bytes of each of eight rows, four neighbouring ones among them. What is read together
// lies in different LDS banks.
template <int DP>
__device__ __forceinline__ constexpr int k_swizzle(int r)
{
    return DP == 128 ? (r & 15) : ((r >> 1) & 7);
}
template <int DP>
__device__ __forceinline__ constexpr int v_swizzle(int r)
{
    return DP == 128 ? (((r & 3) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1)) : ((((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1));
}

// A bit in each half of a pair that holds Inf or NaN, and the pair with zeros in their place.
__device__ __forceinline__ uint32_t infinite_bf16x2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t finite_bf16x2(uint32_t x)
{
    const uint32_t bad = infinite_bf16x2(x);
    return x & ~((bad - (bad >> 15)) | bad);
}

// One tile's step of the softmax: sc holds a lane's scores, softmax_exp makes them p; m and l are the row's. softmax_max returns the
// factor of what was summed before, 1 for most tiles: the maximum that is taken off follows the row's true one only when that is
// more than 2^8 ahead, so that p stays below 2^8, which changes no relative error, and the sums seldom have to be rescaled. Each
// row decides for itself. (Four chains of maxima and sums: a chain's next instruction waits for eight clocks.)
template <int M, int N>
__device__ __forceinline__ float softmax_max(const typename Mfma<M>::acc (&sc)[N], float c, float *m)
{
    constexpr int kAcc = M * M / 64;
    float tops[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) tops[i] = sc[0][i];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = n == 0 ? 4 : 0; i < kAcc; ++i) tops[i % 4] = fmaxf(tops[i % 4], sc[n][i]);
    const float top = row_max<M>(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))) * c;
    float alpha = 1.0f;
    if (top > *m + kLag) {
        alpha = __builtin_amdgcn_exp2f(*m - top);
        *m = top;
    }
    return alpha;
}

// The maximum that is taken off; 0 while a row has seen no key.
__device__ __forceinline__ float taken_off(float m) { return m == kMinusInf ? 0.0f : m; }

template <int M, int N>
__device__ __forceinline__ void softmax_exp(typename Mfma<M>::acc (&sc)[N], float c, float m, float *l)
{
    constexpr int kAcc = M * M / 64;
    float sums[4] = {*l, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            sc[n][i] = __builtin_amdgcn_exp2f(fmaf(sc[n][i], c, -m));
            sums[i % 4] += sc[n][i];
        }
    *l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// m is a rounded product, and p takes it off the exact one: their difference, half a step of m, must stay small against the range of
// p. Below 2^24 it is 1/2 at most. Above, each score is rounded as m was, and leaves softmax_exp no m to take off. (It is divided by
// c because softmax_exp multiplies; c is no less than 2^-104 there, and the quotient a number.) Rare, and tested where sums are
// rescaled: with a branch of its own 8192 tokens of 32 heads of 64 took 313 us, 311 so, 310 without.
__device__ __forceinline__ bool large_max(float m) { return fabsf(m) >= 0x1p24f; }

template <int M, int N>
__device__ __forceinline__ void take_off_large(typename Mfma<M>::acc (&sc)[N], float c, float inv_c, float *m)
{
#pragma clang fp contract(off)
    const bool large = large_max(*m);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < M * M / 64; ++i) sc[n][i] = large ? (sc[n][i] * c - *m) * inv_c : sc[n][i];
    *m = large ? 0.0f : *m;
}

// Inf and NaN among the values of keys that a row does not see must not meet its p of zero. So in a tile that some row sees only a
// part of, zeros take their place, and what their products would have been is added to the rows that see them: Inf itself,
// as any p > 0 times Inf, and NaN where p has underflowed to 0. So a row gets the same from such a tile as from one that all rows see.

// A bit for each of a lane's p, those that have underflowed.
template <int M, int N>
__device__ __forceinline__ uint32_t underflowed(const typename Mfma<M>::acc (&p)[N])
{
    constexpr int kAcc = M * M / 64;
    uint32_t bits = 0;
#pragma unroll
    for (int i = N * kAcc - 1; i >= 0; --i) {
        bits = bits + bits + (p[i / kAcc][i % kAcc] < 0x1p-126f);
        __builtin_amdgcn_sched_barrier(0);  // (one after the other: registers are scarce here, and time is not)
    }
    return bits;
}

// Adds a key's values that are Inf or NaN, read from memory, to the sums of a lane whose row sees it. The key is the j-th of the
// tile, and lost its row's underflowed().
template <int M, int N>
__device__ __forceinline__ void add_infinite(typename Mfma<M>::acc (&o)[N], const char *values, int dim, int part, bool sees, int j, uint32_t lost)
{
    constexpr int kUnit = 256 / M, kQuads = M * M / 256;
    // the lane that has the key's p, and its number there
    const int lane = threadIdx.x & 63, holder = (lane & (M - 1)) | ((j / 4) % (64 / M) * M);
    const bool none = (__shfl(lost, holder) >> (j / M * (M * M / 64) + j % M / kUnit * 4 + j % 4)) & 1;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int g = 0; g < kQuads; ++g) {
            const int col = b * M + g * kUnit + part * 4;
            u32x2 x = {0, 0};
            if (col < dim) x = *reinterpret_cast<const u32x2 *>(values + col * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t bits = i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16;
                o[b][g * 4 + i] += sees && (bits & 0x7f800000u) == 0x7f800000u ? __uint_as_float(none ? bits | 0x7fc00000u : bits) : 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);  // (one load at a time: registers are scarce here, and time is not)
        }
}

// A row's maximum and sum, by one lane of it, and four of its columns: the result, or a chunk's part of it.
__device__ __forceinline__ void put_row(const AttentionParams &p, int chunk, int64_t at, float m, float l, bool by_this_lane)
{
    if (!by_this_lane) return;
    if (p.chunks > 1) {
        float *const to = p.part_ml + (chunk * p.q_rows * p.q_heads + at) * 2;
        to[0] = m;
        to[1] = l;
    } else if (p.lse) {
        p.lse[at] = l == 0.0f ? kMinusInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}
__device__ __forceinline__ void put4(const AttentionParams &p, int chunk, int64_t row, int head, int col, f32x4 x, float inv)
{
    if (col >= p.dim) return;
    if (p.chunks > 1) {
        const int64_t slot = (chunk * p.q_rows + row) * p.q_heads + head;
        *reinterpret_cast<f32x4 *>(p.part + slot * p.dim + col) = x;
    } else {
        const u32x2 y = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
        *reinterpret_cast<u32x2 *>(p.out + row * p.out_stride + (static_cast<int64_t>(head) * p.dim + col) * 2) = y;
    }
}

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes to a lane from a buffer to LDS address `to` + 16 lane; the caller waits (vmcnt) before anybody reads them.
// STREAMED: not to be kept in the caches.
template <bool STREAMED>
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, uint32_t from, uint32_t scalar_from, uint32_t to)
{
    if constexpr (STREAMED)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                     :
                     : "s"(to), "v"(from), "s"(rsrc), "s"(scalar_from)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :
                     : "s"(to), "v"(from), "s"(rsrc), "s"(scalar_from)
                     : "memory");
}
__device__ __forceinline__ i32x4 buffer_of(const char *p, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return {static_cast<int>(a), static_cast<int>((a >> 32) & 0xffff), static_cast<int>(bytes), 0x00020000};
}

// Sum over this lane and those before it.
__device__ __forceinline__ int sum_upto(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last of each 16 lanes to the next 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to lanes 32 ... 63
    return v;
}

__device__ __forceinline__ int max_upto(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xa, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xc, 0xf, false));
    return v;
}

// The place of a workgroup's tile: its sequence, the tile's number in it.
struct Place {
    Sequence s;
    int tile;
    bool found;
};
// Every wave finds it by itself, 64 sequences at a time, a lane each: the i-th tile of TILE rows. Up to 64 sequences, the
// tiles with the most keys come first, whatever sequence they are of, so that what runs last is short (16 sequences of 8192 tokens,
// 32 / 8 heads: 125 us, 130 in the sequences' order); more of them are taken in their order, each one's last tiles first.
template <int TILE>
__device__ __forceinline__ Place find_place(const AttentionParams &p, int i)
{
    const int lane = threadIdx.x & 63;
    Place at = {};
    for (int b0 = 0; b0 < p.n_seqs; b0 += 64) {
        const int b = min(b0 + lane, p.n_seqs - 1);
        const int qa = p.q_offsets[b], qb = p.q_offsets[b + 1], ka = p.k_offsets[b], kb = p.k_offsets[b + 1];
        const int q0 = clamp_row(qa, 0, p.q_rows), q1 = clamp_row(qb, q0, p.q_rows);
        const int k0 = clamp_row(ka, 0, p.k_rows), k1 = clamp_row(kb, k0, p.k_rows);
        const int n = b0 + lane < p.n_seqs ? ((q1 - q0) * p.group + TILE - 1) / TILE : 0;
        int of = n, upto = sum_upto(n), first = 0;  // tiles of this lane's to choose from, and the first one's number
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (i >= total) {
            i -= total;
            continue;
        }
        if (p.n_seqs > 1 && p.n_seqs <= 64) {
            // A tile's rank counts the tiles' rows that its keys are long: with a causal mask it grows from tile to tile.
            const int64_t keys = p.causal ? max(k1 - k0 - (q1 - q0), 0) : k1 - k0;
            const int rank = static_cast<int>(min(keys * p.group / TILE, int64_t(1) << 24)), step = p.causal ? 1 : 0;
            auto of_rank = [&](int least) TW_INLINE {  // tiles of all sequences of this rank or a higher one
                return __builtin_amdgcn_readlane(sum_upto(step ? min(max(rank + n - least, 0), n) : rank >= least ? n : 0), 63);
            };
            int lo = 0, hi = __builtin_amdgcn_readlane(max_upto(n > 0 ? rank + step * (n - 1) : 0), 63) + 1;
            while (hi - lo > 1) {
                const int mid = lo + (hi - lo) / 2;
                if (of_rank(mid) > i) lo = mid;
                else hi = mid;
            }
            i -= of_rank(lo + 1);
            of = step ? (rank <= lo && lo < rank + n ? 1 : 0) : rank == lo ? n : 0;
            first = step ? lo - rank : 0;
            upto = sum_upto(of);
        }
        const int l = __builtin_ctzll(__ballot(upto > i));
        at.s.q0 = __builtin_amdgcn_readlane(q0, l);
        at.s.k0 = __builtin_amdgcn_readlane(k0, l);
        at.s.q_len = __builtin_amdgcn_readlane(q1, l) - static_cast<int>(at.s.q0);
        at.s.k_len = __builtin_amdgcn_readlane(k1, l) - static_cast<int>(at.s.k0);
        at.tile = __builtin_amdgcn_readlane(first, l) + __builtin_amdgcn_readlane(upto, l) - 1 - i;
        at.found = true;
        return at;
    }
    return at;
}

// Whether the rows are single tokens of the first sequences, one each, and the sequences behind have none: the i-th tile is then
// the i-th sequence's. (Every start is looked at; that the rows are no more than the sequences bounds the last one's.)
__device__ __forceinline__ bool single_tokens(const AttentionParams &p)
{
    const int lane = threadIdx.x & 63, first = clamp_row(p.q_offsets[0], 0, p.q_rows);
    const int rows = clamp_row(p.q_offsets[p.n_seqs], first, p.q_rows) - first;
    bool single = rows <= p.n_seqs;
#pragma unroll 8
    for (int b = lane; b < p.n_seqs; b += 64) single &= clamp_row(p.q_offsets[b], 0, p.q_rows) - first == min(b, rows);
    return __all(single);
}

// Few rows to a sequence, single tokens or a few of each: tiles of 16 or 32 rows of a group's list, whose keys four waves share. Bound
// by what comes from memory. Each wave has keys of its own, 32 at a time, and a place in the LDS for them: the next ones are
// asked for as soon as a product has read the ones before, and nothing but the result ties the waves to each other. Two
// workgroups to a compute unit keep up to 128 KB on their way. Where a tile has all of its sequence's rows its keys are not kept in
// the caches: 48 tokens over 6000 keys, 64 / 8 heads, 107 us, 122 if kept; 4 tokens over 8192 keys 20.9, 22.0.
template <int DP, int RB>
struct FewShape {
    static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16 * RB, kKeys = 32;
    static constexpr int kRowBytes = DP * 2, kTileBytes = kKeys * kRowBytes;
    static constexpr int kPieces = DP / 8, kLoadRows = 64 / kPieces, kLoads = kKeys / kLoadRows;
    static constexpr int kJoinBytes = kWaves * kRows * (DP + 2) * 4;
    static constexpr int kLds = kWaves * 2 * kTileBytes > kJoinBytes ? kWaves * 2 * kTileBytes : kJoinBytes;
};

template <int N>
__device__ __forceinline__ void all_but_landed()  // the N newest loads may be under way
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

template <int DP, int RB>
__global__ __launch_bounds__(256, 2) void attention_few_kernel(AttentionParams p)
{
    using Shape = FewShape<DP, RB>;
    constexpr int kSteps = DP / 32, kBlocks = DP / 16;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, part = lane / 16, row_lane = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int kv_head = blockIdx.x % p.kv_heads;
    const int rest = blockIdx.x / p.kv_heads;
    const int chunk = rest % p.chunks, i = rest / p.chunks;
    Place at = {};
    const Sequence own = sequence(p, min(i, p.n_seqs - 1));
    if (p.group > Shape::kRows || !single_tokens(p)) at = find_place<Shape::kRows>(p, i);
    else if (i < p.n_seqs) at.s = own;
    const Sequence &s = at.s;
    const int list = s.q_len * p.group, r0 = at.tile * Shape::kRows;
    if (r0 >= list) return;  // (no tile is left for this workgroup)
    const Keys keys = chunk_keys(p, s.k_len, chunk);
    const int past = s.k_len - s.q_len;

    // where this lane's 16 bytes of a load come from: the piece that lies in its place of the swizzled tile
    const int load_row = lane / Shape::kPieces, place = lane % Shape::kPieces;
    const char *const k_head = p.k + s.k0 * p.k_stride + static_cast<int64_t>(kv_head) * p.dim * 2;
    const char *const v_head = p.v + s.k0 * p.v_stride + static_cast<int64_t>(kv_head) * p.dim * 2;
    char *const mine = lds + wave * 2 * Shape::kTileBytes;
    const uint32_t k_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char_ptr_t)mine)), v_at = k_at + Shape::kTileBytes;

    // fragments' places
    const int i16 = lane & 15, v_row = 4 * part + (i16 >> 2);
    const char *k_frag[kSteps], *v_frag[kBlocks];
#pragma unroll
    for (int x = 0; x < kSteps; ++x) k_frag[x] = mine + row_lane * Shape::kRowBytes + (((4 * x + part) ^ k_swizzle<DP>(row_lane)) << 4);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
        v_frag[b] = mine + Shape::kTileBytes + v_row * Shape::kRowBytes + (((2 * b + ((i16 & 3) >> 1)) ^ v_swizzle<DP>(v_row)) << 4) + (i16 & 1) * 8;

    const int last_pos = list_pos(p, min(r0 + Shape::kRows, list) - 1);
    const int end = min(keys.end, p.causal ? last_pos + past + 1 : s.k_len);
    const int first_last = min(keys.end - 1, p.causal ? list_pos(p, r0) + past : s.k_len - 1);  // the last key that the first row sees

    const bool alone = list <= Shape::kRows;  // no other tile has a use for these keys
    auto load_rows = [&](const char *base, int64_t stride, int key0, uint32_t to, auto swizzle) TW_INLINE {
        const int rows = min(Shape::kKeys, end - key0);
        const i32x4 rsrc = buffer_of(base + key0 * stride, rows > 0 ? static_cast<uint32_t>((rows - 1) * stride + p.dim * 2) : 0);
        auto load = [&](auto streamed) TW_INLINE {
#pragma unroll
            for (int i = 0; i < Shape::kLoads; ++i) {
                const int col = (place ^ swizzle(i * Shape::kLoadRows + load_row)) * 8;
                load_to_lds<decltype(streamed)::value>(rsrc, col < p.dim ? static_cast<uint32_t>(load_row * stride + col * 2) : kPastTensor,
                                                       static_cast<uint32_t>(i * Shape::kLoadRows * stride), to + i * 1024);
            }
        };
        if (alone) load(std::true_type{});
        else load(std::false_type{});
    };
    auto load_keys = [&](int key0) TW_INLINE { load_rows(k_head, p.k_stride, key0, k_at, [](int row) { return k_swizzle<DP>(row); }); };
    auto load_values = [&](int key0) TW_INLINE { load_rows(v_head, p.v_stride, key0, v_at, [](int row) { return v_swizzle<DP>(row); }); };

    int key0 = keys.begin + wave * Shape::kKeys;
    constexpr int kOn = Shape::kWaves * Shape::kKeys;
    load_keys(key0);
    load_values(key0);
    int last[RB];  // keys [0, last] are visible to this lane's rows
    bf16x8 qf[RB][kSteps];
    f32x4 o[RB][kBlocks] = {};
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = r0 + rb * 16 + row_lane, pos = list_pos(p, r), head = kv_head * p.group + r - pos * p.group;
        last[rb] = r < list ? min(p.causal ? pos + past : s.k_len - 1, keys.end - 1) : -1;
        m[rb] = kMinusInf;
        l[rb] = 0.0f;
#pragma unroll
        for (int x = 0; x < kSteps; ++x) {
            u32x4 q = {0, 0, 0, 0};
            const int col = x * 32 + part * 8;
            if (r < list && col < p.dim)
                q = *reinterpret_cast<const u32x4 *>(p.q + (s.q0 + pos) * p.q_stride + (static_cast<int64_t>(head) * p.dim + col) * 2);
            qf[rb][x] = __builtin_bit_cast(bf16x8, q);
        }
    }
    for (; key0 < end; key0 += kOn) {
        f32x4 sc[RB][2] = {};
        all_but_landed<Shape::kLoads>();
#pragma unroll
        for (int x = 0; x < kSteps; ++x)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(k_frag[x] + n * 16 * Shape::kRowBytes);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) sc[rb][n] = Mfma<16>::run(kf, qf[rb][x], sc[rb][n]);
            }
        lds_read();
        load_keys(key0 + kOn);  // (past the end: no bytes, but as many loads to wait for)
        const bool masked = first_last < key0 + Shape::kKeys - 1;
        if (masked) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int seen = last[rb] - key0 - 4 * part;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n * 16 + i > seen) sc[rb][n][i] = kMinusInf;
            }
        }
        u32x4 pf[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float alpha = softmax_max<16>(sc[rb], p.c, &m[rb]);
            float off = taken_off(m[rb]);
            if (__any(alpha != 1.0f || large_max(off))) {
                l[rb] *= alpha;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[rb][b] *= alpha;
                if (__builtin_expect(__any(large_max(off)), 0)) take_off_large<16>(sc[rb], p.c, p.inv_c, &off);
            }
            softmax_exp<16>(sc[rb], p.c, off, &l[rb]);
            pf[rb] = {pack_bf16x2(sc[rb][0][0], sc[rb][0][1]), pack_bf16x2(sc[rb][0][2], sc[rb][0][3]),
                      pack_bf16x2(sc[rb][1][0], sc[rb][1][1]), pack_bf16x2(sc[rb][1][2], sc[rb][1][3])};
        }
        all_but_landed<Shape::kLoads>();
        if (masked) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < Shape::kLoads; ++i) {
                u32x4 *const x = reinterpret_cast<u32x4 *>(mine + Shape::kTileBytes + i * 1024 + lane * 16);
                u32x4 v = *x;
                uint32_t here = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    here |= infinite_bf16x2(v[w]);
                    v[w] = finite_bf16x2(v[w]);
                }
                if (here) *x = v;
                bad |= here;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (__builtin_expect(__any(bad != 0), 0)) {
                uint32_t lost[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) lost[rb] = underflowed<16>(sc[rb]);
#pragma unroll 1
                for (int j = key0; j < min(key0 + Shape::kKeys, end); ++j)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        add_infinite<16>(o[rb], v_head + j * p.v_stride, p.dim, part, j <= last[rb], j - key0, lost[rb]);
            }
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            u32x4 vf;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const u32x2 x = __builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr_t)(v_frag[b] + e * 16 * Shape::kRowBytes)));
                vf[2 * e] = x[0];
                vf[2 * e + 1] = x[1];
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                o[rb][b] = Mfma<16>::run(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pf[rb]), o[rb][b]);
        }
        lds_read();
        load_values(key0 + kOn);
    }

    // the waves' maxima, sums and sums of v pass through the LDS and are joined in the order of the waves, by sixteen
    // threads to a row
    all_but_landed<0>();
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(lds);
    float *const ml = sums + Shape::kWaves * Shape::kRows * DP;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int slot = wave * Shape::kRows + rb * 16 + row_lane;
        const float sum = row_sum<16>(l[rb]);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) *reinterpret_cast<f32x4 *>(sums + slot * DP + ((b * 4 + part) ^ (row_lane & 7)) * 4) = o[rb][b];
        if (part == 0) {
            ml[slot * 2] = m[rb];
            ml[slot * 2 + 1] = sum;
        }
    }
    __syncthreads();
    constexpr int kFours = DP / 64;  // of a thread's columns
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int jr = rb * 16 + (threadIdx.x >> 4), j16 = threadIdx.x & 15, r = r0 + jr;
        if (r >= list) continue;
        float top = kMinusInf, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < Shape::kWaves; ++w) top = fmaxf(top, ml[(w * Shape::kRows + jr) * 2]);
        const float top_use = top == kMinusInf ? 0.0f : top;
        f32x4 x[kFours] = {};
#pragma unroll
        for (int w = 0; w < Shape::kWaves; ++w) {
            const int from = w * Shape::kRows + jr;
            const float f = __builtin_amdgcn_exp2f(ml[from * 2] - top_use);
            sum += f * ml[from * 2 + 1];
#pragma unroll
            for (int b = 0; b < kFours; ++b)
                x[b] += f * *reinterpret_cast<const f32x4 *>(sums + from * DP + ((b * 16 + j16) ^ (jr & 7)) * 4);
        }
        const int pos = list_pos(p, r), head = kv_head * p.group + r - pos * p.group;
        put_row(p, chunk, (s.q0 + pos) * p.q_heads + head, top, sum, j16 == 0);
        // a row that sees no key has a sum of 0
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        // (a chunk of no keys has no columns to put: the sum of 0 says so)
        if (p.chunks == 1 || keys.begin < keys.end) {
#pragma unroll
            for (int b = 0; b < kFours; ++b) put4(p, chunk, s.q0 + pos, head, (b * 16 + j16) * 4, x[b], inv);
        }
    }
}

// A batch of many rows: 32 rows of a group's list to a wave, and tiles of 64 keys that come straight into the LDS while the
// tile before is worked on.
//
// 128 columns leave room for two waves of a SIMD. Eight that share their keys are faster where there are rows enough (4096 rows of a
// 16384-token prompt, 64 / 8 heads: 1.64 ms; two workgroups of four: 1.79). 64 columns leave room for three workgroups of four
// (8192 tokens, 32 heads: 305 us; two of eight: 322).
template <int DP, int WAVES>
struct WideShape {
    static constexpr int kWaves = WAVES;
    static constexpr int kThreads = 64 * kWaves, kRows = 32 * kWaves, kKeys = 64;
    static constexpr int kRowBytes = DP * 2, kTileBytes = kKeys * kRowBytes;
    static constexpr int kPieces = DP / 8;
    static constexpr int kLoads = kTileBytes / (16 * kThreads);  // of 16 bytes to a lane, for K or V of a tile
    static constexpr int kLoadRows = 64 / kPieces;               // rows of a wave's load
    static constexpr int kStageBytes = 2 * kTileBytes;           // K, V
    // The rows of q pass through the second stage before its first tile comes, or a place of their own if they are too many,
    // and the results through the same place in the end.
    static constexpr int kQBytes = kRows * kRowBytes, kQAt = kQBytes <= kStageBytes ? kStageBytes : 2 * kStageBytes;
    static constexpr int kLds = kQAt + (kQBytes > kStageBytes ? kQBytes : kStageBytes);
};

template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_wide_kernel(AttentionParams p)
{
    using Shape = WideShape<DP, WAVES>;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    // Of 128 columns the keys' fragments are read four products ahead of their use; left to itself the compiler has each product
    // wait for its own (8192 tokens, 16 heads: 270 us, 263 so). 64 columns have a third wave of the SIMD to fill such waits, if
    // its registers are left to it (310 us, 313 with fragments ahead).
    constexpr int kAhead = DP == 128 ? 4 : 0;
    extern __shared__ __align__(16) char lds[];
    __shared__ int flags[2][Shape::kWaves];  // a wave's pieces of the V tile held Inf or NaN; where rows see a part of the tile
    const int lane = threadIdx.x & 63, half = lane >> 5, row_lane = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int kv_head = blockIdx.x % p.kv_heads;
    const int rest = blockIdx.x / p.kv_heads;
    const int chunk = rest % p.chunks;
    const Place at = find_place<Shape::kRows>(p, rest / p.chunks);
    if (!at.found) return;
    const Sequence &s = at.s;
    const int list = s.q_len * p.group;
    const Keys keys = chunk_keys(p, s.k_len, chunk);
    const int past = s.k_len - s.q_len;

    const int r0 = at.tile * Shape::kRows;
    const int last_pos = list_pos(p, min(r0 + Shape::kRows, list) - 1), first_pos = list_pos(p, r0);
    const int end = min(keys.end, p.causal ? last_pos + past + 1 : s.k_len);
    const int first_last = min(keys.end - 1, p.causal ? first_pos + past : s.k_len - 1);  // the last key that the first row sees
    const int visible = end - keys.begin;  // rows past them read as zeros
    const int tiles = visible > 0 ? (visible + Shape::kKeys - 1) / Shape::kKeys : 0;
    const int whole = min(tiles, max(0, first_last + 1 - keys.begin) / Shape::kKeys);  // tiles that every row sees all of

    // where this lane's 16 bytes of a load come from: the piece that lies in its place of the swizzled tile
    const int load_row = wave * Shape::kLoadRows + lane / Shape::kPieces, place = lane % Shape::kPieces;
    const int k_piece_from = place ^ k_swizzle<DP>(load_row), v_piece_from = place ^ v_swizzle<DP>(load_row);
    static_assert((Shape::kWaves * Shape::kLoadRows) % 16 == 0, "a lane's rows have one swizzle");
    const uint32_t k_from = k_piece_from * 8 < p.dim ? static_cast<uint32_t>(load_row * p.k_stride + k_piece_from * 16) : kPastTensor;
    const uint32_t v_from = v_piece_from * 8 < p.dim ? static_cast<uint32_t>(load_row * p.v_stride + v_piece_from * 16) : kPastTensor;
    const char *const k_head = p.k + (s.k0 + keys.begin) * p.k_stride + static_cast<int64_t>(kv_head) * p.dim * 2;
    const char *const v_head = p.v + (s.k0 + keys.begin) * p.v_stride + static_cast<int64_t>(kv_head) * p.dim * 2;
    const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char_ptr_t)lds));
    auto load_tile = [&](int t) TW_INLINE {
        const int rows = min(Shape::kKeys, visible - t * Shape::kKeys);
        const int64_t row0 = static_cast<int64_t>(t) * Shape::kKeys;
        const i32x4 rk = buffer_of(k_head + row0 * p.k_stride, static_cast<uint32_t>((rows - 1) * p.k_stride + p.dim * 2));
        const i32x4 rv = buffer_of(v_head + row0 * p.v_stride, static_cast<uint32_t>((rows - 1) * p.v_stride + p.dim * 2));
        const uint32_t to = lds_at + (t & 1) * Shape::kStageBytes + wave * 1024;
#pragma unroll
        for (int i = 0; i < Shape::kLoads; ++i) {
            const int64_t rows_on = i * Shape::kWaves * Shape::kLoadRows;
            load_to_lds<false>(rk, k_from, static_cast<uint32_t>(rows_on * p.k_stride), to + i * Shape::kWaves * 1024);
            load_to_lds<false>(rv, v_from, static_cast<uint32_t>(rows_on * p.v_stride), to + Shape::kTileBytes + i * Shape::kWaves * 1024);
        }
    };
    if (tiles > 0) load_tile(0);

    // q's rows come by whole rows, too (fragments straight from memory would be 32 rows' 32 bytes at a time)
    const uint32_t q_at = lds_at + Shape::kQAt + wave * (32 * Shape::kRowBytes);
    if (tiles > 0) {
        const i32x4 q_buffer = buffer_of(p.q + (s.q0 + first_pos) * p.q_stride + static_cast<int64_t>(kv_head) * p.group * p.dim * 2, 0x7fffffffu);
#pragma unroll
        for (int i = 0; i < 32 / Shape::kLoadRows; ++i) {
            const int in_wave = i * Shape::kLoadRows + lane / Shape::kPieces, rq = r0 + wave * 32 + in_wave;
            const int pq = list_pos(p, rq), col = (place ^ k_swizzle<DP>(in_wave)) * 8;
            const uint32_t from = static_cast<uint32_t>((pq - first_pos) * p.q_stride + ((rq - pq * p.group) * p.dim + col) * 2);
            load_to_lds<false>(q_buffer, rq < list && col < p.dim ? from : kPastTensor, 0, q_at + i * 1024);
        }
    }

    const int r = r0 + wave * 32 + row_lane, pos = list_pos(p, r), head = kv_head * p.group + r - pos * p.group;
    // keys [0, last] are visible to this lane's row
    const int last = r < list ? min(p.causal ? pos + past : s.k_len - 1, keys.end - 1) : -1;
    f32x16 o[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = f32x16{};
    float m = kMinusInf, l = 0.0f;

    // fragments' places
    const int i16 = lane & 15, v_row = 4 * half + (i16 >> 2);
    const int k_piece = (half ^ k_swizzle<DP>(row_lane)) << 4;
    const int v_piece = ((((lane / 16) & 1) * 2 + ((i16 & 3) >> 1)) ^ v_swizzle<DP>(v_row)) << 4;
    const char *k_frag[kSteps], *v_frag[kBlocks][2];
#pragma unroll
    for (int t = 0; t < kSteps; ++t) k_frag[t] = lds + row_lane * Shape::kRowBytes + (k_piece ^ (t * 32));
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e)  // a unit of eight rows on, the swizzle of 128 columns differs by a piece
            v_frag[b][e] = lds + Shape::kTileBytes + (v_row + 8 * e) * Shape::kRowBytes + (i16 & 1) * 8 +
                           (v_piece ^ (b * 64) ^ (DP == 128 ? e << 4 : 0));

    bf16x8 qf[kSteps];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int x = 0; x < kSteps; ++x) qf[x] = *reinterpret_cast<const bf16x8 *>(k_frag[x] + Shape::kQAt + wave * 32 * Shape::kRowBytes);

    auto compute = [&](int t, auto stage_, auto masked, bool infinite) TW_INLINE {
        constexpr int kStage = decltype(stage_)::value;
        constexpr bool kMasked = decltype(masked)::value;
        // some row of the wave sees a key of the tile's second half
        const bool both = !kMasked || __any(last >= keys.begin + t * Shape::kKeys + 32);
        f32x16 sc[2] = {};
        auto key_fragment = [&](int n, int x) TW_INLINE {
            return *reinterpret_cast<const bf16x8 *>(k_frag[x] + kStage * Shape::kStageBytes + n * 32 * Shape::kRowBytes);
        };
        // products [from, to) of the tile's 2 kSteps
        auto scores = [&](auto from_, auto to_) TW_INLINE {
            constexpr int kFrom = decltype(from_)::value, kTo = decltype(to_)::value;
            if constexpr (kAhead > 0) {
                bf16x8 kf[kAhead];
#pragma unroll
                for (int i = kFrom; i < kFrom + kAhead; ++i) kf[i % kAhead] = key_fragment(i / kSteps, i % kSteps);
#pragma unroll
                for (int i = kFrom; i < kTo; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    sc[i / kSteps] = Mfma<32>::run(kf[i % kAhead], qf[i % kSteps], sc[i / kSteps]);
                    if (i + kAhead < kTo) kf[i % kAhead] = key_fragment((i + kAhead) / kSteps, (i + kAhead) % kSteps);
                }
                __builtin_amdgcn_sched_barrier(0);
            } else {
#pragma unroll
                for (int i = kFrom; i < kTo; ++i)
                    sc[i / kSteps] = Mfma<32>::run(key_fragment(i / kSteps, i % kSteps), qf[i % kSteps], sc[i / kSteps]);
            }
        };
        using First = std::integral_constant<int, 0>;
        using Half = std::integral_constant<int, kSteps>;
        using All = std::integral_constant<int, 2 * kSteps>;
        if constexpr (kMasked) {
            scores(First{}, Half{});
            if (both) scores(Half{}, All{});
        } else {
            scores(First{}, All{});
        }
        if constexpr (kMasked) {
            const int seen = last - (keys.begin + t * Shape::kKeys) - 4 * half;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (n * 32 + 8 * (i / 4) + i % 4 > seen) sc[n][i] = kMinusInf;
        }
        const float alpha = softmax_max<32>(sc, p.c, &m);
        float off = taken_off(m);
        if (__any(alpha != 1.0f || large_max(off))) {
            l *= alpha;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
            if (__builtin_expect(__any(large_max(off)), 0)) take_off_large<32>(sc, p.c, p.inv_c, &off);
        }
        softmax_exp<32>(sc, p.c, off, &l);
        if constexpr (kMasked) {
            if (__builtin_expect(infinite, 0)) {
                const uint32_t lost = underflowed<32>(sc);
#pragma unroll 1
                for (int j = t * Shape::kKeys; j < min((t + 1) * Shape::kKeys, visible); ++j)
                    add_infinite<32>(o, v_head + j * p.v_stride, p.dim, half, keys.begin + j <= last, j & (Shape::kKeys - 1), lost);
            }
        }
        auto values = [&](int t4) TW_INLINE {
            u32x4 pf;
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[i] = pack_bf16x2(sc[t4 / 2][(t4 & 1) * 8 + 2 * i], sc[t4 / 2][(t4 & 1) * 8 + 2 * i + 1]);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                u32x4 vf;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 x = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                                   (lds_bf16x4_ptr_t)(v_frag[b][e] + kStage * Shape::kStageBytes + t4 * 16 * Shape::kRowBytes)));
                    vf[2 * e] = x[0];
                    vf[2 * e + 1] = x[1];
                }
                o[b] = Mfma<32>::run(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pf), o[b]);
            }
        };
        values(0);
        values(1);
        if (both) {
            values(2);
            values(3);
        }
    };

    // A wave puts zeros in the place of Inf and NaN in the pieces that it has loaded itself, before the barrier that makes them
    // everybody's.
    auto clean_values = [&](int t) TW_INLINE {
        char *const mine = lds + (t & 1) * Shape::kStageBytes + Shape::kTileBytes + threadIdx.x * 16;
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < Shape::kLoads; ++i) {
            u32x4 *const x = reinterpret_cast<u32x4 *>(mine + i * Shape::kWaves * 1024);
            u32x4 v = *x;
            uint32_t here = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                here |= infinite_bf16x2(v[w]);
                v[w] = finite_bf16x2(v[w]);
            }
            if (here) *x = v;
            bad |= here;
        }
        const bool any = __any(bad != 0);
        if (lane == 0) flags[t & 1][wave] = any;
    };
    auto cleaned = [&](int t) TW_INLINE {
        bool infinite = false;
#pragma unroll
        for (int w = 0; w < Shape::kWaves; ++w) infinite |= flags[t & 1][w] != 0;
        return __builtin_amdgcn_readfirstlane(infinite) != 0;
    };

    const bool has_rows = r0 + wave * 32 < list;
    // Between two barriers the next tile comes in, into the other half of the LDS.
    auto turn = [&](int t, auto stage, auto masked) TW_INLINE {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (decltype(masked)::value) clean_values(t);
        __syncthreads();
        if (t + 1 < tiles) load_tile(t + 1);
        if constexpr (decltype(masked)::value) {
            if (!__any(last >= keys.begin + t * Shape::kKeys)) return;
        } else if (!has_rows) {
            return;
        }
        compute(t, stage, masked, decltype(masked)::value && cleaned(t));
    };
    using Stage0 = std::integral_constant<int, 0>;
    using Stage1 = std::integral_constant<int, 1>;
    int t = 0;
    for (; t + 1 < whole; t += 2) {
        turn(t, Stage0{}, std::false_type{});
        turn(t + 1, Stage1{}, std::false_type{});
    }
    if (t < whole) {
        turn(t, Stage0{}, std::false_type{});
        ++t;
    }
    for (; t < tiles; ++t) {
        if (t & 1) turn(t, Stage1{}, std::true_type{});
        else turn(t, Stage0{}, std::true_type{});
    }

    l = row_sum<32>(l);
    if (r < list) put_row(p, chunk, (s.q0 + pos) * p.q_heads + head, m, l, half == 0);
    if (p.chunks > 1) {
        // (a chunk of no keys has no columns to put: the sum of 0 says so)
        if (r < list && keys.begin < keys.end) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    put4(p, chunk, s.q0 + pos, head, b * 32 + g * 8 + half * 4,
                         f32x4{o[b][g * 4], o[b][g * 4 + 1], o[b][g * 4 + 2], o[b][g * 4 + 3]}, 0.0f);
        }
        return;
    }
    // Results leave by whole rows: a wave's go through the part of the LDS that its rows of q came through, where nobody else
    // has been if that is no part of a stage.
    if constexpr (Shape::kQAt < 2 * Shape::kStageBytes) __syncthreads();
    char *const mine = lds + Shape::kQAt + wave * (32 * Shape::kRowBytes);
    // a row that sees no key has a sum of 0
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const u32x2 x = {pack_bf16x2(o[b][g * 4] * inv, o[b][g * 4 + 1] * inv), pack_bf16x2(o[b][g * 4 + 2] * inv, o[b][g * 4 + 3] * inv)};
            *reinterpret_cast<u32x2 *>(mine + row_lane * Shape::kRowBytes + (((b * 4 + g) ^ k_swizzle<DP>(row_lane)) << 4) + half * 8) = x;
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 32 / Shape::kLoadRows; ++i) {
        const int in_wave = i * Shape::kLoadRows + lane / Shape::kPieces, ro = r0 + wave * 32 + in_wave, po = list_pos(p, ro);
        if (ro >= list || place * 8 >= p.dim) continue;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(mine + in_wave * Shape::kRowBytes + ((place ^ k_swizzle<DP>(in_wave)) << 4));
        char *const to = p.out + (s.q0 + po) * p.out_stride + (static_cast<int64_t>(kv_head) * p.group + ro - po * p.group) * p.dim * 2;
        *reinterpret_cast<u32x4 *>(to + place * 16) = x;
    }
}

// The chunks of one row and head joined: a wave each, lane c of it with chunk c's maximum and sum.
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionParams p)
{
    const int lane = threadIdx.x & 63, c0 = lane * 2;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t row = at / p.q_heads;
    if (row >= p.q_rows) return;
    // Everything is asked for at once: whether the row is one of a sequence, and which chunks have columns, comes with them.
    const int first = p.q_offsets[0], end = p.q_offsets[p.n_seqs];
    const int64_t step = p.q_rows * p.q_heads;
    float m = kMinusInf, l = 0.0f;
    if (lane < p.chunks) {
        m = p.part_ml[(lane * step + at) * 2];
        l = p.part_ml[(lane * step + at) * 2 + 1];
    }
    float2 x[8];
    auto load_columns = [&](int c) TW_INLINE {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = {0.0f, 0.0f};
            if (c0 < p.dim && c + i < p.chunks) x[i] = *reinterpret_cast<const float2 *>(p.part + ((c + i) * step + at) * p.dim + c0);
        }
    };
    load_columns(0);
    const bool empty = m == kMinusInf;
    float top = m;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float f = empty ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    const float sum = group_sum(empty && l == 0.0f ? 0.0f : f * l, 6);
    float a = 0.0f, b = 0.0f;
    const uint64_t live = __ballot(!(empty && l == 0.0f));  // (the others' columns were not put)
    for (int c = 0; c < p.chunks; c += 8) {
        if (c > 0) load_columns(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = __shfl(f, (c + i) & 63);
            const bool put = (live >> (c + i)) & 1;
            a = fmaf(w, put ? x[i].x : 0.0f, a);
            b = fmaf(w, put ? x[i].y : 0.0f, b);
        }
    }
    if (row < first || row >= end) return;  // rows of no sequence stay as they are
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (p.lse && lane == 0) p.lse[at] = sum == 0.0f ? kMinusInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    if (c0 < p.dim)
        *reinterpret_cast<uint32_t *>(p.out + row * p.out_stride + ((at - row * p.q_heads) * p.dim + c0) * 2) =
            pack_bf16x2(a * inv, b * inv);
}

// ---- host ----

static uint64_t span(int64_t rows, int64_t stride, int64_t width)
{
    return rows == 0 ? 0 : (static_cast<uint64_t>(rows - 1) * stride + width) * 2u;
}

static constexpr int kMostChunks = 32;  // a lane each in the kernel that joins them

// How a call is launched.
struct AttentionPlan {
    int few;        // blocks of 16 rows of a tile whose four waves share the keys; 0: a wave for each 32 rows of a larger tile
    int waves;      // of a workgroup
    int tile_rows;
    int chunks;     // parts of each sequence's keys, joined by a second kernel where there are more than one
    int min_chunk;  // fewest keys of a part but the last
};

static AttentionPlan attention_plan(const tw_attention_args &a)
{
    AttentionPlan plan;
    const int64_t group = a.q_heads / a.kv_heads, list = a.q_rows * group;
    // Sequences of so few rows on average that tiles of 16 or 32 hold most of them; longer ones among them have more tiles, and all
    // together no more than twice as many as there are sequences. (4 rows each on average, 64 / 8 heads: 4 sequences with up to 1000,
    // 2000, 8000 keys 16.5, 17, 25 us, 14.5, 16.5, 26.5 in the other form; 32 of them with up to 1000, 6000, 8000 keys 22, 90, 99; 29, 96,
    // 127.)
    plan.few = list <= 16 * a.n_seqs ? 1 : list <= 32 * a.n_seqs ? 2 : 0;
    // Four waves, two workgroups to a compute unit, where sequences seldom fill tiles of 256 rows or are short, so that a workgroup's
    // start, search and results are much of its time, beside which the second one works (16 heads of 128, prompts of up to 128 tokens
    // on average, 64 and 128 of them: 44 and 45 us, 59 and 65 with eight; of 512, 16: 79, 82; 64 / 8 heads, 16 chunks of 64 rows over 2000
    // keys: 45, 48). Long sequences of many rows are read less often by tiles of 256 rows (8 heads' 512 rows over 8000 keys of 4
    // sequences: 67, 62).
    const bool short_lists = list <= 256 * a.n_seqs || (list <= 1024 * a.n_seqs && a.k_rows <= 4096 * a.n_seqs);
    plan.waves = plan.few || a.head_dim <= 64 || short_lists ? 4 : 8;
    plan.tile_rows = plan.few ? 16 * plan.few : 32 * plan.waves;
    // Keys are cut where the tiles are too few for the device, if that is estimated to save time: a workgroup takes 1.7 us for 100
    // keys (1.05 in the form for few rows; 0.72 times that for up to 64 columns), its parts 1.4 times their share if every compute
    // unit had one before the cut, and parts cost a second kernel and their sums' way through memory. (One prompt of 1500 tokens,
    // 32 / 8 heads: 43 us whole, 63 in two parts; 512 rows over 8192 keys, 64 / 8 heads: 165 us whole, 141 in two parts, 166 in four;
    // one token over 2500 keys, 32 / 8 heads: 31 us whole, 11 in parts; 16 chunks of 32 rows over up to 8000 keys, 64 / 8 heads:
    // 140 whole, 107 in two parts.) Most tiles of causal prompts are short: parts for each compute unit are enough.
    const int64_t tiles = (plan.few ? a.n_seqs : std::max(list / plan.tile_rows + 1, a.n_seqs)) * a.kv_heads, keys = a.k_rows / a.n_seqs;
    const bool pairs = plan.waves == 4 && 2 * a.q_rows < a.k_rows;
    const int64_t enough = plan.few || pairs ? 512 : 256, wanted = plan.few ? 2048 : enough;
    // (Parts of at least 128, 256, 512 keys: one token over 1500, 32 / 8 heads, 10.6, 10.6, 14.1 us, 8 over up to 800 15.4, 13.5, 17.6; 16
    // rows over 2000, 32 / 8 heads of 128, 14.7, 15.6, 18.9, 16 rows of 4 sequences each 17, 21, 27.)
    plan.min_chunk = plan.few ? 256 : 128;
    plan.chunks = 1;
    if (tiles < enough) {
        const int64_t most = std::min<int64_t>({kMostChunks, (wanted + tiles - 1) / tiles, (keys + plan.min_chunk - 1) / plan.min_chunk});
        const double longest = a.n_seqs == 1 ? keys : 1.5 * keys;
        const double whole_us = longest * (plan.few ? 0.0105 : 0.017) * (a.head_dim > 64 ? 1.0 : 0.72);
        const double sums_us = 8.0 * a.q_rows * a.q_heads * (a.head_dim + 2) / 4e6;
        double best_us = whole_us;
        for (int c = 2; c <= most; ++c) {
            const double us = whole_us / c * (!plan.few && tiles > 256 ? 1.4 : 1.0) + 3.5 + c * sums_us;
            if (us < best_us) {
                best_us = us;
                plan.chunks = c;
            }
        }
    }
    // Whole keys and fewer large tiles than compute units: smaller ones (one prompt of 2000 tokens, 16 heads of 128: 49 us, 56 with
    // eight waves).
    if (plan.waves == 8 && tiles < enough && plan.chunks == 1) plan.waves = 4;
    plan.tile_rows = plan.few ? 16 * plan.few : 32 * plan.waves;
    return plan;
}

// Workgroups of a launch: every sequence may end inside a tile, but none has more tiles than its rows need one by one.
static int64_t attention_grid(const tw_attention_args &a, const AttentionPlan &plan)
{
    const int64_t group = a.q_heads / a.kv_heads, list = a.q_rows * group;
    const int64_t tiles = std::min(list / plan.tile_rows + a.n_seqs, a.q_rows * ((group + plan.tile_rows - 1) / plan.tile_rows));
    return tiles * plan.chunks * a.kv_heads;
}
static int64_t join_grid(const tw_attention_args &a) { return (a.q_rows * a.q_heads + 3) / 4; }

// A launch has fewer than 2^32 threads.
static bool attention_launch_fits(const tw_attention_args &a)
{
    const AttentionPlan plan = attention_plan(a);
    return attention_grid(a, plan) <= INT32_MAX / 256 && (plan.chunks == 1 || join_grid(a) <= INT32_MAX / 256);
}

static tw_status attention_sizes(const tw_attention_args &a)
{
    if (a.n_seqs < 0 || a.q_rows < 0 || a.k_rows < 0 || a.q_heads < 1 || a.kv_heads < 1 || a.head_dim < 1) return TW_ERR_SHAPE;
    if (a.q_heads % a.kv_heads != 0) return TW_ERR_SHAPE;
    if (!(a.scale > 0.0f) || !(a.scale <= 0x1p127f)) return TW_ERR_SHAPE;
    if (a.head_dim % 8 != 0 || a.head_dim > TW_MAX_HEAD_DIM) return TW_ERR_UNSUPPORTED;
    if (a.q_heads > TW_MAX_HEADS || a.n_seqs > TW_MAX_SEQS) return TW_ERR_UNSUPPORTED;
    const int64_t wq = static_cast<int64_t>(a.q_heads) * a.head_dim, wk = static_cast<int64_t>(a.kv_heads) * a.head_dim;
    if (a.q_stride < wq || a.out_stride < wq || a.k_stride < wk || a.v_stride < wk) return TW_ERR_SHAPE;
    for (const int64_t s : {a.q_stride, a.k_stride, a.v_stride, a.out_stride})
        if (s % 8 != 0 || s > TW_MAX_ROW_STRIDE) return TW_ERR_UNSUPPORTED;
    if (a.n_seqs == 0 || a.q_rows == 0) return TW_OK;
    // offsets are 32-bit, and so are the places in a group's list of rows
    if (a.q_rows > INT32_MAX - 1024 || a.k_rows > INT32_MAX - 1024 || a.q_rows * (a.q_heads / a.kv_heads) > INT32_MAX - 1024)
        return TW_ERR_UNSUPPORTED;
    return attention_launch_fits(a) ? TW_OK : TW_ERR_UNSUPPORTED;
}

static int64_t attention_workspace(const tw_attention_args &a)
{
    if (a.n_seqs == 0 || a.q_rows == 0) return 0;
    const AttentionPlan plan = attention_plan(a);
    return plan.chunks == 1 ? 0 : static_cast<int64_t>(plan.chunks) * a.q_rows * a.q_heads * (a.head_dim + 2) * 4;
}

static tw_status launch_attention(void (*kernel)(AttentionParams), std::atomic<int> *allowed, int threads, int lds_bytes,
                                  const AttentionParams &p, int64_t grid, hipStream_t stream)
{
    TW_TRY(allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds_bytes, allowed));
    TW_HIP(launch_kernel(kernel, dim3(static_cast<uint32_t>(grid)), dim3(static_cast<uint32_t>(threads)),
                         static_cast<unsigned>(lds_bytes), stream, p));
    return TW_OK;
}

template <int DP, int RB>
static tw_status launch_few(const AttentionParams &p, int64_t grid, hipStream_t stream)
{
    using Shape = FewShape<DP, RB>;
    static std::atomic<int> allowed[kMaxDevices];
    return launch_attention(attention_few_kernel<DP, RB>, allowed, Shape::kThreads, Shape::kLds, p, grid, stream);
}

template <int DP, int WAVES>
static tw_status launch_wide(const AttentionParams &p, int64_t grid, hipStream_t stream)
{
    using Shape = WideShape<DP, WAVES>;
    static std::atomic<int> allowed[kMaxDevices];
    return launch_attention(attention_wide_kernel<DP, WAVES>, allowed, Shape::kThreads, Shape::kLds, p, grid, stream);
}

template <int DP>
static tw_status launch_attention_for(const AttentionParams &p, const AttentionPlan &plan, int64_t grid, hipStream_t stream)
{
    if (plan.few == 1) return launch_few<DP, 1>(p, grid, stream);
    if (plan.few == 2) return launch_few<DP, 2>(p, grid, stream);
    if constexpr (DP == 128)
        if (plan.waves == 8) return launch_wide<DP, 8>(p, grid, stream);
    return launch_wide<DP, 4>(p, grid, stream);
}

}  // namespace tw

using namespace tw;

extern "C" {

int64_t tw_attention_workspace_bytes(const tw_attention_args *args)
{
    if (!args || attention_sizes(*args) != TW_OK) return -1;
    return attention_workspace(*args);
}

tw_status tw_attention_plan(const tw_attention_args *args, tw_attention_launch *launch)
{
    if (!args || !launch) return TW_ERR_NULL;
    TW_TRY(attention_sizes(*args));
    *launch = {};
    if (args->n_seqs == 0 || args->q_rows == 0) return TW_OK;
    const AttentionPlan plan = attention_plan(*args);
    launch->tile_rows = plan.tile_rows;
    launch->key_waves = plan.few ? 4 : 1;
    launch->chunks = plan.chunks;
    launch->min_chunk = plan.min_chunk;
    return TW_OK;
}

tw_status tw_attention(const tw_attention_args *args, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!args) return TW_ERR_NULL;
    const tw_attention_args &a = *args;
    TW_TRY(attention_sizes(a));
    if (a.n_seqs == 0 || a.q_rows == 0) return TW_OK;
    if (!a.q || !a.out || !a.q_offsets || !a.k_offsets || (a.k_rows > 0 && (!a.k || !a.v))) return TW_ERR_NULL;
    if (!aligned16(a.q) || !aligned16(a.out) || !aligned16(a.k) || !aligned16(a.v)) return TW_ERR_ALIGN;
    for (const void *p : {static_cast<const void *>(a.q_offsets), static_cast<const void *>(a.k_offsets), static_cast<const void *>(a.lse)})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return TW_ERR_ALIGN;
    const int64_t need = attention_workspace(a);
    if (need > 0) {
        if (!workspace) return TW_ERR_NULL;
        if (!aligned16(workspace)) return TW_ERR_ALIGN;
        if (workspace_bytes < need) return TW_ERR_SHAPE;
    }
    const int64_t wq = static_cast<int64_t>(a.q_heads) * a.head_dim, wk = static_cast<int64_t>(a.kv_heads) * a.head_dim;
    struct Range {
        const void *p;
        uint64_t bytes;
    };
    const Range written[] = {{a.out, span(a.q_rows, a.out_stride, wq)},
                             {a.lse, a.lse ? static_cast<uint64_t>(a.q_rows) * a.q_heads * 4u : 0},
                             {workspace, static_cast<uint64_t>(need)}};
    const Range read[] = {{a.q, span(a.q_rows, a.q_stride, wq)},       {a.k, span(a.k_rows, a.k_stride, wk)},
                          {a.v, span(a.k_rows, a.v_stride, wk)},       {a.q_offsets, static_cast<uint64_t>(a.n_seqs + 1) * 4u},
                          {a.k_offsets, static_cast<uint64_t>(a.n_seqs + 1) * 4u}};
    for (int i = 0; i < 3; ++i) {
        for (const Range &r : read)
            if (ranges_overlap(written[i].p, written[i].bytes, r.p, r.bytes)) return TW_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(written[i].p, written[i].bytes, written[j].p, written[j].bytes)) return TW_ERR_ALIAS;
    }

    const AttentionPlan plan = attention_plan(a);
    const int64_t grid = attention_grid(a, plan);
    AttentionParams p;
    p.q = static_cast<const char *>(a.q);
    p.k = static_cast<const char *>(a.k);
    p.v = static_cast<const char *>(a.v);
    p.out = static_cast<char *>(a.out);
    p.lse = a.lse;
    p.q_offsets = a.q_offsets;
    p.k_offsets = a.k_offsets;
    p.part = static_cast<float *>(workspace);
    p.part_ml = p.part + static_cast<int64_t>(plan.chunks) * a.q_rows * a.q_heads * a.head_dim;
    p.q_rows = a.q_rows;
    p.k_rows = a.k_rows;
    p.q_stride = a.q_stride * 2;
    p.k_stride = a.k_stride * 2;
    p.v_stride = a.v_stride * 2;
    p.out_stride = a.out_stride * 2;
    p.n_seqs = static_cast<int>(a.n_seqs);
    p.q_heads = a.q_heads;
    p.kv_heads = a.kv_heads;
    p.group = a.q_heads / a.kv_heads;
    // exact for r < 2^31: floor(2^(31 + s) / G) + 1 with 2^s >= G
    p.group_shift = 31;
    while ((1 << (p.group_shift - 31)) < p.group) ++p.group_shift;
    p.group_magic = static_cast<uint32_t>((uint64_t(1) << p.group_shift) / p.group + 1);
    p.dim = a.head_dim;
    p.causal = a.causal != 0;
    p.chunks = plan.chunks;
    p.min_chunk = plan.min_chunk;
    p.c = static_cast<float>(a.scale * 1.4426950408889634);
    p.inv_c = 1.0f / p.c;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    TW_TRY(a.head_dim > 64 ? launch_attention_for<128>(p, plan, grid, s) : launch_attention_for<64>(p, plan, grid, s));
    if (plan.chunks > 1) {
        TW_HIP(launch_kernel(attention_join_kernel, dim3(static_cast<uint32_t>(join_grid(a))), dim3(256), 0, s, p));
    }
    return TW_OK;
}

}  // extern "C"
