// The gradient of the experts' weights: out[e](m, n) = sum over the rows r of expert e of x[r, m] y[r, n], x and y the rows of what
// the products read and of the gradient of what they wrote. Both operands of the matrix cores lie across the depth, which is the
// expert's rows, as many as there are.
#include <algorithm>
#include <atomic>

#include "tw_group.h"
#include "tw_internal.h"
#include "tw_mfma.h"

namespace tw {

// Tiles of 256 x 256, four waves of 128 x 128 (all 512 registers of a lane: 256 accumulators). Operands come 64 rows at a time
// straight into the LDS, rows of 512 bytes, and every fragment by transposing reads. These bring half of what plain ones do, 32 for
// the 64 products of 32 rows, so there are two sets of fragments of x only; those of y run two blocks ahead, each waited for by
// count. Hence y is read to the end of its 64 rows, and has three slots, x two, whose reads all go out in the first half
// of 32 rows. One barrier for 64 rows, in their middle: the next 64 have landed, x of these and y of the ones before are
// read, and the loads of the 64 after the next take their slots.
static constexpr int kEdge = 256, kStep = 64, kRowBytes = kEdge * 2, kSlotBytes = kStep * kRowBytes, kWaves = 4;
static constexpr int kBlocks = 8;      // of 16 rows, or columns, to a wave
[[maybe_unused]] static constexpr int kYSlots = 2 * kSlotBytes, kLdsBytes = 5 * kSlotBytes;
[[maybe_unused]] static constexpr uint32_t kPast = 0x80000000u;  // out of range with any scalar offset on top

struct GradientParams {
    const char *x, *y;
    char *out;
    Groups groups;
    int M, N;
    int tiles_m, tiles_n, tiles, group_m;
    int run, slots;  // tiles of a run, places of all runs
};

// Fragments: two sets of x, and of y a window of four blocks.
struct GradientFrags {
    u32x2 xlo[2][kBlocks], xhi[2][kBlocks], ylo[4], yhi[4];
    static __device__ __forceinline__ bf16x8 join(u32x2 lo, u32x2 hi)
    {
        const u32x4 t = {lo.x, lo.y, hi.x, hi.y};
        return __builtin_bit_cast(bf16x8, t);
    }
    // Until at most N of this wave's LDS reads are outstanding, and block AT of y is there
    template <int AT, int N>
    __device__ __forceinline__ void wait()
    {
        asm volatile("s_waitcnt lgkmcnt(%[n])" : "+v"(ylo[AT]), "+v"(yhi[AT]) : [n] "n"(N) : "memory");
    }
    // ... and all of set SET of x
    template <int SET, int AT, int N>
    __device__ __forceinline__ void wait_all()
    {
        wait<AT, N>();
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) asm volatile("" : "+v"(xlo[SET][i]), "+v"(xhi[SET][i]));
    }
    // Until no read is under way: what the last trip asked for past the end as well.
    __device__ __forceinline__ void settle()
    {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) asm volatile("" ::"v"(xlo[0][i]), "v"(xhi[0][i]), "v"(xlo[1][i]), "v"(xhi[1][i]));
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" ::"v"(ylo[i]), "v"(yhi[i]));
    }
};

__global__ __launch_bounds__(64 * kWaves) void expert_gradient_kernel(GradientParams p)
{
#if defined(__HIP_DEVICE_COMPILE__)  // as in tw_gemm.hip: the host pass needs the launch stub only
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_m = wave >> 1, wave_n = wave & 1, l15 = lane & 15, lgrp = lane >> 4;
    const int x_pitch = p.M * 2, y_pitch = p.N * 2;

    // Load duty: instruction i of this wave fills rows load_row + 8 i. Row r keeps piece c at c ^ ((r & 3) << 1) ^ (r & 8), so that
    // the eight rows that half a wave's transposing read touches lie in different banks.
    const int load_row = wave * 2 + lane / 32, load_piece = (lane % 32) ^ ((load_row & 3) << 1);
    // Fragment addresses inside a slot; block b lies at ^ (b << 5).
    const int j = l15 >> 2, frag_row = lgrp * 8 + j;
    auto frag_at = [&](int first_col) {
        const int col = first_col + 4 * (l15 & 3);
        return static_cast<uint32_t>(frag_row * kRowBytes + (((col >> 3) ^ (j << 1) ^ ((lgrp & 1) << 3)) << 4) + (col & 7) * 2);
    };
    const uint32_t x_at = frag_at(wave_m * 128), y_at = frag_at(wave_n * 128);

    // Tiles go to the XCDs in runs of as many as they have compute units: those of a run share rows and columns in the XCD's L2, and
    // every XCD has its part of each expert, whose depths differ (contiguous eighths instead, 8 experts: 1.8 times as long).
    for (int w = blockIdx.x; w < p.slots; w += gridDim.x) {
        const int turn = w / kXcds / p.run, lin = (turn * kXcds + w % kXcds) * p.run + w / kXcds - turn * p.run;
        if (lin >= p.tiles) continue;
        const int of_expert = p.tiles_m * p.tiles_n, e = lin / of_expert;
        const TileAt at = tile_at(lin - e * of_expert, p.tiles_m, p.tiles_n, p.group_m);
        int carry = first_group_row(p.groups);
        GroupRows rows = {};
        for (int first = 0; first <= e; first += 64) rows = group_rows(p.groups, first, lane, &carry);
        const int begin = __builtin_amdgcn_readlane(rows.begin, e & 63), depth = __builtin_amdgcn_readlane(rows.end, e & 63) - begin;
        const int m0 = at.m * kEdge, n0 = at.n * kEdge;
        const int steps = depth > kStep ? static_cast<int>((static_cast<uint32_t>(depth) + kStep - 1) / kStep) : 1;
        const char *const x = p.x + static_cast<int64_t>(begin) * x_pitch, *const y = p.y + static_cast<int64_t>(begin) * y_pitch;

        f32x4 acc[kBlocks][kBlocks];
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int m = 0; m < kBlocks; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float z;  // (by an instruction that the compiler takes for a definition: see tw_gemm.hip)
                    asm volatile("v_accvgpr_write_b32 %0, 0" : "=a"(z));
                    acc[n][m][i] = z;
                }

        // this lane's offsets in rows of even and odd instructions
        uint32_t x_off[2], y_off[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int c = (load_piece ^ (q * 8)) * 8;
            x_off[q] = m0 + c < p.M ? static_cast<uint32_t>(load_row * x_pitch + (m0 + c) * 2) : kPast;
            y_off[q] = n0 + c < p.N ? static_cast<uint32_t>(load_row * y_pitch + (n0 + c) * 2) : kPast;
        }
        struct Fetch {
            __amdgpu_buffer_rsrc_t x, y;  // the step's rows: those past the expert's lie outside
            lds_char_ptr_t to_x, to_y;
        };
        auto fetch_of = [&](int step, uint32_t slot_x, uint32_t slot_y) {
            // (in 32 bits: there are no scalar comparisons of 64)
            const uint32_t row = static_cast<uint32_t>(step) * kStep, all = static_cast<uint32_t>(depth);
            const uint32_t n = row < all ? min(all - row, static_cast<uint32_t>(kStep)) : 0u;
            const int64_t from = n > 0 ? row : 0;
            return Fetch{make_rsrc(x + from * x_pitch, n * static_cast<uint32_t>(x_pitch)),
                         make_rsrc(y + from * y_pitch, n * static_cast<uint32_t>(y_pitch)),
                         (lds_char_ptr_t)(lds + slot_x + wave * 1024), (lds_char_ptr_t)(lds + slot_y + wave * 1024)};
        };
        auto fetch_one = [&](const Fetch &f, auto i_tag) {
            constexpr int i = decltype(i_tag)::value;
            if constexpr (i < 8)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(f.x, (lds_ptr_t)(f.to_x + i * kWaves * 1024), 16, x_off[i & 1], 8 * i * x_pitch, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(f.y, (lds_ptr_t)(f.to_y + (i - 8) * kWaves * 1024), 16, y_off[i & 1],
                                                         8 * (i - 8) * y_pitch, 0, 0);
        };
        constexpr int kLoads = 16;
        auto wait_vm = [&](auto n_tag) {
            constexpr int n = decltype(n_tag)::value;
            __builtin_amdgcn_s_waitcnt(((n >> 4) << 14) | 0x0F70 | (n & 15));  // vmcnt(n)
            __builtin_amdgcn_s_barrier();
        };

        // all waves are done with the previous tile's results in the LDS
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        auto slot_x = [](int s) { return static_cast<uint32_t>(s * kSlotBytes); };
        auto slot_y = [](int s) { return static_cast<uint32_t>(kYSlots + s * kSlotBytes); };
        static_for<2>([&](auto s) {
            const Fetch f = fetch_of(decltype(s)::value, slot_x(decltype(s)::value), slot_y(decltype(s)::value));
            static_for<kLoads>([&](auto i) { fetch_one(f, i); });
        });
        wait_vm(std::integral_constant<int, kLoads>{});  // the first 64 rows have landed

        GradientFrags r;
        // half h of a fragment of block b, 32 rows kk of a slot
        auto read_y = [&](uint32_t slot, auto kk_tag, auto b_tag, auto at_tag, auto h_tag) {
            constexpr int kk = decltype(kk_tag)::value, b = decltype(b_tag)::value, to = decltype(at_tag)::value & 3, kOff = kk * kSubK * kRowBytes;
            const uint32_t addr = (slot + y_at) ^ (b << 5);
            if constexpr (decltype(h_tag)::value == 0) r.ylo[to] = lds_read_tr8<kOff>(addr);
            else r.yhi[to] = lds_read_tr8<kOff + 4 * kRowBytes>(addr);
        };
        auto read_x = [&](uint32_t slot, auto kk_tag, auto set_tag, auto i_tag) {
            constexpr int kk = decltype(kk_tag)::value, set = decltype(set_tag)::value, b = decltype(i_tag)::value / 2, kOff = kk * kSubK * kRowBytes;
            const uint32_t addr = (slot + x_at) ^ (b << 5);
            if constexpr (decltype(i_tag)::value % 2 == 0) r.xlo[set][b] = lds_read_tr8<kOff>(addr);
            else r.xhi[set][b] = lds_read_tr8<kOff + 4 * kRowBytes>(addr);
        };
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        static_for<2 * kBlocks>([&](auto i) { read_x(slot_x(0), I0{}, I0{}, i); });
        static_for<2>([&](auto b) { static_for<2>([&](auto h) { read_y(slot_y(0), I0{}, b, b, h); }); });
        // reads of x that go out during block nb of 32 rows (negative: of the 32 before)
        constexpr auto x_reads = [](int nb) { return (nb < 0 ? nb + kBlocks : nb) < kBlocks / 2 ? 4 : 0; };
        // 32 rows, of the slot's half `sub`, x in set `sub`. x of the next 32 comes from next_x, the first two blocks of y from next_y.
        auto roll = [&](auto sub_tag, uint32_t y_here, uint32_t next_x, uint32_t next_y, const Fetch &f, auto &&late) {
            constexpr int sub = decltype(sub_tag)::value, first = sub * kBlocks;
            using Next = std::integral_constant<int, 1 - sub>;
            static_for<kBlocks>([&](auto nb_tag) {
                constexpr int nb = decltype(nb_tag)::value, at = (first + nb) & 3;
                constexpr int newer = x_reads(nb - 2) + 2 + x_reads(nb - 1);  // issued after those of this block's fragment
                if constexpr (nb == 0) r.template wait_all<sub, at, 2>();
                else r.template wait<at, newer>();
                static_for<kBlocks>([&](auto mb_tag) {
                    constexpr int mb = decltype(mb_tag)::value, m = nb * kBlocks + mb;
                    acc[nb][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(GradientFrags::join(r.ylo[at], r.yhi[at]),
                                                                          GradientFrags::join(r.xlo[sub][mb], r.xhi[sub][mb]), acc[nb][mb], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (mb < 2) {
                        using To = std::integral_constant<int, first + nb + 2>;
                        if constexpr (nb + 2 < kBlocks) read_y(y_here, sub_tag, std::integral_constant<int, nb + 2>{}, To{}, mb_tag);
                        else read_y(next_y, Next{}, std::integral_constant<int, nb + 2 - kBlocks>{}, To{}, mb_tag);
                    }
                    if constexpr (x_reads(nb) > 0 && mb >= 2 && mb < 6) read_x(next_x, Next{}, Next{}, std::integral_constant<int, 4 * nb + mb - 2>{});
                    if constexpr (sub == 1)
                        static_for<kLoads>([&](auto t_tag) {
                            if constexpr (decltype(t_tag)::value * (kBlocks * kBlocks) / kLoads + 2 == m) fetch_one(f, t_tag);
                        });
                    if constexpr (m == kBlocks * kBlocks * 3 / 4) late();
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        };
        uint32_t here_x = slot_x(0), next_x = slot_x(1), here_y = slot_y(0), next_y = slot_y(1), free_y = slot_y(2);
        Fetch f = fetch_of(2, here_x, free_y);
        for (int s = 0; s < steps; ++s) {
            roll(I0{}, here_y, here_x, here_y, f, [&] { f = fetch_of(s + 2, here_x, free_y); });
            wait_vm(I0{});
            roll(I1{}, here_y, next_x, next_y, f, [] {});
            const uint32_t x0 = here_x, y0 = here_y;
            here_x = next_x;
            next_x = x0;
            here_y = next_y;
            next_y = free_y;
            free_y = y0;
        }
        r.settle();
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): loads past the end still target the LDS

        // Results through the LDS, each wave in a region of its own, rows padded by 32 bytes, so that a store covers whole rows.
        char *const out = p.out + (static_cast<int64_t>(e) * p.M + m0) * y_pitch;
        const int rows_m = min(kEdge, p.M - m0);
        const __amdgpu_buffer_rsrc_t to = make_rsrc(out, static_cast<uint32_t>(rows_m * y_pitch));
        constexpr int kPitch = 16 * kBlocks * 2 + 32, kRegion = 16 * kBlocks * kPitch;
        static_assert(kWaves * kRegion <= kLdsBytes, "the waves' regions");
        __builtin_amdgcn_s_barrier();  // every wave has its last fragments
        const uint32_t region = static_cast<uint32_t>(wave * kRegion), put = region + l15 * kPitch + lgrp * 8;
#pragma unroll
        for (int m = 0; m < kBlocks; ++m) {
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) {
                const u32x2 v = {pack_bf16x2(acc[n][m][0], acc[n][m][1]), pack_bf16x2(acc[n][m][2], acc[n][m][3])};
                *reinterpret_cast<__attribute__((address_space(3))) u32x2 *>(static_cast<uintptr_t>(put + m * 16 * kPitch + n * 32)) = v;
            }
            __builtin_amdgcn_sched_barrier(0);  // one block row's accumulators at a time
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the region is this wave's own
        const int col = n0 + wave_n * 128 + (lane % 16) * 8, row = lane / 16;
        const uint32_t to_off = col < p.N ? static_cast<uint32_t>((wave_m * 128 + row) * y_pitch + col * 2) : kPast;
        const uint32_t get = region + row * kPitch + (lane % 16) * 16;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const u32x4 v = *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(static_cast<uintptr_t>(get + i * 4 * kPitch));
            __builtin_amdgcn_raw_buffer_store_b128(v, to, to_off + static_cast<uint32_t>(4 * i * y_pitch), 0, kStorePolicy);  // (no scalar offset: see st())
        }
    }
#endif
}

// Few rows to an expert, or few tiles: the results are most of what moves, and a large tile's start and end most of its time. Tiles of 128 x 128,
// four waves of 64 x 64, four workgroups to a compute unit, so that one's loads run beside the others' products and stores; 32 rows at a
// time, two slots, and the results through the LDS by whole rows. 1172 rows of 16 experts, [2048 x 1024] each: 26.0 to 16.7 us; 400 of 8,
// [4096 x 3584]: 82 to 55 (three workgroups 61, with three slots as well).
static constexpr int kThinEdge = 128, kThinStep = 32, kThinRowBytes = kThinEdge * 2, kThinSlot = 2 * kThinStep * kThinRowBytes;
static constexpr int kThinPitch = kThinRowBytes + 32, kThinLds = kThinEdge * kThinPitch, kThinAtOnce = 4;
static_assert(2 * kThinSlot <= kThinLds, "the slots lie in the results' room");

__global__ __launch_bounds__(64 * kWaves, kThinAtOnce) void expert_gradient_thin_kernel(GradientParams p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_m = wave >> 1, wave_n = wave & 1, l15 = lane & 15, lgrp = lane >> 4;
    const int x_pitch = p.M * 2, y_pitch = p.N * 2;
    // Instruction i of this wave fills rows load_row + 16 i. Row r keeps piece c at c ^ ((r & 3) << 1) ^ (r & 8).
    const int load_row = wave * 4 + lane / 16, load_piece = (lane % 16) ^ ((load_row & 3) << 1) ^ (load_row & 8);
    const int j = l15 >> 2, frag_row = lgrp * 8 + j;
    auto frag_at = [&](int first_col) {
        const int col = first_col + 4 * (l15 & 3);
        return static_cast<uint32_t>(frag_row * kThinRowBytes + (((col >> 3) ^ (j << 1) ^ ((lgrp & 1) << 3)) << 4) + (col & 7) * 2);
    };
    const uint32_t x_at = frag_at(wave_m * 64), y_at = kThinStep * kThinRowBytes + frag_at(wave_n * 64);

    for (int w = blockIdx.x; w < p.slots; w += gridDim.x) {
        const int turn = w / kXcds / p.run, lin = (turn * kXcds + w % kXcds) * p.run + w / kXcds - turn * p.run;
        if (lin >= p.tiles) continue;
        const int of_expert = p.tiles_m * p.tiles_n, e = lin / of_expert;
        const TileAt at = tile_at(lin - e * of_expert, p.tiles_m, p.tiles_n, p.group_m);
        int carry = first_group_row(p.groups);
        GroupRows rows = {};
        for (int first = 0; first <= e; first += 64) rows = group_rows(p.groups, first, lane, &carry);
        const int begin = __builtin_amdgcn_readlane(rows.begin, e & 63), depth = __builtin_amdgcn_readlane(rows.end, e & 63) - begin;
        const int m0 = at.m * kThinEdge, n0 = at.n * kThinEdge;
        const int steps = static_cast<int>((static_cast<uint32_t>(depth) + kThinStep - 1) / kThinStep);
        const char *const x = p.x + static_cast<int64_t>(begin) * x_pitch, *const y = p.y + static_cast<int64_t>(begin) * y_pitch;
        const int c = load_piece * 8;
        const uint32_t x_off = m0 + c < p.M ? static_cast<uint32_t>(load_row * x_pitch + (m0 + c) * 2) : kPast;
        const uint32_t y_off = n0 + c < p.N ? static_cast<uint32_t>(load_row * y_pitch + (n0 + c) * 2) : kPast;
        auto fetch = [&](int step, int slot) {
            const uint32_t row = static_cast<uint32_t>(step) * kThinStep, n = min(static_cast<uint32_t>(depth) - row, static_cast<uint32_t>(kThinStep));
            const __amdgpu_buffer_rsrc_t rx = make_rsrc(x + static_cast<int64_t>(row) * x_pitch, n * static_cast<uint32_t>(x_pitch));
            const __amdgpu_buffer_rsrc_t ry = make_rsrc(y + static_cast<int64_t>(row) * y_pitch, n * static_cast<uint32_t>(y_pitch));
            const lds_char_ptr_t to = (lds_char_ptr_t)(lds + slot * kThinSlot + wave * 1024);
            static_for<2>([&](auto i_tag) {
                constexpr int i = decltype(i_tag)::value;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_ptr_t)(to + i * kWaves * 1024), 16, x_off, 16 * i * x_pitch, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ry, (lds_ptr_t)(to + (i + 2) * kWaves * 1024), 16, y_off, 16 * i * y_pitch, 0, 0);
            });
        };

        f32x4 acc[4][4];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int m = 0; m < 4; ++m) acc[n][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // all waves are done with the previous tile's results in the LDS
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        if (steps > 0) fetch(0, 0);
        for (int s = 0; s < steps; ++s) {
            if (s + 1 < steps) {
                fetch(s + 1, (s + 1) & 1);
                __builtin_amdgcn_s_waitcnt(0x0F74);  // vmcnt(4): this step's
            } else {
                __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
            }
            __builtin_amdgcn_s_barrier();
            const uint32_t slot = static_cast<uint32_t>((s & 1) * kThinSlot);
            u32x2 xlo[4], xhi[4], ylo[4], yhi[4];
            static_for<4>([&](auto b_tag) {
                constexpr int b = decltype(b_tag)::value;
                const uint32_t ax = (slot + x_at) ^ (b << 5), ay = (slot + y_at) ^ (b << 5);
                xlo[b] = lds_read_tr8<0>(ax);
                xhi[b] = lds_read_tr8<4 * kThinRowBytes>(ax);
                ylo[b] = lds_read_tr8<0>(ay);
                yhi[b] = lds_read_tr8<4 * kThinRowBytes>(ay);
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int b = 0; b < 4; ++b) asm volatile("" : "+v"(xlo[b]), "+v"(xhi[b]), "+v"(ylo[b]), "+v"(yhi[b]));
            __builtin_amdgcn_s_barrier();  // every wave has this slot's fragments
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(GradientFrags::join(ylo[n], yhi[n]), GradientFrags::join(xlo[m], xhi[m]),
                                                                        acc[n][m], 0, 0, 0);
        }

        // (every wave has its last fragments: the barrier above, or nothing was loaded)
        const uint32_t put = static_cast<uint32_t>((wave_m * 64 + l15) * kThinPitch + wave_n * 128 + lgrp * 8);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const u32x2 v = {pack_bf16x2(acc[n][m][0], acc[n][m][1]), pack_bf16x2(acc[n][m][2], acc[n][m][3])};
                *reinterpret_cast<__attribute__((address_space(3))) u32x2 *>(static_cast<uintptr_t>(put + m * 16 * kThinPitch + n * 32)) = v;
            }
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        char *const out = p.out + (static_cast<int64_t>(e) * p.M + m0) * y_pitch;
        const __amdgpu_buffer_rsrc_t to = make_rsrc(out, static_cast<uint32_t>(min(kThinEdge, p.M - m0) * y_pitch));
        const int row = wave * 32 + lane / 16, col = n0 + (lane % 16) * 8;
        const uint32_t to_off = col < p.N ? static_cast<uint32_t>(row * y_pitch + col * 2) : kPast;
        const uint32_t get = static_cast<uint32_t>(row * kThinPitch + (lane % 16) * 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const u32x4 v = *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(static_cast<uintptr_t>(get + i * 4 * kThinPitch));
            __builtin_amdgcn_raw_buffer_store_b128(v, to, to_off + static_cast<uint32_t>(4 * i * y_pitch), 0, kStorePolicy);  // (no scalar offset: see st())
        }
    }
#endif
}

// us, tiles of 256 x 256 and of 128 x 128. By the rows of an expert: 8 experts' [4096 x 3584], 300 rows each 127 and 116, 500 rows 163 and 160; [4096 x
// 2048], 1000 rows 162 and 169; 128 experts' [2048 x 1024], 250 rows 327 and 267, 500 rows 440 and 426; 64 experts' [2816 x 1408], 375 rows 357 and 295.
// Where half of the compute units would have no large tile: 8 experts' [1024 x 1024], 500 rows 27 and 17, 4000 rows 155 and 119.
static bool thin_tiles(int64_t rows, int64_t M, int64_t N, int n_experts, int cus)
{
    const int64_t large = ((M + kEdge - 1) / kEdge) * ((N + kEdge - 1) / kEdge) * n_experts;
    return rows < 400 * int64_t(n_experts) || 2 * large <= cus;
}

// Tiles of a run of neighbouring ones in an XCD, and the places of all runs, which are as many in each XCD.
struct GradientRuns {
    int64_t run, slots;
};
static GradientRuns gradient_runs(int64_t tiles, int at_once, int cus)
{
    const int64_t run = std::min<int64_t>((tiles + kXcds - 1) / kXcds, std::max(1, cus * at_once / kXcds));
    return {run, ((tiles + run - 1) / run + kXcds - 1) / kXcds * kXcds * run};
}

GroupLaunch plan_expert_gradient(int64_t rows, int64_t M, int64_t N, int n_experts, int cus)
{
    const bool thin = thin_tiles(rows, M, N, n_experts, cus);
    const int edge = thin ? kThinEdge : kEdge, at_once = thin ? kThinAtOnce : 1;
    const int64_t tiles = (M + edge - 1) / edge * ((N + edge - 1) / edge) * n_experts, slots = gradient_runs(tiles, at_once, cus).slots;
    // Workgroups that take tile after tile where these are few, else one for each: 2048 small tiles 13.4-20.4 us and 15.1-20.4, 7168 42-63 and 43-60, 16384 102-168 and 94-163.
    const bool stay = !thin || slots <= int64_t(4) * cus * at_once;
    return {edge, edge, tiles, std::min<int64_t>(slots, stay ? cus * at_once : 1 << 20)};
}

tw_status launch_expert_gradient(const void *x, const void *y, void *out, const int32_t *offsets, int64_t rows, int64_t M, int64_t N,
                                 int n_experts, hipStream_t stream)
{
    int cus = 0;
    TW_TRY(current_cu_count(&cus));
    const GroupLaunch l = plan_expert_gradient(rows, M, N, n_experts, cus);
    if (l.tiles > (1 << 30)) return TW_ERR_UNSUPPORTED;
    const bool thin = l.tile_rows == kThinEdge;
    const GradientRuns runs = gradient_runs(l.tiles, thin ? kThinAtOnce : 1, cus);
    GradientParams p = {};
    p.x = static_cast<const char *>(x);
    p.y = static_cast<const char *>(y);
    p.out = static_cast<char *>(out);
    p.groups = {offsets, n_experts, static_cast<int>(rows)};
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.tiles_m = static_cast<int>((M + l.tile_rows - 1) / l.tile_rows);
    p.tiles_n = static_cast<int>((N + l.tile_cols - 1) / l.tile_cols);
    p.tiles = static_cast<int>(l.tiles);
    p.run = static_cast<int>(runs.run);
    p.slots = static_cast<int>(runs.slots);
    p.group_m = tile_group_m(p.tiles_m, p.run, l.tile_rows, l.tile_cols, cus);
    const dim3 grid(static_cast<uint32_t>(l.workgroups));
    if (thin) {
        TW_HIP(launch_kernel(expert_gradient_thin_kernel, grid, dim3(64 * kWaves), kThinLds, stream, p));
        return TW_OK;
    }
    static std::atomic<int> allowed[kMaxDevices];
    TW_TRY(allow_dynamic_lds(reinterpret_cast<const void *>(expert_gradient_kernel), kLdsBytes, allowed));
    TW_HIP(launch_kernel(expert_gradient_kernel, grid, dim3(64 * kWaves), kLdsBytes, stream, p));
    return TW_OK;
}

}  // namespace tw
