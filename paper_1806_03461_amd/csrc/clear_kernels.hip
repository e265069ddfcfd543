// gfx950 kernels of layers in the clear: the 8-bit matrix product, and the two row operators that feed it (norm, gated activation).
#include "clear_kernels.h"

#include <algorithm>
#include <type_traits>

namespace tfhe {

typedef int v4i __attribute__((ext_vector_type(4)));

// The same value, but for the compiler another: what follows from it is computed anew, not kept in registers from before.
__device__ __forceinline__ int again(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// ---- the product ---------------------------------------------------------------------------------------------------

// 16 bytes of a row from byte `at` on, of which only those before `k` count: the rest is 0 and not read.  At the row's end the last
// 16 bytes are read and shifted down, one load in any case.
__device__ __forceinline__ v4i load_16(const int8_t *row, int at, int k) {
    v4i v = {0, 0, 0, 0};
    if (k >= 16) {
        const int from = std::min(at, k - 16), bits = 8 * std::min(at - from, 16);
        uint64_t half[2];
        __builtin_memcpy(half, row + from, 16);
        if (bits >= 64) half[0] = bits < 128 ? half[1] >> (bits - 64) : 0, half[1] = 0;
        else if (bits > 0) half[0] = half[0] >> bits | half[1] << (64 - bits), half[1] >>= bits;
        __builtin_memcpy(&v, half, 16);
    } else {
        for (int j = 0; j < 16; ++j)
            if (at + j < k) v[j >> 2] |= (int)(uint8_t)row[at + j] << (8 * (j & 3));
    }
    return v;
}

// v[0 .. 3] = p[0 .. left - 1], the rest as they are
template <class T>
__device__ __forceinline__ void load_4(T (&v)[4], const T *p, int left) {
    if (left == 4) {
        __builtin_memcpy(v, p, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) v[e] = p[e];
    }
}

// past: past the caches' order of what to keep
template <class T>
__device__ __forceinline__ void store_4(T *p, const T (&v)[4], int left, bool past) {
    typedef unsigned char Bytes __attribute__((ext_vector_type(sizeof v), aligned(sizeof(T))));
    if (left == 4 && past) {
        Bytes b;
        __builtin_memcpy(&b, v, sizeof v);
        __builtin_nontemporal_store(b, reinterpret_cast<Bytes *>(p));
    } else if (left == 4) {
        __builtin_memcpy(p, v, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) p[e] = v[e];
    }
}

// What four neighbouring channels j .. j + 3, of which `left` exist, bring to their outputs.
struct Channels {
    float scale[4];
    int bias[4];        // bits of the floats or the whole numbers that they are
    int left;
};

// The outputs of token i and channels j .. j + 3 from their sums.
__device__ __forceinline__ void finish_4(const DenseClearArgs &a, int64_t i, int64_t j, v4i acc, float x_scale, const Channels &c) {
    const int64_t at = i * a.ldo + j;
    if (a.kind >= BNN_CLEAR_I32) {
        if (a.kind == BNN_CLEAR_I32) {
            int o[4];
            for (int e = 0; e < 4; ++e) o[e] = (int)((unsigned)acc[e] + (unsigned)c.bias[e]);
            store_4(static_cast<int *>(a.out) + at, o, c.left, a.past);
        } else {
            const int8_t no = a.kind == BNN_CLEAR_SIGN ? -1 : 0;
            int8_t o[4];
            for (int e = 0; e < 4; ++e) o[e] = (int64_t)acc[e] + c.bias[e] >= 0 ? (int8_t)1 : no;
            store_4(static_cast<int8_t *>(a.out) + at, o, c.left, a.past);
        }
        return;
    }
    float y[4];
    for (int e = 0; e < 4; ++e) y[e] = (float)acc[e] * x_scale * c.scale[e] + __int_as_float(c.bias[e]);
    if (a.kind == BNN_CLEAR_F32) {
        store_4(static_cast<float *>(a.out) + at, y, c.left, a.past);
    } else if (a.kind == BNN_CLEAR_BF16) {
        __bf16 o[4];
        for (int e = 0; e < 4; ++e) o[e] = (__bf16)y[e];
        store_4(static_cast<__bf16 *>(a.out) + at, o, c.left, a.past);
    } else {
        _Float16 o[4];
        for (int e = 0; e < 4; ++e) o[e] = (_Float16)y[e];
        store_4(static_cast<_Float16 *>(a.out) + at, o, c.left, a.past);
    }
}

// Waits until at most `left` of the wave's loads into LDS are under way, then meets the workgroup.
template <int left>
__device__ __forceinline__ void landed_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(left) : "memory");
}

// The same with all loads, and all of the wave's reads and writes of LDS.
__device__ __forceinline__ void settled_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Memory that buffer loads see: `bytes` from p on.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const int8_t *p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p), (short)0, bytes, 0x00020000);
}

// 16 bytes a lane from memory into LDS: lane l's go to `to` + 16 l.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, int offset, int step, int8_t *to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, offset, step, 0, 0);
}

// Tiles of (WT * RT * 16) tokens by (WC * RC * 16) channels, a workgroup of WT x WC waves each, every wave RT x RC products of 16 by 16.
// (Products of 32 by 32 do the same work with half the instructions, but read and write every sum twice as often: on all CUs and random operands,
// where power sets the clock, 3.2 Pop/s of them against 3.9 of these.)
// BK bytes of k are a step, and four steps have a place in LDS: the wave holds one step's operands in registers and reads the
// next one's behind each row of products, and the loads of the two after that are under way.  The places are four arrays and the loop is unrolled over
// them, or the compiler would take each read of LDS to depend on the loads into it and wait for them all.  A row's 16-byte pieces lie in LDS at place (piece ^
// something of the row), so that eight lanes that read the same piece of eight rows meet all banks.
// The channels are the products' rows: a lane then holds four neighbouring channels of a token.
//   DIRECT: rows begin at multiples of 4 bytes, and pieces go from memory to LDS directly, but for the last step if k is no whole number of
//   steps.  Otherwise all go through registers, two or four steps ahead.
template <int WT, int WC, int RT, int RC, int BK, bool DIRECT>
__global__ void __launch_bounds__(64 * WT * WC, 2) dense_tile_kernel(DenseClearArgs a) {
    constexpr int kThreads = 64 * WT * WC, kWaves = WT * WC, TT = 16 * WT * RT, TC = 16 * WC * RC;
    constexpr int kPerRow = BK / 16;                        // pieces a row
    constexpr int kRows = kThreads / kPerRow;               // rows of one piece a thread
    constexpr int kXPieces = TT / kRows, kPieces = (TT + TC) / kRows;
    constexpr int kStage = (TT + TC) * BK, kInner = BK / 64;
    constexpr int kRow = 16 * RC + 4;                       // words of a token's channels as its sums pass through LDS
    static_assert(kXPieces * kRows == TT && kPieces * kRows == TT + TC && kRows % 8 == 0, "whole pieces a thread");
    constexpr int kPerPlace = (kWaves + 3) / 4;             // waves whose sums pass through one place
    static_assert(kPerPlace * 32 * kRow * 4 <= kStage, "the sums pass through the operands' LDS");
    __shared__ __attribute__((aligned(1024))) int8_t place_0[kStage], place_1[kStage], place_2[kStage], place_3[kStage];
    int8_t *const place[4] = {place_0, place_1, place_2, place_3};
    __shared__ __attribute__((aligned(16))) float x_scales[TT], w_scales[TC];
    __shared__ __attribute__((aligned(16))) int biases[TC];
    static_assert(TT <= kThreads && TC <= kThreads, "a thread a token or channel");
    const unsigned across = (unsigned)((a.n + TC - 1) / TC), down = (unsigned)((a.m + TT - 1) / TT), tiles = across * down;
    const int whole = a.k / BK, steps = (a.k + BK - 1) / BK;
    const auto turned = [](int row) { return BK == 128 ? row & 7 : (row >> 1) & 3; };
    for (unsigned id = blockIdx.x; id < tiles; id += gridDim.x) {
        // (found anew for each tile: kept from one to the next, addresses would take registers from the sums)
        const int t = again(threadIdx.x), lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
        // Workgroups go round the eight XCDs; each XCD gets neighbouring tiles, four token tiles by all channels at a time, so that
        // its L2 is asked for the same rows.
        const unsigned xcd = id & 7, share = tiles >> 3, over = tiles & 7, lin = xcd * share + std::min(xcd, over) + (id >> 3);
        const unsigned band = lin / (4 * across), in_band = lin - band * 4 * across, first = band * 4, high = std::min(down - first, 4u);
        const int64_t i0 = (int64_t)(first + in_band % high) * TT, j0 = (int64_t)(in_band / high) * TC;

        // what the outputs take, asked for now and laid aside before the first product
        const bool x_mine = t < TT && i0 + t < a.m, w_mine = t < TC && j0 + t < a.n;
        const float my_x_scale = x_mine && a.x_scale ? a.x_scale[i0 + t] : 1.0f, my_w_scale = w_mine && a.w_scale ? a.w_scale[j0 + t] : 1.0f;
        const int my_bias = w_mine && a.bias ? static_cast<const int *>(a.bias)[j0 + t] : 0;
        // piece p of a thread: row p * kRows + t / kPerRow of the tile's tokens, then of its channels
        const int my_row = t / kPerRow, piece = t % kPerRow ^ turned(my_row);
        const int x_last = (int)std::min<int64_t>(a.m - i0, TT) - 1, w_last = (int)std::min<int64_t>(a.n - j0, TC) - 1;
        using Offset = std::conditional_t<DIRECT, int, int64_t>;        // from the tile's first row; strides are small if DIRECT
        const auto row_offset = [&](int p) {
            // beyond the last row: that row again, never stored
            return p < kXPieces ? (Offset)std::min(p * kRows + my_row, x_last) * (Offset)a.ldx
                                : (Offset)std::min((p - kXPieces) * kRows + my_row, w_last) * (Offset)a.ldw;
        };
        Offset offset[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) offset[p] = row_offset(p) + 16 * piece;
        const int8_t *const x_rows = a.x + i0 * a.ldx, *const w_rows = a.w + j0 * a.ldw;
        const auto through = [&](v4i (&held)[kPieces], int s, auto... is_whole) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                const int8_t *from = (p < kXPieces ? x_rows : w_rows) + offset[p];
                if ((is_whole || ... || (s < whole))) __builtin_memcpy(&held[p], from + BK * s, 16);
                else held[p] = load_16(from - 16 * piece, BK * s + 16 * piece, a.k);
            }
        };
        const auto settle = [&](const v4i (&held)[kPieces], int8_t *to) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *reinterpret_cast<v4i *>(to + (p * kThreads + t) * 16) = held[p];
        };

        const auto lay_aside = [&] {
            if (t < TT) x_scales[t] = my_x_scale;
            if (t < TC) w_scales[t] = my_w_scale, biases[t] = my_bias;
        };
        v4i acc[RT][RC] = {};
        // operands of 64 bytes of k: the channels' in turn, a token row's in the place of the one before
        v4i fx[RT], fw[2][RC];
        const int row_x = (wave / WC) * 16 * RT + (lane & 15), row_w = TT + (wave % WC) * 16 * RC + (lane & 15);
        const auto operand = [&](const int8_t *from, int at_row, int kk) {
            return *reinterpret_cast<const v4i *>(from + at_row * BK + 16 * ((4 * kk + (lane >> 4)) ^ turned(lane & 15)));
        };
        const auto first_operands = [&] {
#pragma unroll
            for (int c = 0; c < RC; ++c) fw[0][c] = operand(place[0], row_w + 16 * c, 0);
#pragma unroll
            for (int r = 0; r < RT; ++r) fx[r] = operand(place[0], row_x + 16 * r, 0);
        };
        // the step in place I, the next one's operands coming in; behind the last step they are whatever lies there, and not used
        const auto multiply = [&](auto at) {
            constexpr int I = decltype(at)::value;
#pragma unroll
            for (int kk = 0; kk < kInner; ++kk) {
                const int turn = kInner == 1 ? I & 1 : kk & 1, next = kk + 1 < kInner ? kk + 1 : 0;
                const int8_t *from = place[kk + 1 < kInner ? I : (I + 1) % 4];
#pragma unroll
                for (int c = 0; c < RC; ++c) fw[turn ^ 1][c] = operand(from, row_w + 16 * c, next);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
#pragma unroll
                    for (int c = 0; c < RC; ++c) acc[r][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[turn][c], fx[r], acc[r][c], 0, 0, 0);
                    fx[r] = operand(from, row_x + 16 * r, next);
                    // left to itself the compiler reads just before use, and lets products of the next step pass the border
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // four steps, each with its place as a constant
        const auto by_four = [](auto &&one) {
            one(std::integral_constant<int, 0>{});
            one(std::integral_constant<int, 1>{});
            one(std::integral_constant<int, 2>{});
            one(std::integral_constant<int, 3>{});
        };
        int s = 0;
        if constexpr (DIRECT) {
            // bytes of the tile's rows, from its first row's beginning to its last row's end
            const int x_bytes = x_last * (int)a.ldx + a.k, w_bytes = w_last * (int)a.ldw + a.k;
            const auto xr = buffer_of(x_rows, x_bytes), wr = buffer_of(w_rows, w_bytes);
            constexpr bool kEarly = RT * RC < 16;                  // registers for the last, partial step from the start on
            v4i held[kEarly ? kPieces : 1];
            const auto fetch = [&](int s, int8_t *to) {
#pragma unroll
                for (int p = 0; p < kPieces; ++p) {
                    int8_t *at = to + p * 16 * kThreads + 1024 * wave;
                    if (p < kXPieces) load_to_lds(xr, offset[p], BK * s, at);
                    else load_to_lds(wr, offset[p], BK * s, at);
                }
            };
            const auto prepare = [&](int s, int8_t *to) {
                if (s < whole) {
                    fetch(s, to);
                } else if (s < steps) {
                    if constexpr (kEarly) {
                        settle(held, to);
                    } else {
                        const int late = again(t);
#pragma unroll 1
                        for (int p = 0; p < kPieces; ++p) {
                            const int r = late / kPerRow, piece = late % kPerRow ^ turned(r);
                            const int8_t *from = p < kXPieces ? x_rows + (int64_t)std::min(p * kRows + r, x_last) * a.ldx
                                                              : w_rows + (int64_t)std::min((p - kXPieces) * kRows + r, w_last) * a.ldw;
                            *reinterpret_cast<v4i *>(to + (p * kThreads + late) * 16) = load_16(from, BK * s + 16 * piece, a.k);
                        }
                    }
                }
            };
            if constexpr (kEarly)
                if (whole < steps) through(held, whole);
            prepare(0, place[0]);
            prepare(1, place[1]);
            prepare(2, place[2]);
            lay_aside();
            if (whole >= 3) landed_and_meet<2 * kPieces>();
            else settled_and_meet();
            first_operands();
            // At each step: the next one has come, and everyone is done with the one before, whose place the following loads take.  Its operands
            // were read while the step before it was multiplied, and waited for since.
            for (; s + 6 < whole; s += 4)
                by_four([&](auto at) {
                    constexpr int I = decltype(at)::value;
                    landed_and_meet<kPieces>();
                    fetch(s + I + 3, place[(I + 3) % 4]);
                    multiply(at);
                });
            for (; s < steps; s += 4)
                by_four([&](auto at) {
                    constexpr int I = decltype(at)::value;
                    if (s + I < steps) {
                        settled_and_meet();
                        prepare(s + I + 3, place[(I + 3) % 4]);
                        multiply(at);
                    }
                });
        } else {
            constexpr int kSets = RT * RC >= 16 ? 2 : 4;            // steps under way to registers, as many as there is room for
            v4i held[kSets][kPieces];
#pragma unroll
            for (int h = 0; h < kSets; ++h)
                if (h < steps) through(held[h], h);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h < steps) settle(held[h], place[h]);
                if (h + kSets < steps) through(held[h], h + kSets);
            }
            lay_aside();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            first_operands();
            // without conditions as long as there are whole steps, or the compiler would not know how many loads it may leave under way
            const auto four_steps = [&](auto all) {
                by_four([&](auto at) {
                    constexpr int I = decltype(at)::value, kSet = (I + 2) % kSets;
                    if (all || s + I < steps) {
                        // the next step is there, and everyone is done with the one before the last, whose place the one after the next takes
                        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                        if (all || s + I + 2 < steps) settle(held[kSet], place[(I + 2) % 4]);
                        if (all || s + I + 2 + kSets < steps) through(held[kSet], s + I + 2 + kSets, all);
                        multiply(at);
                    }
                });
            };
            for (; s + 5 + kSets < whole; s += 4) four_steps(std::true_type{});
            for (; s < steps; s += 4) four_steps(std::false_type{});
        }
        settled_and_meet();
        // The wave's sums go through LDS of its own, 32 tokens at a time, so that its stores are whole
        // stretches of a token's channels.  A lane has the same four channels of every token.
        const int late = again(t) & 63;         // the lane
        constexpr int kFours = 4 * RC, kTurns = 32 * kFours / 64;
        static_assert(RT % 2 == 0 && 64 % kFours == 0, "32 tokens at a time, a lane the same channels");
        int8_t *const my_place = wave / kPerPlace == 0 ? place_0 : wave / kPerPlace == 1 ? place_1 : wave / kPerPlace == 2 ? place_2 : place_3;
        int *own = reinterpret_cast<int *>(my_place) + wave % kPerPlace * 32 * kRow;
        const int wave_t = (wave / WC) * 16 * RT, wave_c = (wave % WC) * 16 * RC + 4 * (late % kFours);
        const int64_t j = j0 + wave_c;
        Channels channels;
        channels.left = a.n - j < 4 ? (int)(a.n - j) : 4;
        __builtin_memcpy(channels.scale, w_scales + wave_c, 16);
        __builtin_memcpy(channels.bias, biases + wave_c, 16);
#pragma unroll
        for (int r = 0; r < RT; r += 2) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int c = 0; c < RC; ++c)
                    *reinterpret_cast<v4i *>(own + (16 * half + (late & 15)) * kRow + 16 * c + 4 * (late >> 4)) = acc[r + half][c];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            v4i sums[kTurns];
            float x_scale[kTurns];
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int token = late / kFours + 64 / kFours * u;
                sums[u] = *reinterpret_cast<const v4i *>(own + token * kRow + 4 * (late % kFours));
                x_scale[u] = x_scales[wave_t + 16 * r + token];
            }
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int64_t i = i0 + wave_t + 16 * r + late / kFours + 64 / kFours * u;
                if (i < a.m && channels.left > 0) finish_4(a, i, j, sums[u], x_scale[u], channels);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        if (id + gridDim.x < tiles) settled_and_meet();       // before the next tile's loads
    }
}

// Few tokens (up to 16 RT): the weights are read once and that is what it costs.  A workgroup takes 16 RC channels, its waves
// consecutive parts of k, 64 bytes at a time; the weights go from memory to the products' registers without LDS, the waves' sums meet there.
// Two blocks under way a wave leave registers for 28 waves a CU (one token, 10240 -> 4096 8.8 us, four 10.7, eight 10.0).
// One token on weights that the 256 MB behind the L2s keep from one call to the next, and on weights from memory (a ring of 640 MB), the smallest call being
// 2.0 us: 4096 -> 4096 4.9 and 6.5 us, 10240 -> 4096 8.6 and 11.2, 4096 -> 131072, which they cannot keep, 89, 6.0 TB/s.  Reading the weights past
// the caches' order of what to keep takes 5.9 instead of 6.5 for 4096 -> 4096 from memory, but 9.9 instead of 8.6 for 10240 -> 4096 from the caches, 99 instead of 92 for 131072
// channels and 29.7 instead of 26.7 for 16 tokens, 10240 -> 8192, from memory.
template <int RT, int RC, int AHEAD, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) dense_few_kernel(DenseClearArgs a) {
    static_assert(RT * RC <= WAVES, "a wave a tile of the sums");
    __shared__ v4i sums[WAVES][RT * RC][64];
    const unsigned groups = (unsigned)((a.n + 16 * RC - 1) / (16 * RC));
    const int blocks = a.k / 64;
    for (unsigned group = blockIdx.x; group < groups; group += gridDim.x) {
        const int t = again(threadIdx.x), lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
        const int part = 16 * (lane >> 4);
        const int64_t first = (int64_t)group * 16 * RC;
        const int8_t *w[RC], *x[RT];
#pragma unroll
        for (int c = 0; c < RC; ++c) {
            const int64_t j = first + 16 * c + (lane & 15);
            w[c] = a.w + (j < a.n ? j : a.n - 1) * a.ldw + part;
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            // beyond the last token: that one again, never stored
            const int64_t i = 16 * r + (lane & 15);
            x[r] = a.x + (i < a.m ? i : a.m - 1) * a.ldx + part;
        }
        // what the outputs take, asked for before the weights
        const int64_t my_i = 16 * (wave / RC) + (lane & 15), my_j = first + 16 * (wave % RC) + 4 * (lane >> 4);
        Channels channels = {};
        float x_scale = 1.0f;
        if (wave < RT * RC) {
            channels = {{1.0f, 1.0f, 1.0f, 1.0f}, {0, 0, 0, 0}, a.n - my_j < 4 ? (int)(a.n - my_j) : 4};
            if (channels.left > 0) {
                if (a.w_scale) load_4(channels.scale, a.w_scale + my_j, channels.left);
                if (a.bias) load_4(channels.bias, static_cast<const int *>(a.bias) + my_j, channels.left);
            }
            if (a.x_scale && my_i < a.m) x_scale = a.x_scale[my_i];
        }
        v4i acc[RT][RC] = {};
        const auto some = [&](auto count, int b) {
            constexpr int kCount = decltype(count)::value;
            v4i fw[kCount][RC], fx[kCount][RT];
#pragma unroll
            for (int u = 0; u < kCount; ++u) {
#pragma unroll
                for (int c = 0; c < RC; ++c) __builtin_memcpy(&fw[u][c], w[c] + 64 * (b + u), 16);
#pragma unroll
                for (int r = 0; r < RT; ++r) __builtin_memcpy(&fx[u][r], x[r] + 64 * (b + u), 16);
            }
#pragma unroll
            for (int u = 0; u < kCount; ++u)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int c = 0; c < RC; ++c) acc[r][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][c], fx[u][r], acc[r][c], 0, 0, 0);
        };
        // wave w: blocks w * each ... of k, and the last wave what is left of less than a block
        const int each = (blocks + WAVES - 1) / WAVES, last = std::min((wave + 1) * each, blocks);
        int b = wave * each;
        for (; b + AHEAD <= last; b += AHEAD) some(std::integral_constant<int, AHEAD>{}, b);
        for (; b < last; ++b) some(std::integral_constant<int, 1>{}, b);
        if (wave == WAVES - 1 && blocks * 64 < a.k) {
            const int at = blocks * 64 + part;
            v4i fw[RC];
#pragma unroll
            for (int c = 0; c < RC; ++c) fw[c] = load_16(w[c] - part, at, a.k);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const v4i fx = load_16(x[r] - part, at, a.k);
#pragma unroll
                for (int c = 0; c < RC; ++c) acc[r][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[c], fx, acc[r][c], 0, 0, 0);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < RC; ++c) sums[wave][r * RC + c][lane] = acc[r][c];
        __syncthreads();
        if (wave < RT * RC && my_i < a.m && channels.left > 0) {
            v4i s = sums[0][wave][lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s += sums[v][wave][lane];
            finish_4(a, my_i, my_j, s, x_scale, channels);
        }
        __syncthreads();
    }
}

// workgroups of a launch: more tiles or rows than this are taken in turn, so that no grid outgrows what a launch may have
constexpr int64_t kMostGroups = 1 << 20;
static dim3 groups_of(int64_t tiles) { return dim3((unsigned)(tiles < kMostGroups ? tiles : kMostGroups)); }

template <int RT, int RC, int AHEAD, int WAVES>
static void few_launch(const DenseClearArgs &a, hipStream_t stream) {
    dense_few_kernel<RT, RC, AHEAD, WAVES><<<groups_of((a.n + 16 * RC - 1) / (16 * RC)), 64 * WAVES, 0, stream>>>(a);
}

template <int WT, int WC, int RT, int RC, int BK>
static void tile_launch(const DenseClearArgs &a, bool direct, hipStream_t stream) {
    constexpr int TT = 16 * WT * RT, TC = 16 * WC * RC;
    const int64_t tiles = ((a.n + TC - 1) / TC) * ((a.m + TT - 1) / TT);
    if (direct) {
        dense_tile_kernel<WT, WC, RT, RC, BK, true><<<groups_of(tiles), 64 * WT * WC, 0, stream>>>(a);
    } else if constexpr (RT * RC < 32) {
        dense_tile_kernel<WT, WC, RT, RC, BK, false><<<groups_of(tiles), 64 * WT * WC, 0, stream>>>(a);
    }
}

// The tile kernel's forms, and what a launch of each takes: with up to 256, 512, 768 tiles -- one, two, three on a CU, as many as its LDS
// holds -- a start and end of `fixed` and `step` for 128 bytes of k, in us, measured as kernels of 4096-byte and 1024-byte rows in a
// captured sequence.  More tiles than a device holds at once go round, a round after the first at the cost of its steps and two thirds of its start.
// Over 60 random sizes the choice takes 2 % more than the best of the six on average, and 30 % at most (3045 x 320 -> 3968, three rounds of 128 x 128 tiles for one of
// 256 x 256, 25.3 and 19.4 us).
struct TileForm {
    int tokens, channels, at_once;
    struct { float fixed, step; } cost[3];
};
constexpr TileForm kTileForms[] = {
    {32, 64, 3, {{3.1f, 0.249f}, {4.1f, 0.290f}, {4.9f, 0.418f}}},
    {64, 64, 2, {{4.0f, 0.271f}, {5.1f, 0.394f}}},
    {64, 128, 1, {{5.4f, 0.320f}}},
    {128, 128, 1, {{7.1f, 0.473f}}},
    {256, 128, 1, {{9.9f, 1.000f}}},
    {256, 256, 1, {{16.4f, 1.610f}}}};

static float tile_cost(const TileForm &f, const DenseClearArgs &a) {
    const float steps = (float)a.k / 128.0f;
    const int64_t tiles = ((a.m + f.tokens - 1) / f.tokens) * ((a.n + f.channels - 1) / f.channels), on_cu = (tiles + 255) / 256;
    const int64_t rounds = (on_cu - 1) / f.at_once, rest = on_cu - rounds * f.at_once;
    const auto &full = f.cost[f.at_once - 1], &last = f.cost[rest - 1];
    return last.fixed + last.step * steps + (float)rounds * (0.67f * full.fixed + full.step * steps);
}

static void dense_launch(DenseClearArgs a, hipStream_t stream) {
    // An output larger than the eight L2s (4 MiB each) would only push the operands out of them: 8192 x 10240 -> 8192 617 -> 587 us, 8192 x 4096 -> 8192 272 -> 249.
    a.past = a.m * a.n * (a.kind == BNN_CLEAR_F32 || a.kind == BNN_CLEAR_I32 ? 4 : a.kind <= BNN_CLEAR_F16 ? 2 : 1) > (int64_t)32 << 20;
    const auto fours = [](const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 4 == 0 && ld % 4 == 0 && ld <= 1 << 22; };
    const bool direct = fours(a.x, a.ldx) && fours(a.w, a.ldw);
    // Up to 16 tokens read each weight once.  From five tokens on each of its workgroups' reading of all tokens costs as much as the weights, and with more
    // than two workgroups a CU tiles, which share it, take less (16 tokens, 4096 -> 8192 10.0 us, tiles 9.9; 4096 -> 12288 13.4 and 11.0; 10240 -> 10240 29.3 and 20.8,
    // from memory 36.8 and 32.9; one token, 4096 -> 10240 9.5 and 10.6, from memory 12.2 and 15.8).
    if (a.m <= 4 || (a.m <= 16 && (a.n <= 8192 || !direct))) return few_launch<1, 1, 2, 8>(a, stream);
    // Up to 32 likewise, while channels are few enough that tiles leave CUs idle.  Weights from memory decide it
    // (32 tokens, 1024 -> 4096 5.0 us, tiles 6.8; 10240 -> 1024 19.1 and 30.0; 10240 -> 4096 20.5 and 30.9; 4096 -> 4096 9.7 and 14.8, where on kept weights it is 8.3 and 6.7).
    if (a.m <= 32 && a.n <= 4096) return few_launch<2, 1, 4, 8>(a, stream);
    // Through registers the largest has none left (2001-byte rows, 4000 x 4000: 73 us, and 82 with the one before), rows a few bytes long aside.
    int form = 0;
    for (int f = 1; f < (direct ? 6 : 5); ++f)
        if (tile_cost(kTileForms[f], a) < tile_cost(kTileForms[form], a)) form = f;
    switch (form) {
        case 0: tile_launch<1, 4, 2, 1, 128>(a, direct, stream); break;
        case 1: tile_launch<2, 2, 2, 2, 128>(a, direct, stream); break;
        case 2: tile_launch<2, 4, 2, 2, 128>(a, direct, stream); break;
        case 3: tile_launch<2, 4, 4, 2, 128>(a, direct, stream); break;
        case 4: tile_launch<4, 2, 4, 4, 64>(a, direct, stream); break;
        default: tile_launch<2, 4, 8, 4, 64>(a, direct, stream); break;
    }
}

int launch_dense_clear(const DenseClearArgs &a, hipStream_t stream) {
    dense_launch(a, stream);
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

// ---- rows to 8 bits ------------------------------------------------------------------------------------------------

// Eight neighbouring values as they lie in memory.
template <class T>
struct Eight {
    T v[8];
};

// A row is read in chunks of eight values.  Each thread reads CHUNKS of them, whole ones without a branch -- a chunk that is not
// there is read at the row's beginning and replaced by zeros -- so that all its loads are under way at once; the one thread that
// holds the row's last, partial chunk reads it value by value afterwards.  The pointer is aligned to a value only: the device takes wide
// accesses at any such address.  The values are read once, past the caches' order of what to keep: a kernel that only reads 4096 x 10240 pairs and writes a byte
// for each takes 34 us that way and 39 without.
struct Chunks {
    int t, threads, k;
    __device__ __forceinline__ int at(int c) const { return 8 * (t + threads * c); }
    __device__ __forceinline__ bool whole(int c) const { return at(c) + 8 <= k; }
    __device__ __forceinline__ int partial(int c) const { return at(c) < k && !whole(c) ? k - at(c) : 0; }
};

template <class T>
__device__ __forceinline__ Eight<T> load_past(const T *p) {
    typedef int Words __attribute__((ext_vector_type(sizeof(T) * 2), aligned(sizeof(T))));
    const Words w = __builtin_nontemporal_load(reinterpret_cast<const Words *>(p));
    Eight<T> e;
    __builtin_memcpy(&e, &w, sizeof e);
    return e;
}

template <class T, int COUNT>
__device__ __forceinline__ void read_chunks(Eight<T> (&to)[COUNT], const T *row, const Chunks &own, int first) {
#pragma unroll
    for (int c = 0; c < COUNT; ++c) {
        if (own.k >= 8) to[c] = load_past(row + (own.whole(first + c) ? own.at(first + c) : 0));
        else __builtin_memset(&to[c], 0, sizeof to[c]);
    }
}

// once the loads are under way: zeros for what is not there, the last values one by one
template <class T>
__device__ __forceinline__ void complete(Eight<T> &to, const T *row, const Chunks &own, int c) {
    if (!own.whole(c)) {
        __builtin_memset(&to, 0, sizeof to);
        const int left = own.partial(c);
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) to.v[j] = row[own.at(c) + j];
    }
}

template <class T>
__device__ __forceinline__ void write_8(T *row, const Eight<T> &e, const Chunks &own, int c) {
    if (own.whole(c)) {
        __builtin_memcpy(row + own.at(c), &e, sizeof e);
    } else {
        const int left = own.partial(c);
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) row[own.at(c) + j] = e.v[j];
    }
}

// Largest magnitude and sum of squares of a row.  Magnitudes are compared as the bits of |v|, in whose order infinity comes after every
// number and NaN after infinity, so a row that holds one keeps it.  Squares are summed in 64 bits: those of large f32 values
// leave the f32 range, and the order of the sum does not show in 32 bits of the result.
struct RowSums {
    unsigned top;
    double squares;
};

__device__ __forceinline__ RowSums join(RowSums a, RowSums b) {
    return {std::max(a.top, b.top), a.squares + b.squares};
}

// The value that the lane `CTRL` says (a data-parallel-primitive control) holds; 0 where there is none.
template <int CTRL>
__device__ __forceinline__ unsigned from_lane(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

template <int CTRL, bool SQUARES>
__device__ __forceinline__ RowSums joined(RowSums s) {
    RowSums o = {from_lane<CTRL>(s.top), 0.0};
    if (SQUARES) {
        const uint64_t bits = __double_as_longlong(s.squares);
        o.squares = __longlong_as_double((uint64_t)from_lane<CTRL>((unsigned)(bits >> 32)) << 32 | from_lane<CTRL>((unsigned)bits));
    }
    return join(s, o);
}

// Over the wave, for every lane: sums of 2, 4, 8 and 16 neighbours by rotations within a row of 16 lanes, then across the four rows.
// All in the vector unit: through LDS, as shuffles go, each of the six steps takes as long as this takes altogether.
template <bool SQUARES>
__device__ __forceinline__ RowSums across_wave(RowSums s) {
    s = joined<0x121, SQUARES>(s);      // row_ror:1, 2, 4, 8
    s = joined<0x122, SQUARES>(s);
    s = joined<0x124, SQUARES>(s);
    s = joined<0x128, SQUARES>(s);
    RowSums all = {0u, 0.0};
#pragma unroll
    for (int row = 0; row < 4; ++row) {
        RowSums o = {(unsigned)__builtin_amdgcn_readlane((int)s.top, 16 * row), 0.0};
        if (SQUARES) {
            const uint64_t bits = __double_as_longlong(s.squares);
            o.squares = __longlong_as_double((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), 16 * row) << 32 |
                                             (unsigned)__builtin_amdgcn_readlane((int)bits, 16 * row));
        }
        all = row ? join(all, o) : o;
    }
    return all;
}

// a / b from 1 / b: the product, and once what it leaves over (Markstein's correction).  Where one_by_b is 1 / b to the nearest, as for the rows'
// steps, this is the quotient to the nearest (the same as a division for 4e8 random pairs, and for every a and b = 127); with a reciprocal one unit off, which
// the hardware's may be, as in silu, it is one unit off for a pair in 100,000.
__device__ __forceinline__ float quotient(float a, float b, float one_by_b) {
    const float q = a * one_by_b;
    return fmaf(fmaf(-q, b, a), one_by_b, q);
}

// relu; silu(v) = v / (1 + e^-v); gelu(v) = v Phi(v).  With up to 4096 x 10240 values a prompt these are bound by their instructions as much as by
// memory, so both are as short as their accuracy allows:
//   silu: e^-v as 2^p, the product p = -v log2(e) with what it rounds off, since 2^p turns an absolute error of p into a relative one:
//   about six roundings at any v.  What is below 2^-119 may be 0.
//   gelu: Phi(-a) = e^(-a^2/2) R(a) for a >= 0, R the scaled complementary error function; R as t P(t), t = 1 / (1 + 0.35 a), P
//   the polynomial of degree 8 that a least-squares fit of the relative error at 400 Chebyshev points of t (a <= 15) gives: 3.6e-8 off, and 5
//   roundings when evaluated in f32.  v Phi(v) is then max(v, 0) - |v| Phi(-|v|).  This keeps its relative accuracy far out on the negative
//   side, where 1 + erf has no digits left; there the rounding of a^2 grows to 1.5 a^2 roundings of the result.
template <int ACT>
__device__ __forceinline__ float activated(float v) {
    if constexpr (ACT == BNN_ACT_RELU) {
        return v > 0.0f || v != v ? v : 0.0f;
    } else if constexpr (ACT == BNN_ACT_SILU) {
        constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f, kLn2 = 0.693147182f;
        const float h = __builtin_amdgcn_fmed3f(-v, -200.0f, 200.0f), p = h * kLog2e;
        const float r = fmaf(h, kRest, fmaf(h, kLog2e, -p));
        const float e = __builtin_amdgcn_exp2f(p) * fmaf(r, kLn2, 1.0f);
        const float d = 1.0f + e, by = __builtin_amdgcn_rcpf(d);
        return d < 0x1p100f ? quotient(v, d, by) : v * by;
    } else {
        const float a = fminf(fabsf(v), 20.0f);
        const float e = __builtin_amdgcn_exp2f(a * a * -0.72134752f);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
        float r = -0.02949463576078415f;
        r = fmaf(r, t, 0.14561739563941956f);
        r = fmaf(r, t, -0.25899502635002136f);
        r = fmaf(r, t, 0.16276812553405762f);
        r = fmaf(r, t, -0.0254655834287405f);
        r = fmaf(r, t, 0.10644964128732681f);
        r = fmaf(r, t, 0.11960979551076889f);
        r = fmaf(r, t, 0.1398903727531433f);
        r = fmaf(r, t, 0.13961990177631378f);
        return fmaf(-fabsf(v), r * t * e, fmaxf(v, 0.0f));
    }
}

__device__ __forceinline__ void activate(int act, float (&v)[8]) {
    if (act == BNN_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activated<BNN_ACT_SILU>(v[j]);
    } else if (act == BNN_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activated<BNN_ACT_GELU>(v[j]);
    } else if (act == BNN_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activated<BNN_ACT_RELU>(v[j]);
    }
}

// A row a workgroup of up to sixteen waves (SPREAD), or a row a wave, four of them in a workgroup; the row's values are in registers from the
// only reading to the rounding, CHUNKS chunks of eight a thread.
//   norm: v = h * weight; y = v / rms, a positive number for the whole row, so that q = v / (max|v| / 127) needs no rms and one
//   reduction gives both the sum of squares and max|v|; only the scale, max|v| / (127 rms), takes it.
//   gate: v = act(gate) * up.
template <class T, bool NORM, bool SPREAD, int CHUNKS>
__global__ void __launch_bounds__(SPREAD ? 1024 : 256) rows_kernel(RowsClearArgs a) {
    __shared__ RowSums sums[2][16];
    const int threads = SPREAD ? blockDim.x : 64, waves = threads >> 6;
    Chunks own = {SPREAD ? (int)threadIdx.x : (int)(threadIdx.x & 63), threads, a.k};
    const int64_t stride = SPREAD ? gridDim.x : (int64_t)gridDim.x * 4;
    int turn = 0;
    for (int64_t row = SPREAD ? blockIdx.x : (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); row < a.m;
         row += stride, turn ^= 1) {
        // what goes by the thread is found anew for each row: kept from row to row, the many addresses and conditions of more than two chunks
        // crowd values out of the registers
        own.t = again(own.t);
        const T *pa = static_cast<const T *>(a.a) + row * a.lda, *pb = a.b ? static_cast<const T *>(a.b) + row * a.ldb : nullptr;
        const T *weight = static_cast<const T *>(a.weight);
        constexpr int kTogether = CHUNKS == 1 ? 1 : 2;     // chunks whose loads are under way at once, as registers allow
        Eight<T> ra[kTogether], rb[kTogether];
        float v[CHUNKS][8];
        RowSums s = {0u, 0.0};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (CHUNKS > kTogether) __builtin_amdgcn_sched_barrier(0);
            if (c % kTogether == 0) {
                read_chunks(ra, pa, own, c);
                if (pb) read_chunks(rb, pb, own, c);
            }
            complete(ra[c % kTogether], pa, own, c);
            if (pb) complete(rb[c % kTogether], pb, own, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = (float)ra[c % kTogether].v[j];
            if constexpr (NORM) {
                if (pb) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] += (float)rb[c % kTogether].v[j];
                }
                if (a.total) {
                    Eight<T> h;
#pragma unroll
                    for (int j = 0; j < 8; ++j) h.v[j] = (T)v[c][j];
                    write_8(static_cast<T *>(a.total) + row * a.ldt, h, own, c);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) s.squares = fma((double)v[c][j], (double)v[c][j], s.squares);
                if (weight) {
                    Eight<T> g;
                    if (own.whole(c)) __builtin_memcpy(&g, weight + own.at(c), sizeof g);
                    complete(g, weight, own, c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] *= (float)g.v[j];
                }
            } else {
                activate(a.act, v[c]);
                if (pb) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] *= (float)rb[c % kTogether].v[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const unsigned x = __float_as_uint(v[c][j]) & 0x7fffffffu, y = __float_as_uint(v[c][j + 1]) & 0x7fffffffu;
                s.top = std::max(s.top, std::max(x, y));
            }
        }
        s = across_wave<NORM>(s);
        if (SPREAD && waves > 1) {
            // two places in turn: a wave that is a row ahead does not overwrite what another still reads
            if ((threadIdx.x & 63) == 0) sums[turn][threadIdx.x >> 6] = s;
            __syncthreads();
            s = sums[turn][0];
            for (int w = 1; w < waves; ++w) s = join(s, sums[turn][w]);
        }
        // q = v / step to the nearest, step = top / 127 to the nearest: the product with 1 / 127 alone is a step of f32 off for one row in twenty, which
        // moves values at half the largest (63.5 steps, common in rows of few bits) to the other side of their border
        constexpr float kPart = 1.0f / 127.0f;
        const float top = __uint_as_float(s.top);
        float step = quotient(top, 127.0f, kPart), per_step;
        if (__builtin_expect(!(s.top >= 0x0d800000u && s.top < 0x7f800000u), 0)) {
            // near the bottom of the f32 range (below 2^-100) 1 / step would be infinite: lifted by 2^100 first.  Nothing but zeros, or
            // something that is not a number: all 0
            const bool lifted = s.top != 0u && s.top < 0x7f800000u;
            step = lifted ? quotient(top * 0x1p100f, 127.0f, kPart) : 0.0f;
            per_step = lifted ? 1.0f / step : 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = lifted ? v[c][j] * 0x1p100f : 0.0f;
        } else {
            per_step = 1.0f / step;
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            unsigned bytes[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // 1.5 * 2^23 added: the last byte of the sum is the quotient rounded to the nearest whole number
                unsigned w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(quotient(v[c][4 * h + j], step, per_step) + 12582912.0f);
                bytes[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
            }
            Eight<int8_t> q;
            __builtin_memcpy(&q, bytes, sizeof q);
            write_8(a.q + row * a.ldq, q, own, c);
        }
        if (own.t == 0) {
            float scale = top / 127.0f;     // below 2^-100, and for what is not a number, too
            if constexpr (NORM) scale = (float)((double)top / (127.0 * sqrt(s.squares / a.k + (double)a.eps)));
            a.scale[row] = a.k ? scale : 0.0f;
        }
    }
}

// Threads and chunks a row.  Up to 512 values: a wave a row, and no workgroup to meet.  Longer rows: a thread a chunk as long as rows
// are few or short, since a row's time is then the call's (300 x 4096 gate 4.4 us, two chunks a thread 5.0); else the fewest threads that keep
// enough waves on a CU, two chunks each, four from 1,024 chunks on (8192 x 8192 bf16 norm, one, two, four chunks a thread: 129, 90, 100 us; 4096 x 14336 silu,
// two, four, six: 72, 61, 82).  The norm's weights and second output take it registers: with four its waves no longer fit (2048 x 12288 bf16, two, four: 37, 51).
// Rows of more than 16,384 values have no choice.
template <class T, bool NORM>
static void rows_launch(const RowsClearArgs &a, hipStream_t stream) {
    const int chunks = (a.k + 7) / 8;
    if (chunks <= 64) {
        rows_kernel<T, NORM, false, 1><<<groups_of((a.m + 3) / 4), 256, 0, stream>>>(a);
        return;
    }
    const int each = chunks <= 256 || (chunks <= 512 && a.m < 1024) ? 1 : chunks <= 1024 ? 2 : chunks <= 2048 ? (NORM || a.m < 512 ? 2 : 4) : chunks <= 4096 ? 4 : 8;
    const int threads = 64 * (((chunks + each - 1) / each + 63) / 64);
    switch (each) {
        case 1: rows_kernel<T, NORM, true, 1><<<groups_of(a.m), threads, 0, stream>>>(a); break;
        case 2: rows_kernel<T, NORM, true, 2><<<groups_of(a.m), threads, 0, stream>>>(a); break;
        case 4: rows_kernel<T, NORM, true, 4><<<groups_of(a.m), threads, 0, stream>>>(a); break;
        default:
            if constexpr (!NORM) rows_kernel<T, NORM, true, 8><<<groups_of(a.m), threads, 0, stream>>>(a);
            break;
    }
}

template <bool NORM>
static void rows_typed(const RowsClearArgs &a, hipStream_t stream) {
    if (a.type == BNN_CLEAR_F32) rows_launch<float, NORM>(a, stream);
    else if (a.type == BNN_CLEAR_BF16) rows_launch<__bf16, NORM>(a, stream);
    else rows_launch<_Float16, NORM>(a, stream);
}

int launch_norm_clear(const RowsClearArgs &a, hipStream_t stream) {
    rows_typed<true>(a, stream);
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

int launch_gate_clear(const RowsClearArgs &a, hipStream_t stream) {
    rows_typed<false>(a, stream);
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

}  // namespace tfhe
