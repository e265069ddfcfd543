// gfx950 kernels of layers in the clear: the 8-bit matrix product, and the two row operators that feed it (norm, gated activation).
#include "clear_kernels.h"

#include <algorithm>

namespace tfhe {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

// ---- the product ---------------------------------------------------------------------------------------------------

// 16 bytes of a row from byte `at` on, of which only those before `k` count: the rest is 0 and not read.
__device__ __forceinline__ v4i load_16(const int8_t *row, int at, int k) {
    v4i v = {0, 0, 0, 0};
    if (at + 16 <= k) {
        __builtin_memcpy(&v, row + at, 16);
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

template <class T>
__device__ __forceinline__ void store_4(T *p, const T (&v)[4], int left) {
    if (left == 4) {
        __builtin_memcpy(p, v, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) p[e] = v[e];
    }
}

// The outputs of four neighbouring channels of token i, j .. j + 3, of which those below n exist, from their sums.
__device__ __forceinline__ void finish_4(const DenseClearArgs &a, int64_t i, int64_t j, v4i acc) {
    const int left = a.n - j < 4 ? (int)(a.n - j) : 4;
    const int64_t at = i * a.ldo + j;
    if (a.kind >= BNN_CLEAR_I32) {
        int b[4] = {0, 0, 0, 0};
        if (a.bias) load_4(b, static_cast<const int *>(a.bias) + j, left);
        if (a.kind == BNN_CLEAR_I32) {
            int o[4];
            for (int e = 0; e < 4; ++e) o[e] = (int)((unsigned)acc[e] + (unsigned)b[e]);
            store_4(static_cast<int *>(a.out) + at, o, left);
        } else {
            const int8_t no = a.kind == BNN_CLEAR_SIGN ? -1 : 0;
            int8_t o[4];
            for (int e = 0; e < 4; ++e) o[e] = (int64_t)acc[e] + b[e] >= 0 ? (int8_t)1 : no;
            store_4(static_cast<int8_t *>(a.out) + at, o, left);
        }
        return;
    }
    float sw[4] = {1.0f, 1.0f, 1.0f, 1.0f}, b[4] = {0.0f, 0.0f, 0.0f, 0.0f}, y[4];
    const float sx = a.x_scale ? a.x_scale[i] : 1.0f;
    if (a.w_scale) load_4(sw, a.w_scale + j, left);
    if (a.bias) load_4(b, static_cast<const float *>(a.bias) + j, left);
    for (int e = 0; e < 4; ++e) y[e] = (float)acc[e] * sx * sw[e] + b[e];
    if (a.kind == BNN_CLEAR_F32) {
        store_4(static_cast<float *>(a.out) + at, y, left);
    } else if (a.kind == BNN_CLEAR_BF16) {
        __bf16 o[4];
        for (int e = 0; e < 4; ++e) o[e] = (__bf16)y[e];
        store_4(static_cast<__bf16 *>(a.out) + at, o, left);
    } else {
        _Float16 o[4];
        for (int e = 0; e < 4; ++e) o[e] = (_Float16)y[e];
        store_4(static_cast<_Float16 *>(a.out) + at, o, left);
    }
}

// Waits until at most `left` of the wave's loads into LDS are under way and its reads of LDS have come, then meets the workgroup.
template <int left>
__device__ __forceinline__ void landed_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(left) : "memory");
}

// Tiles of (WT * RT * 32) tokens by (WC * RC * 32) channels, a workgroup of WT x WC waves each, every wave RT x RC products of 32 by 32.
// 128 bytes of k at a time go through LDS, the next 128 under way while these are multiplied.  A row's eight 16-byte pieces lie in
// LDS at place (piece ^ row % 8), so that the eight lanes that read one piece of eight rows meet all banks.
// The channels are the products' rows: a lane then holds four neighbouring channels of a token.
//   ALIGNED: rows begin at multiples of 16 bytes and k is one too; pieces go from memory to LDS directly.  Otherwise through registers.
template <int WT, int WC, int RT, int RC, bool ALIGNED>
__global__ void __launch_bounds__(64 * WT * WC, 2) dense_tile_kernel(DenseClearArgs a) {
    constexpr int kThreads = 64 * WT * WC, kWaves = WT * WC, TT = 32 * WT * RT, TC = 32 * WC * RC;
    constexpr int kPieces = (TT + TC) * 8 / kThreads;       // of 16 bytes, a thread
    constexpr int kXPieces = TT * 8 / kThreads;
    constexpr int kRow = 32 * RC + 4;                       // words of a token's channels as the sums pass through LDS
    static_assert(kWaves * 32 * kRow * 4 <= 2 * (TT + TC) * 128, "the sums pass through the operands' LDS");
    static_assert(kXPieces * kThreads == TT * 8 && kPieces * kThreads == (TT + TC) * 8, "whole pieces a thread");
    __shared__ __attribute__((aligned(1024))) int8_t lds[2][(TT + TC) * 128];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t across = (a.n + TC - 1) / TC, down = (a.m + TT - 1) / TT, tiles = across * down;
    const int steps = (a.k + 127) / 128;
    for (int64_t id = blockIdx.x; id < tiles; id += gridDim.x) {
        // Workgroups go round the eight XCDs; each XCD gets neighbouring tiles, four token tiles by all channels at a time, so that
        // its L2 is asked for the same rows.
        const int64_t xcd = id & 7, share = tiles >> 3, over = tiles & 7;
        const int64_t lin = xcd * share + (xcd < over ? xcd : over) + (id >> 3);
        const int64_t band = lin / (4 * across), in_band = lin - band * 4 * across, first = band * 4, high = down - first < 4 ? down - first : 4;
        const int64_t i0 = (first + in_band % high) * TT, j0 = in_band / high * TC;

        // piece p of a thread: row p * kThreads / 8 + t / 8 of the tile's tokens, then of its channels
        const int place = t & 7, row8 = t >> 3, piece = place ^ (row8 & 7);
        const int8_t *row[kPieces];
        int offset[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const bool is_x = p < kXPieces;
            const int64_t r = (is_x ? i0 : j0) + (p - (is_x ? 0 : kXPieces)) * (kThreads / 8) + row8, rows = is_x ? a.m : a.n;
            const int64_t kept = r < rows ? r : rows - 1;       // beyond the last row: that row again, never stored
            if (ALIGNED) offset[p] = (int)((kept - (is_x ? i0 : j0)) * (is_x ? a.ldx : a.ldw)) + 16 * piece;
            else row[p] = is_x ? a.x + kept * a.ldx : a.w + kept * a.ldw;
        }
        const int64_t x_end = ((a.m - i0 < TT ? a.m - i0 : TT) - 1) * a.ldx + a.k, w_end = ((a.n - j0 < TC ? a.n - j0 : TC) - 1) * a.ldw + a.k;
        const auto xr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.x + i0 * a.ldx), (short)0, (int)x_end, 0x00020000);
        const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + j0 * a.ldw), (short)0, (int)w_end, 0x00020000);
        v4i held[ALIGNED ? 1 : kPieces];
        const auto fetch = [&](int s, int8_t *to) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                if constexpr (ALIGNED) {
                    // a piece beyond k: an offset beyond the buffer, which reads as 0
                    const int at = 128 * s + 16 * piece < a.k ? offset[p] : (int)0x80000000;
                    const auto lds_at = (__attribute__((address_space(3))) void *)(to + p * 16 * kThreads + 1024 * wave);
                    if (p < kXPieces) __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, lds_at, 16, at, 128 * s, 0, 0);
                    else __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, lds_at, 16, at, 128 * s, 0, 0);
                } else {
                    held[p] = load_16(row[p], 128 * s + 16 * piece, a.k);
                }
            }
        };
        const auto settle = [&](int8_t *to) {
            if constexpr (!ALIGNED) {
#pragma unroll
                for (int p = 0; p < kPieces; ++p) *reinterpret_cast<v4i *>(to + (p * kThreads + t) * 16) = held[p];
            }
        };

        v16i acc[RT][RC] = {};
        const int at_x = (wave / WC) * 32 * RT + (lane & 31), at_w = TT + (wave % WC) * 32 * RC + (lane & 31);
        if (steps > 0) {
            fetch(0, lds[0]);
            settle(lds[0]);
        }
        landed_and_meet<0>();
        for (int s = 0; s < steps; ++s) {
            const int8_t *from = lds[s & 1];
            if (s + 1 < steps) fetch(s + 1, lds[(s + 1) & 1]);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int where = 16 * ((2 * kk + (lane >> 5)) ^ (lane & 7));
                v4i fx[RT], fw[RC];
#pragma unroll
                for (int r = 0; r < RT; ++r) fx[r] = *reinterpret_cast<const v4i *>(from + (at_x + 32 * r) * 128 + where);
#pragma unroll
                for (int c = 0; c < RC; ++c) fw[c] = *reinterpret_cast<const v4i *>(from + (at_w + 32 * c) * 128 + where);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int c = 0; c < RC; ++c) acc[r][c] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[c], fx[r], acc[r][c], 0, 0, 0);
            }
            if (s + 1 < steps) settle(lds[(s + 1) & 1]);
            landed_and_meet<0>();
        }
        // The wave's sums go through LDS of its own, 32 tokens at a time, so that its stores are whole stretches of a token's channels.
        int *own = reinterpret_cast<int *>(&lds[0][0]) + wave * 32 * kRow;
        const int64_t wave_i = i0 + (wave / WC) * 32 * RT, wave_j = j0 + (wave % WC) * 32 * RC;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
            for (int c = 0; c < RC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v4i four = {acc[r][c][4 * e], acc[r][c][4 * e + 1], acc[r][c][4 * e + 2], acc[r][c][4 * e + 3]};
                    *reinterpret_cast<v4i *>(own + (lane & 31) * kRow + 32 * c + 8 * e + 4 * (lane >> 5)) = four;
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int at = lane; at < 32 * 8 * RC; at += 64) {
                const int64_t i = wave_i + 32 * r + at / (8 * RC), j = wave_j + 4 * (at % (8 * RC));
                if (i < a.m && j < a.n) finish_4(a, i, j, *reinterpret_cast<const v4i *>(own + at / (8 * RC) * kRow + 4 * (at % (8 * RC))));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
    }
}

// Few tokens (up to 16 RT): the weights are read once and that is what it costs.  A workgroup takes 16 channels, its eight waves
// 64-byte blocks of k in turn; the weights go from memory to the products' registers without LDS, the waves' sums meet there.
template <int RT>
__global__ void __launch_bounds__(512) dense_few_kernel(DenseClearArgs a) {
    constexpr int kWaves = 8, kAhead = RT == 1 ? 8 : 4;
    __shared__ v4i sums[kWaves][RT][64];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t groups = (a.n + 15) / 16;
    const int blocks = a.k / 64, part = 16 * (lane >> 4);
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t j = group * 16 + (lane & 15), kept = j < a.n ? j : a.n - 1;
        const int8_t *w = a.w + kept * a.ldw + part;
        const int8_t *x[RT];
        for (int r = 0; r < RT; ++r) {
            const int64_t i = 16 * r + (lane & 15);
            x[r] = i < a.m ? a.x + i * a.ldx + part : nullptr;
        }
        v4i acc[RT] = {};
        // wave w: blocks w * each ... of k, and the last wave what is left of less than a block
        const int each = (blocks + kWaves - 1) / kWaves, last = (wave + 1) * each < blocks ? (wave + 1) * each : blocks;
        for (int b = wave * each; b < last; b += kAhead) {
            v4i fw[kAhead], fx[kAhead][RT];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int at = 64 * (b + u < last ? b + u : last - 1);
                __builtin_memcpy(&fw[u], w + at, 16);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    fx[u][r] = v4i{0, 0, 0, 0};
                    if (x[r] && b + u < last) __builtin_memcpy(&fx[u][r], x[r] + at, 16);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u][r], acc[r], 0, 0, 0);
        }
        if (wave == kWaves - 1 && blocks * 64 < a.k) {
            const int at = blocks * 64 + part;
            const v4i fw = load_16(w - part, at, a.k);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const v4i fx = x[r] ? load_16(x[r] - part, at, a.k) : v4i{0, 0, 0, 0};
                acc[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, fx, acc[r], 0, 0, 0);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) sums[wave][r][lane] = acc[r];
        __syncthreads();
        if (t < 64 * RT) {
            const int r = t >> 6;
            v4i s = sums[0][r][lane];
            for (int v = 1; v < kWaves; ++v) s += sums[v][r][lane];
            const int64_t i = 16 * r + (lane & 15), first = group * 16 + 4 * (lane >> 4);
            if (i < a.m && first < a.n) finish_4(a, i, first, s);
        }
        __syncthreads();
    }
}

// workgroups of a launch: more tiles or rows than this are taken in turn, so that no grid outgrows what a launch may have
constexpr int64_t kMostGroups = 1 << 20;
static dim3 groups_of(int64_t tiles) { return dim3((unsigned)(tiles < kMostGroups ? tiles : kMostGroups)); }

template <int WT, int WC, int RT, int RC>
static void tile_launch(const DenseClearArgs &a, bool aligned, hipStream_t stream) {
    const int64_t tiles = ((a.n + 32 * WC * RC - 1) / (32 * WC * RC)) * ((a.m + 32 * WT * RT - 1) / (32 * WT * RT));
    if (aligned) dense_tile_kernel<WT, WC, RT, RC, true><<<groups_of(tiles), 64 * WT * WC, 0, stream>>>(a);
    else dense_tile_kernel<WT, WC, RT, RC, false><<<groups_of(tiles), 64 * WT * WC, 0, stream>>>(a);
}

static void dense_launch(const DenseClearArgs &a, hipStream_t stream) {
    // FORM-BEGIN
    const auto sixteen = [](const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 16 == 0 && ld <= 1 << 22; };
    const bool aligned = a.k % 16 == 0 && sixteen(a.x, a.ldx) && sixteen(a.w, a.ldw);
    const auto tiles = [&](int64_t side) { return ((a.m + side - 1) / side) * ((a.n + side - 1) / side); };
    int form = a.m <= 16 ? 1 : a.m <= 32 ? 2 : a.m <= 64 ? 3 : tiles(256) >= 192 ? 6 : tiles(128) >= 192 ? 5 : 4;
    // FORM-END
    switch (form) {
        case 1: dense_few_kernel<1><<<groups_of((a.n + 15) / 16), 512, 0, stream>>>(a); break;
        case 2: dense_few_kernel<2><<<groups_of((a.n + 15) / 16), 512, 0, stream>>>(a); break;
        case 3: dense_few_kernel<4><<<groups_of((a.n + 15) / 16), 512, 0, stream>>>(a); break;
        case 4: tile_launch<2, 2, 1, 1>(a, aligned, stream); break;
        case 5: tile_launch<2, 2, 2, 2>(a, aligned, stream); break;
        default: tile_launch<2, 4, 4, 2>(a, aligned, stream); break;
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
// accesses at any such address.  The values are read once, past the caches' order of what to keep: 4096 x 10240 pairs in 34 us instead of 39.
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

// relu; silu(v) = v / (1 + e^-v); gelu(v) = v Phi(v).  With up to 4096 x 10240 values a prompt these are bound by their instructions as much as by
// memory, so both are as short as their accuracy allows:
//   silu: e^-v as 2^p, the product p = -v log2(e) with what it rounds off, since 2^p turns an absolute error of p into a relative one:
//   about eight roundings at any v.  What is below 2^-119 may be 0.
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
        return v * __builtin_amdgcn_rcpf(1.0f + e);
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
//   norm: v = h * weight; y = v / rms, a positive number for the whole row, so that q = 127 v / max|v| needs no rms and one
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
        asm volatile("" : "+v"(own.t));
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
        // q = 127 v / top
        const float top = __uint_as_float(s.top);
        float steps = 127.0f / top;
        if (__builtin_expect(!(s.top >= 0x0d800000u && s.top < 0x7f800000u), 0)) {
            if (s.top != 0u && s.top < 0x7f800000u) {
                // near the bottom of the f32 range (below 2^-100) 127 / top would be infinite: lifted by 2^100 first
                steps = 127.0f / (top * 0x1p100f);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] *= 0x1p100f;
            } else {
                // nothing but zeros, or something that is not a number
                steps = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] = 0.0f;
            }
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            unsigned bytes[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // 1.5 * 2^23 added: the last byte of the sum is the product rounded to the nearest whole number, once
                unsigned w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(fmaf(v[c][4 * h + j], steps, 12582912.0f));
                bytes[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
            }
            Eight<int8_t> q;
            __builtin_memcpy(&q, bytes, sizeof q);
            write_8(a.q + row * a.ldq, q, own, c);
        }
        if (own.t == 0) {
            double scale = (double)top / 127.0;
            if (NORM) scale /= sqrt(s.squares / a.k + (double)a.eps);
            a.scale[row] = a.k ? (float)scale : 0.0f;
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
    int each = chunks <= 256 || (chunks <= 512 && a.m < 1024) ? 1 : chunks <= 1024 ? 2 : chunks <= 2048 ? (NORM || a.m < 512 ? 2 : 4) : chunks <= 4096 ? 4 : 8;
    // ROWS
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
