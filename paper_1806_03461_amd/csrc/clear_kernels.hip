// gfx950 kernels of layers in the clear: the 8-bit matrix product, and the two row operators that feed it (norm, gated activation).
#include "clear_kernels.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace tfhe {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

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

template <int KIND>
__device__ __forceinline__ void store_out(const DenseClearArgs &a, int64_t i, int64_t j, int acc) {
    const int64_t at = i * a.ldo + j;
    if constexpr (KIND >= BNN_CLEAR_I32) {
        const int b = a.bias ? static_cast<const int *>(a.bias)[j] : 0;
        if constexpr (KIND == BNN_CLEAR_I32) {
            static_cast<int *>(a.out)[at] = (int)((unsigned)acc + (unsigned)b);
        } else {
            const bool one = (int64_t)acc + b >= 0;
            if constexpr (KIND == BNN_CLEAR_SIGN) static_cast<int8_t *>(a.out)[at] = one ? 1 : -1;
            else static_cast<uint8_t *>(a.out)[at] = one;
        }
    } else {
        float y = (float)acc;
        if (a.x_scale) y *= a.x_scale[i];
        if (a.w_scale) y *= a.w_scale[j];
        if (a.bias) y += static_cast<const float *>(a.bias)[j];
        if constexpr (KIND == BNN_CLEAR_F32) static_cast<float *>(a.out)[at] = y;
        else if constexpr (KIND == BNN_CLEAR_BF16) static_cast<__hip_bfloat16 *>(a.out)[at] = __float2bfloat16(y);
        else static_cast<__half *>(a.out)[at] = __float2half(y);
    }
}

// 64 tokens by 64 channels a workgroup of four waves, each 32 by 32; 64 bytes of k at a time through LDS.
template <int KIND>
__global__ void __launch_bounds__(256) dense_tile_kernel(DenseClearArgs a) {
    __shared__ v4i xs[64][5], ws[64][5];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t across = (a.n + 63) / 64, tiles = across * ((a.m + 63) / 64);
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t i0 = tile / across * 64, j0 = tile % across * 64;
        const int row = t >> 2, part = t & 3;
        const int64_t xi = i0 + row < a.m ? i0 + row : a.m - 1, wj = j0 + row < a.n ? j0 + row : a.n - 1;
        v4i acc[2][2] = {};
        for (int k0 = 0; k0 < a.k; k0 += 64) {
            const v4i x = load_16(a.x + xi * a.ldx, k0 + 16 * part, a.k), w = load_16(a.w + wj * a.ldw, k0 + 16 * part, a.k);
            __syncthreads();
            xs[row][part] = x;
            ws[row][part] = w;
            __syncthreads();
            v4i fx[2], fw[2];
            for (int r = 0; r < 2; ++r) {
                fx[r] = xs[(wave >> 1) * 32 + 16 * r + (lane & 15)][lane >> 4];
                fw[r] = ws[(wave & 1) * 32 + 16 * r + (lane & 15)][lane >> 4];
            }
            for (int r = 0; r < 2; ++r)
                for (int c = 0; c < 2; ++c) acc[r][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[c], fx[r], acc[r][c], 0, 0, 0);
        }
        for (int r = 0; r < 2; ++r)
            for (int c = 0; c < 2; ++c)
                for (int e = 0; e < 4; ++e) {
                    const int64_t i = i0 + (wave >> 1) * 32 + 16 * r + (lane & 15);
                    const int64_t j = j0 + (wave & 1) * 32 + 16 * c + 4 * (lane >> 4) + e;
                    if (i < a.m && j < a.n) store_out<KIND>(a, i, j, acc[r][c][e]);
                }
        __syncthreads();
    }
}

// workgroups of a launch: more tiles or rows than this are taken in turn, so that no grid outgrows what a launch may have
constexpr int64_t kMostGroups = 1 << 20;

template <int KIND>
static void dense_launch(const DenseClearArgs &a, hipStream_t stream) {
    const int64_t tiles = ((a.n + 63) / 64) * ((a.m + 63) / 64);
    dense_tile_kernel<KIND><<<dim3((unsigned)(tiles < kMostGroups ? tiles : kMostGroups)), 256, 0, stream>>>(a);
}

int launch_dense_clear(const DenseClearArgs &a, hipStream_t stream) {
    switch (a.kind) {
        case BNN_CLEAR_F32: dense_launch<BNN_CLEAR_F32>(a, stream); break;
        case BNN_CLEAR_BF16: dense_launch<BNN_CLEAR_BF16>(a, stream); break;
        case BNN_CLEAR_F16: dense_launch<BNN_CLEAR_F16>(a, stream); break;
        case BNN_CLEAR_I32: dense_launch<BNN_CLEAR_I32>(a, stream); break;
        case BNN_CLEAR_SIGN: dense_launch<BNN_CLEAR_SIGN>(a, stream); break;
        default: dense_launch<BNN_CLEAR_BITS>(a, stream); break;
    }
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

// ---- rows to 8 bits ------------------------------------------------------------------------------------------------

// Eight neighbouring values of a row, `left` of which exist (those beyond are 0 and not touched).  The pointer is aligned to an
// element only; the device takes wide accesses at any such address.
template <class T>
struct Eight {
    T v[8];
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__hip_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f32(float v, float &o) { o = v; }
__device__ __forceinline__ void from_f32(float v, __hip_bfloat16 &o) { o = __float2bfloat16(v); }
__device__ __forceinline__ void from_f32(float v, __half &o) { o = __float2half(v); }

template <class T>
__device__ __forceinline__ void load_8(const T *p, int left, float (&out)[8]) {
    if (left >= 8) {
        Eight<T> e;
        __builtin_memcpy(&e, p, sizeof e);
        for (int j = 0; j < 8; ++j) out[j] = to_f32(e.v[j]);
    } else {
        for (int j = 0; j < 8; ++j) out[j] = j < left ? to_f32(p[j]) : 0.0f;
    }
}

template <class T>
__device__ __forceinline__ void store_8(T *p, int left, const float (&in)[8]) {
    if (left >= 8) {
        Eight<T> e;
        for (int j = 0; j < 8; ++j) from_f32(in[j], e.v[j]);
        __builtin_memcpy(p, &e, sizeof e);
    } else {
        for (int j = 0; j < 8; ++j)
            if (j < left) from_f32(in[j], p[j]);
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
    return {a.top > b.top ? a.top : b.top, a.squares + b.squares};
}

template <bool SQUARES>
__device__ __forceinline__ RowSums across_wave(RowSums s) {
    for (int step = 1; step < 64; step <<= 1) {
        RowSums o = {__shfl_xor(s.top, step), 0.0};
        if (SQUARES) o.squares = __shfl_xor(s.squares, step);
        s = join(s, o);
    }
    return s;
}

// e^(hi + lo) to about three roundings: the product with log2(e) keeps what it rounds off, since 2^p turns an absolute error of p into a
// relative one.  Results below 2^-126 may be 0.
__device__ __forceinline__ float exp_of(float hi, float lo) {
    constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f, kLn2 = 0.693147182f;
    const float p = hi * kLog2e;
    const float r = fmaf(hi, kLog2e, -p) + fmaf(hi, kRest, lo * kLog2e);
    return __builtin_amdgcn_exp2f(p) * fmaf(r, kLn2, 1.0f);
}

// silu(v) = v / (1 + e^-v), from e^-|v| so that nothing overflows.
// gelu(v) = v Phi(v).  Phi(-a) = e^(-a^2/2) R(a) for a >= 0, R the scaled complementary error function; R as t P(t), t = 1 / (1 + 0.35 a), P
// the polynomial of degree 8 that a least-squares fit of the relative error at 400 Chebyshev points of t (a <= 15) gives: 3.6e-8 off, and 5 roundings in
// all when evaluated in f32.  The form keeps its relative accuracy far out on the negative side, where 1 + erf has no digits left.
template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if constexpr (ACT == BNN_ACT_RELU) {
        return v > 0.0f || v != v ? v : 0.0f;
    } else if constexpr (ACT == BNN_ACT_SILU) {
        const float e = exp_of(-fminf(fabsf(v), 200.0f), 0.0f);
        return v * ((v < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e));
    } else if constexpr (ACT == BNN_ACT_GELU) {
        const float a = fminf(fabsf(v), 20.0f), s = a * a;
        const float e = exp_of(-0.5f * s, -0.5f * fmaf(a, a, -s));
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
        const float phi = r * t * e;
        return v * (v < 0.0f ? phi : 1.0f - phi);
    } else {
        return v;
    }
}

// One row a workgroup of THREADS (a wave a row, four rows a workgroup, for THREADS = 64), its values in registers from the only
// reading to the rounding: CHUNKS chunks of eight a thread.
//   norm: v = h * weight; y = v / rms, a positive number for the whole row, so that q = 127 v / max|v| needs no rms and one
//   reduction gives both the sum of squares and max|v|; only the scale, max|v| / (127 rms), takes it.
//   gate: v = act(gate) * up.
template <class T, bool NORM, int ACT, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS == 64 ? 256 : THREADS) rows_kernel(RowsClearArgs a) {
    constexpr int kWaves = THREADS / 64, kRows = THREADS == 64 ? 4 : 1;
    __shared__ RowSums sums[2][kWaves];
    const int t = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (THREADS == 64 ? threadIdx.x >> 6 : 0); row < a.m;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const T *pa = static_cast<const T *>(a.a) + row * a.lda, *pb = a.b ? static_cast<const T *>(a.b) + row * a.ldb : nullptr;
        float v[CHUNKS][8];
        RowSums s = {0u, 0.0};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = 8 * (t + THREADS * c), left = a.k - at;
            for (int j = 0; j < 8; ++j) v[c][j] = 0.0f;
            if (left <= 0) continue;
            float o[8];
            load_8(pa + at, left, v[c]);
            if constexpr (NORM) {
                if (a.b) {
                    load_8(pb + at, left, o);
                    for (int j = 0; j < 8; ++j) v[c][j] += o[j];
                }
                if (a.total) store_8(static_cast<T *>(a.total) + row * a.ldt + at, left, v[c]);
                for (int j = 0; j < 8; ++j) s.squares = fma((double)v[c][j], (double)v[c][j], s.squares);
                if (a.weight) {
                    load_8(static_cast<const T *>(a.weight) + at, left, o);
                    for (int j = 0; j < 8; ++j) v[c][j] *= o[j];
                }
            } else {
                for (int j = 0; j < 8; ++j) v[c][j] = activate<ACT>(v[c][j]);
                if (a.b) {
                    load_8(pb + at, left, o);
                    for (int j = 0; j < 8; ++j) v[c][j] *= o[j];
                }
            }
            for (int j = 0; j < 8; ++j) {
                const unsigned bits = __float_as_uint(v[c][j]) & 0x7fffffffu;
                s.top = s.top > bits ? s.top : bits;
            }
        }
        s = across_wave<NORM>(s);
        if constexpr (kWaves > 1) {
            // two places in turn: a wave that is a row ahead does not overwrite what another still reads
            if ((t & 63) == 0) sums[turn][t >> 6] = s;
            __syncthreads();
            s = sums[turn][0];
            for (int w = 1; w < kWaves; ++w) s = join(s, sums[turn][w]);
        }
        const float top = __uint_as_float(s.top);
        if (t == 0) {
            double scale = (double)top / 127.0;
            if (NORM) scale /= sqrt(s.squares / a.k + (double)a.eps);
            a.scale[row] = a.k ? (float)scale : 0.0f;
        }
        // q = 127 v / top; rows near the bottom of the f32 range are lifted by 2^100 first, or 127 / top would be infinite
        const float lift = top < 0x1p-100f ? 0x1p100f : 1.0f;
        const float steps = s.top != 0u && s.top < 0x7f800000u ? 127.0f / (top * lift) : 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = 8 * (t + THREADS * c), left = a.k - at;
            if (left <= 0) continue;
            unsigned bytes[2] = {0u, 0u};
            for (int j = 0; j < 8; ++j) {
                // 1.5 * 2^23 added: the sum's last bits are the product rounded to the nearest whole number, once
                float w = fmaf(v[c][j] * lift, steps, 12582912.0f);
                if (steps == 0.0f) w = 12582912.0f;
                bytes[j >> 2] |= (__float_as_uint(w) & 0xffu) << (8 * (j & 3));
            }
            int8_t *q = a.q + row * a.ldq + at;
            if (left >= 8) {
                __builtin_memcpy(q, bytes, 8);
            } else {
                for (int j = 0; j < 8; ++j)
                    if (j < left) q[j] = (int8_t)(bytes[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

template <class T, bool NORM, int ACT>
static void rows_launch(const RowsClearArgs &a, hipStream_t stream) {
    const int64_t chunks = (a.k + 7) / 8;
    const auto groups = [&](int64_t rows) { return dim3((unsigned)(rows < kMostGroups ? rows : kMostGroups)); };
    if (chunks <= 64) rows_kernel<T, NORM, ACT, 64, 1><<<groups((a.m + 3) / 4), 256, 0, stream>>>(a);
    else if (chunks <= 256) rows_kernel<T, NORM, ACT, 256, 1><<<groups(a.m), 256, 0, stream>>>(a);
    else if (chunks <= 1024) rows_kernel<T, NORM, ACT, 1024, 1><<<groups(a.m), 1024, 0, stream>>>(a);
    else if (chunks <= 2048) rows_kernel<T, NORM, ACT, 1024, 2><<<groups(a.m), 1024, 0, stream>>>(a);
    else rows_kernel<T, NORM, ACT, 1024, 8><<<groups(a.m), 1024, 0, stream>>>(a);
}

template <bool NORM, int ACT>
static void rows_typed(const RowsClearArgs &a, hipStream_t stream) {
    if (a.type == BNN_CLEAR_F32) rows_launch<float, NORM, ACT>(a, stream);
    else if (a.type == BNN_CLEAR_BF16) rows_launch<__hip_bfloat16, NORM, ACT>(a, stream);
    else rows_launch<__half, NORM, ACT>(a, stream);
}

int launch_norm_clear(const RowsClearArgs &a, hipStream_t stream) {
    rows_typed<true, 0>(a, stream);
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

int launch_gate_clear(const RowsClearArgs &a, hipStream_t stream) {
    switch (a.act) {
        case BNN_ACT_RELU: rows_typed<false, BNN_ACT_RELU>(a, stream); break;
        case BNN_ACT_SILU: rows_typed<false, BNN_ACT_SILU>(a, stream); break;
        case BNN_ACT_GELU: rows_typed<false, BNN_ACT_GELU>(a, stream); break;
        default: rows_typed<false, BNN_ACT_IDENTITY>(a, stream); break;
    }
    TFHE_HIP(hipGetLastError());
    return TFHE_OK;
}

}  // namespace tfhe
