// Launchers of the gfx950 kernels of layers in the clear (clear_kernels.hip), called by clear_layers.cpp, which checks the arguments.
#pragma once
#include "common.h"

namespace tfhe {

struct DenseClearArgs {
    const int8_t *x, *w;            // [m][k] with row stride ldx, [n][k] with row stride ldw
    const float *x_scale, *w_scale; // [m], [n]; NULL = 1
    const void *bias;               // [n] float or int32, or NULL
    void *out;                      // [m][n] with row stride ldo
    int64_t ldx, ldw, ldo;
    int64_t m, n;
    int k;
    int kind;                       // BNN_CLEAR_F32 ... BNN_CLEAR_BITS
    bool past;                      // set by the launcher: stores past the caches' order of what to keep
};

struct RowsClearArgs {
    const void *a, *b;              // norm: x and the residual or NULL; gate: gate and up or NULL
    const void *weight;             // norm: [k] or NULL
    void *total;                    // norm: x + residual, or NULL
    int8_t *q;
    float *scale;
    int64_t lda, ldb, ldt, ldq;
    int64_t m;
    int k;
    float eps;
    int type;                       // BNN_CLEAR_F32, BNN_CLEAR_BF16 or BNN_CLEAR_F16
    int act;
};

// largest k of a product: 128 * 128 * k stays below 2^31
constexpr int64_t kMaxDenseClearK = 131071;
// longest rows: 1,024 threads hold one in registers, the norm's 32 values each, the gate's 64.  With 64 the norm, which holds weights and a second output beside
// them, needs 200 bytes a lane of scratch, which the runtime would allocate at its first launch.
constexpr int64_t kMaxNormClear = 32768, kMaxGateClear = 65536;

int launch_dense_clear(const DenseClearArgs &a, hipStream_t stream);
int launch_norm_clear(const RowsClearArgs &a, hipStream_t stream);
int launch_gate_clear(const RowsClearArgs &a, hipStream_t stream);

}  // namespace tfhe
