// Entry points of layers in the clear: argument checks, then one launch on the caller's stream.  Nothing is allocated,
// kept or synchronised, so any number of calls may overlap and be captured.
#include <cmath>

#include "clear_kernels.h"

namespace tfhe {

static bool is_aligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

static size_t type_bytes(int kind) {
    switch (kind) {
        case BNN_CLEAR_F32: case BNN_CLEAR_I32: return 4;
        case BNN_CLEAR_BF16: case BNN_CLEAR_F16: return 2;
        default: return 1;
    }
}

static int check_rows(int64_t m, int64_t k, int64_t most) {
    if (m < 0 || k < 0 || m > INT32_MAX) return set_error(TFHE_E_SIZE, "%lld rows of %lld values", (long long)m, (long long)k);
    if (k > most) return set_error(TFHE_E_SIZE, "rows of %lld values: at most %lld", (long long)k, (long long)most);
    return TFHE_OK;
}

static int check_stride(const char *what, int64_t ld, int64_t width) {
    if (ld < width || ld > (int64_t)1 << 40)
        return set_error(TFHE_E_SIZE, "row stride %lld of %s does not hold rows of %lld", (long long)ld, what, (long long)width);
    return TFHE_OK;
}

static int check_pointer(const char *what, const void *p, size_t bytes) {
    if (!p) return set_error(TFHE_E_NULL, "NULL %s", what);
    if (!is_aligned(p, bytes)) return set_error(TFHE_E_PARAM, "%s is not aligned to its %zu-byte elements", what, bytes);
    return TFHE_OK;
}

static int dense_clear(const DenseClearArgs &a, int64_t k, void *stream) {
    if (a.kind < BNN_CLEAR_F32 || a.kind > BNN_CLEAR_BITS) return set_error(TFHE_E_PARAM, "unknown output kind %d", a.kind);
    if (int rc = check_rows(a.m, k, kMaxDenseClearK)) return rc;
    if (a.n < 0 || a.n > INT32_MAX) return set_error(TFHE_E_SIZE, "%lld channels", (long long)a.n);
    if (int rc = check_stride("x", a.ldx, k)) return rc;
    if (int rc = check_stride("w", a.ldw, k)) return rc;
    if (int rc = check_stride("out", a.ldo, a.n)) return rc;
    if (a.kind >= BNN_CLEAR_I32 && (a.x_scale || a.w_scale)) return set_error(TFHE_E_PARAM, "whole-number outputs take no scales");
    if (a.m == 0 || a.n == 0) return TFHE_OK;
    if ((a.m + 31) / 32 * ((a.n + 63) / 64) > INT32_MAX)      // the kernels count tiles in 32 bits
         return set_error(TFHE_E_SIZE, "%lld x %lld outputs are too many", (long long)a.m, (long long)a.n);
    if (k > 0) {
        if (int rc = check_pointer("x", a.x, 1)) return rc;
        if (int rc = check_pointer("w", a.w, 1)) return rc;
    }
    if (int rc = check_pointer("out", a.out, type_bytes(a.kind))) return rc;
    if (!is_aligned(a.x_scale, 4) || !is_aligned(a.w_scale, 4) || !is_aligned(a.bias, 4))
        return set_error(TFHE_E_PARAM, "scales or bias not aligned to their 4-byte elements");
    return launch_dense_clear(a, static_cast<hipStream_t>(stream));
}

static int check_8bit_rows(const RowsClearArgs &a, int64_t k, int64_t most) {
    if (a.type < BNN_CLEAR_F32 || a.type > BNN_CLEAR_F16) return set_error(TFHE_E_PARAM, "unknown input type %d", a.type);
    if (int rc = check_rows(a.m, k, most)) return rc;
    return check_stride("q", a.ldq, k);
}

static int norm_clear(const RowsClearArgs &a, int64_t k, void *stream) {
    if (int rc = check_8bit_rows(a, k, kMaxNormClear)) return rc;
    if (!(a.eps > 0) || !(a.eps < INFINITY)) return set_error(TFHE_E_PARAM, "eps must be positive and finite");
    if (int rc = check_stride("x", a.lda, k)) return rc;
    if (a.b)
        if (int rc = check_stride("residual", a.ldb, k)) return rc;
    if (a.total)
        if (int rc = check_stride("total", a.ldt, k)) return rc;
    if (a.m == 0) return TFHE_OK;
    const size_t bytes = type_bytes(a.type);
    if (k > 0) {
        if (int rc = check_pointer("x", a.a, bytes)) return rc;
        if (int rc = check_pointer("q", a.q, 1)) return rc;
        if (!is_aligned(a.b, bytes) || !is_aligned(a.weight, bytes) || !is_aligned(a.total, bytes))
            return set_error(TFHE_E_PARAM, "residual, weight or total is not aligned to its %zu-byte elements", bytes);
    }
    if (int rc = check_pointer("scale", a.scale, 4)) return rc;
    return launch_norm_clear(a, static_cast<hipStream_t>(stream));
}

static int gate_clear(const RowsClearArgs &a, int64_t k, void *stream) {
    if (int rc = check_8bit_rows(a, k, kMaxGateClear)) return rc;
    if (a.act < BNN_ACT_IDENTITY || a.act > BNN_ACT_GELU) return set_error(TFHE_E_PARAM, "unknown activation %d", a.act);
    if (int rc = check_stride("gate", a.lda, k)) return rc;
    if (a.b)
        if (int rc = check_stride("up", a.ldb, k)) return rc;
    if (a.m == 0) return TFHE_OK;
    const size_t bytes = type_bytes(a.type);
    if (k > 0) {
        if (int rc = check_pointer("gate", a.a, bytes)) return rc;
        if (int rc = check_pointer("q", a.q, 1)) return rc;
        if (!is_aligned(a.b, bytes)) return set_error(TFHE_E_PARAM, "up is not aligned to its %zu-byte elements", bytes);
    }
    if (int rc = check_pointer("scale", a.scale, 4)) return rc;
    return launch_gate_clear(a, static_cast<hipStream_t>(stream));
}

}  // namespace tfhe

using namespace tfhe;

extern "C" {

int bnn_dense_clear(const int8_t *x, int64_t ldx, const int8_t *w, int64_t ldw, const float *x_scale, const float *w_scale,
                    const void *bias, void *out, int64_t ldo, int kind, int64_t m, int64_t n, int64_t k, void *stream) {
    return guarded([&]() -> int {
        return dense_clear({x, w, x_scale, w_scale, bias, out, ldx, ldw, ldo, m, n, (int)k, kind, false}, k, stream);
    });
}

int bnn_rms_norm_clear(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, float eps, void *total,
                       int64_t ldt, int8_t *q, int64_t ldq, float *scale, int type, int64_t m, int64_t k, void *stream) {
    return guarded([&]() -> int {
        return norm_clear({x, residual, weight, total, q, scale, ldx, ldr, ldt, ldq, m, (int)k, eps, type, 0}, k, stream);
    });
}

int bnn_gate_clear(const void *gate, int64_t ldg, const void *up, int64_t ldu, int act, int8_t *q, int64_t ldq, float *scale,
                   int type, int64_t m, int64_t k, void *stream) {
    return guarded([&]() -> int {
        return gate_clear({gate, up, nullptr, nullptr, q, scale, ldg, ldu, 0, ldq, m, (int)k, 0.0f, type, act}, k, stream);
    });
}

}  // extern "C"
