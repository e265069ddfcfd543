// The checks in front of the layers in the clear, under sanitizers: every refusal, the extremes of every argument, and what reaches a launcher.
// The launchers are stubs that look at what they were given.
#include <cmath>
#include <cstdio>
#include <cstdlib>

#include "../../paper_1806_03461_amd/csrc/clear_kernels.h"

static int launched = 0;

namespace tfhe {
int launch_dense_clear(const DenseClearArgs &a, hipStream_t) {
    if (a.k < 0 || a.k > kMaxDenseClearK || a.m < 1 || a.n < 1 || a.ldx < a.k || a.ldw < a.k || a.ldo < a.n || !a.out) std::abort();
    ++launched;
    return TFHE_OK;
}
int launch_norm_clear(const RowsClearArgs &a, hipStream_t) {
    if (a.k < 0 || a.k > kMaxNormClear || a.m < 1 || !(a.eps > 0) || !a.scale) std::abort();
    ++launched;
    return TFHE_OK;
}
int launch_gate_clear(const RowsClearArgs &a, hipStream_t) {
    if (a.k < 0 || a.k > kMaxGateClear || a.m < 1 || !a.scale) std::abort();
    ++launched;
    return TFHE_OK;
}
}  // namespace tfhe

int main() {
    alignas(16) static char mem[64];
    int8_t *const b = reinterpret_cast<int8_t *>(mem);
    float *const f = reinterpret_cast<float *>(mem);
    const int64_t ends[] = {INT64_MIN, -1, 0, 1, 63, 64, 65, 131071, 131072, 65536, 65537, INT32_MAX, (int64_t)INT32_MAX + 1, (int64_t)1 << 40, INT64_MAX};
    int accepted = 0, refused = 0;
    const auto count = [&](int rc) { rc == TFHE_OK ? ++accepted : ++refused; };
    for (int64_t v : ends)
        for (int64_t w : ends)
            for (int kind = -1; kind <= 6; ++kind) {
                count(bnn_dense_clear(b, w, b, w, nullptr, nullptr, f, mem, 64, kind, v, 64, w, nullptr));
                count(bnn_dense_clear(b, 64, b, v, f, f, nullptr, mem, w, kind, v, w, 64, nullptr));
                count(bnn_dense_clear(nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr, mem, w, kind, v, w, 0, nullptr));
                count(bnn_rms_norm_clear(mem, v, mem, v, mem, 1e-5f, mem, v, b, v, f, kind, w, v, nullptr));
                count(bnn_gate_clear(mem, v, nullptr, 0, kind, b, v, f, BNN_CLEAR_BF16, w, v, nullptr));
                count(bnn_gate_clear(mem + 1, 64, mem, 64, BNN_ACT_SILU, b, 64, f, kind, v, 64, nullptr));
            }
    for (float eps : {0.0f, -1.0f, INFINITY, NAN})
        if (bnn_rms_norm_clear(mem, 8, nullptr, 0, nullptr, eps, nullptr, 0, b, 8, f, BNN_CLEAR_F32, 1, 8, nullptr) != TFHE_E_PARAM) return 1;
    if (!launched || !accepted || !refused) return 2;
    std::printf("clear layers' checks: ok (%d accepted, %d refused, %d launched)\n", accepted, refused, launched);
    return 0;
}
