// The int32 result of an int8 product times its row and column scales.
#include <hip/hip_runtime.h>

#include "launch.h"
#include "operators.h"

namespace sparsert {

namespace {

struct DequantArgs {
    const int32_t *C;
    const float *row, *col;
    void *Y;
    int32_t M, N, ldc, ldy;
};

template <typename T> __global__ __launch_bounds__(256) void dequantize_kernel(const DequantArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(i / a.N), n = (int)(i % a.N);
    if (m >= a.M) return;
    const float c = (float)a.C[((size_t)blockIdx.y * a.M + m) * a.ldc + n];
    const float v = c * (a.col ? a.col[(size_t)blockIdx.y * a.N + n] : 1.0f) * (a.row ? a.row[m] : 1.0f);
    static_cast<T *>(a.Y)[((size_t)blockIdx.y * a.M + m) * a.ldy + n] = (T)v;
}

}  // namespace

int launch_dequantize(const DequantCall &c, std::string &err) {
    const sparsert_dequant &d = c.d;
    DequantArgs a{c.C, c.row, c.col, c.Y, d.M, d.N, d.ldc, d.ldy};
    const void *kernel = d.dtype == SPARSERT_F16 ? (const void *)dequantize_kernel<_Float16> : (const void *)dequantize_kernel<float>;
    return launch_operator(kernel, dim3((uint32_t)(((int64_t)d.M * d.N + 255) / 256), d.batch), 256, a, c.stream, err);
}

}  // namespace sparsert
