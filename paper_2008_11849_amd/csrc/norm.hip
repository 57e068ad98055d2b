// Root-mean-square norm over the features of every token, with the residual's addition and, for int8 products, quantisation.
#include <hip/hip_runtime.h>

#include <cmath>

#include "launch.h"
#include "operators.h"

namespace sparsert {

namespace {

struct NormArgs {
    const void *X, *R;
    const float *gamma;
    void *H, *Y;
    float *scale;
    int32_t K, N, ldx, ldh, ldy;
    float eps;
};

// The larger of two sizes by their bits: as numbers, and above them infinity and what is undefined.
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }

constexpr int kCols = 8, kRows = 32;   // columns of a workgroup, and the threads that share the rows of each

template <typename T, bool QUANT>
__global__ __launch_bounds__(kCols *kRows) void norm_kernel(const NormArgs a) {
    __shared__ float sums[kRows][kCols], tops[kRows][kCols], factor[kCols];
    const int c = threadIdx.x % kCols, r = threadIdx.x / kCols, n = blockIdx.x * kCols + c;
    const T *X = static_cast<const T *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx;
    const T *R = a.R ? static_cast<const T *>(a.R) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr;
    T *H = a.H ? static_cast<T *>(a.H) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr;
    auto sum_at = [&](int k) { return (float)X[(size_t)k * a.ldx + n] + (R ? (float)R[(size_t)k * a.ldh + n] : 0.0f); };
    float s = 0.0f, top = 0.0f;
    if (n < a.N)
        for (int k = r; k < a.K; k += kRows) {
            const float h = sum_at(k);
            s = __builtin_fmaf(h, h, s);
            top = larger(top, fabsf(a.gamma ? h * a.gamma[k] : h));
        }
    sums[r][c] = s;
    tops[r][c] = top;
    __syncthreads();
    if (r == 0) {
        for (int i = 1; i < kRows; ++i) s += sums[i][c], top = larger(top, tops[i][c]);
        const float inv = 1.0f / sqrtf(s / (float)a.K + a.eps);
        if constexpr (QUANT) {
            const bool sound = s < INFINITY && top < INFINITY, some = top >= 0x1p-100f;
            factor[c] = sound && some ? 127.0f / top : 0.0f;
            if (n < a.N) a.scale[(size_t)blockIdx.y * a.N + n] = !sound ? NAN : some ? top * inv / 127.0f : 0.0f;
        } else {
            factor[c] = inv;
        }
    }
    __syncthreads();
    if (n >= a.N) return;
    const float f = factor[c];
    for (int k = r; k < a.K; k += kRows) {
        const float h = sum_at(k), v = a.gamma ? h * a.gamma[k] : h;
        if (H) H[(size_t)k * a.ldh + n] = (T)h;
        const size_t at = ((size_t)blockIdx.y * a.K + k) * a.ldy + n;
        if constexpr (QUANT) static_cast<int8_t *>(a.Y)[at] = f == 0.0f ? (int8_t)0 : (int8_t)rintf(v * f);
        else static_cast<T *>(a.Y)[at] = (T)(v * f);
    }
}

}  // namespace

int launch_norm(const NormCall &c, std::string &err) {
    const sparsert_norm &d = c.d;
    NormArgs a{c.X, c.R, c.gamma, c.H, c.Y, c.scale, d.K, d.N, d.ldx, d.ldh, d.ldy, d.eps};
    const bool half = d.dtype == SPARSERT_F16, quant = d.out_dtype == SPARSERT_I8;
    const void *kernel = half ? quant ? (const void *)norm_kernel<_Float16, true> : (const void *)norm_kernel<_Float16, false>
                              : quant ? (const void *)norm_kernel<float, true> : (const void *)norm_kernel<float, false>;
    return launch_operator(kernel, dim3((d.N + kCols - 1) / kCols, d.batch), kCols * kRows, a, c.stream, err);
}

bool stream_of_current_device(void *stream) {
    if (reinterpret_cast<uintptr_t>(stream) <= 2) return true;   // the null stream and its per-thread form go by the current device
    hipDevice_t of = -1;
    int current = -1;
    if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &of) != hipSuccess || hipGetDevice(&current) != hipSuccess) return false;
    return of == current;
}

}  // namespace sparsert
