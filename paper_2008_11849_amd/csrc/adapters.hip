// Low-rank adapters of many requests beside a projection that they share, in two kernels:
//   shrink  t[n, j] = sum_k down[a][j, k] x[k, n]         for the adapter a of every token
//   expand  Y[m, n] = c[m, n] + alpha[a] sum_j up[a][m, j] t[n, j]
#include <hip/hip_runtime.h>

#include "launch.h"
#include "operators.h"

namespace sparsert {

namespace {

struct ShrinkArgs {
    const void *X, *down;
    const int32_t *index;
    float *t;
    int32_t K, N, ldx, rank, count;
};

struct ExpandArgs {
    const void *C, *up;
    const int32_t *index;
    const float *alpha, *row, *col, *t;
    void *Y;
    int32_t M, N, ldc, ldy, rank, count;
};

// One wave per token and row of `down`.
template <typename X, typename W> __global__ __launch_bounds__(64) void shrink_kernel(const ShrinkArgs a) {
    const int n = blockIdx.x / a.rank, j = blockIdx.x % a.rank;
    const size_t token = (size_t)blockIdx.y * a.N + n;
    const int id = a.index[token];
    if (id < 0 || id >= a.count) return;
    const X *x = static_cast<const X *>(a.X) + (size_t)blockIdx.y * a.K * a.ldx + n;
    const W *w = static_cast<const W *>(a.down) + ((size_t)id * a.rank + j) * a.K;
    float s = 0.0f;
    for (int k = threadIdx.x; k < a.K; k += 64) s = __builtin_fmaf((float)x[(size_t)k * a.ldx], (float)w[k], s);
    for (int i = 32; i; i >>= 1) s += __shfl_xor(s, i);
    if (threadIdx.x == 0) a.t[token * a.rank + j] = s;
}

template <typename C, typename W> __global__ __launch_bounds__(256) void expand_kernel(const ExpandArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(i / a.N), n = (int)(i % a.N);
    if (m >= a.M) return;
    const size_t token = (size_t)blockIdx.y * a.N + n;
    const int id = a.index[token];
    float s = 0.0f;
    if (id >= 0 && id < a.count) {
        const W *u = static_cast<const W *>(a.up) + ((size_t)id * a.M + m) * a.rank;
        for (int j = 0; j < a.rank; ++j) s = __builtin_fmaf((float)u[j], a.t[token * a.rank + j], s);
        if (a.alpha) s *= a.alpha[id];
    }
    float y = (float)static_cast<const C *>(a.C)[((size_t)blockIdx.y * a.M + m) * a.ldc + n] + (std::is_same<C, int32_t>::value ? 0.0f : s);
    if constexpr (std::is_same<C, int32_t>::value) {
        const float col = a.col ? a.col[token] : 1.0f;
        y = y * col * (a.row ? a.row[m] : 1.0f) + s * col;
    }
    static_cast<W *>(a.Y)[((size_t)blockIdx.y * a.M + m) * a.ldy + n] = (W)y;
}

}  // namespace

size_t adapters_workspace(const sparsert_adapter_set &d) { return (size_t)d.batch * d.N * d.rank * sizeof(float); }

int launch_adapters(const AdaptersCall &c, std::string &err) {
    const sparsert_adapter_set &d = c.d;
    const bool half = d.dtype == SPARSERT_F16, i8 = d.x_dtype == SPARSERT_I8;
    if ((int64_t)d.N * d.rank >= (1ll << 31)) { err = "too many workgroups"; return SPARSERT_EUNSUPPORTED; }
    ShrinkArgs s{c.X, c.down, c.index, static_cast<float *>(c.workspace), d.K, d.N, d.ldx, d.rank, d.count};
    const void *shrink = i8 ? half ? (const void *)shrink_kernel<int8_t, _Float16> : (const void *)shrink_kernel<int8_t, float>
                            : half ? (const void *)shrink_kernel<_Float16, _Float16> : (const void *)shrink_kernel<float, float>;
    if (int rc = launch_operator(shrink, dim3(d.N * d.rank, d.batch), 64, s, c.stream, err)) return rc;
    ExpandArgs e{c.C, c.up, c.index, c.alpha, c.row, c.col, static_cast<float *>(c.workspace), c.Y, d.M, d.N, d.ldc, d.ldy, d.rank, d.count};
    const void *expand = i8 ? half ? (const void *)expand_kernel<int32_t, _Float16> : (const void *)expand_kernel<int32_t, float>
                            : half ? (const void *)expand_kernel<_Float16, _Float16> : (const void *)expand_kernel<float, float>;
    return launch_operator(expand, dim3((uint32_t)(((int64_t)d.M * d.N + 255) / 256), d.batch), 256, e, c.stream, err);
}

}  // namespace sparsert
