// The int32 result of an int8 product times its row and column scales: y = c col row, in binary32, rounded once.
//
// Bound by memory: every element is read and written once.  4096 rows of 4093 in 4097, to binary32, 134 MB: 28.4 us, 4.7 TB/s, nine tenths of a
// large copy's rate (rows of odd pitch begin anywhere: vectors are read and written wherever they lie).  768 x 1024 to half: 2.5 us, of which 1.7
// are a kernel that does nothing.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "launch.h"
#include "operators.h"
#include "strips.h"

namespace sparsert {

struct DequantArgs {
    const int32_t *C;
    const float *row, *col;
    void *Y;
    int32_t M, N, ldc, ldy;
};

// Strips as wide as the row allows, so that a wave reads a kilobyte of it at once. A workgroup of 256 threads does a strip of V * L columns in
// kDequantPasses * 256 / L rows: thread t has the V columns of lane t % L in the rows t / L, t / L + 256 / L, ...  All of its rows are fetched
// before the first is scaled.
constexpr int kDequantThreads = 256, kDequantPasses = 4;

template <typename T, int V, int L> __global__ __launch_bounds__(kDequantThreads) void dequantize_kernel(const DequantArgs a) {
    constexpr int W = V * L, ROWS = kDequantThreads / L, BLOCK = ROWS * kDequantPasses;
    const int strips = (a.N + W - 1) / W, blocks = (a.M + BLOCK - 1) / BLOCK;
    const int task = task_of(blockIdx.x, strips * blocks);
    if (task >= strips * blocks) return;
    const int strip = task % strips, first = task / strips * BLOCK;
    const int row = (int)threadIdx.x / L;
    const Columns<V> columns(strip * W + (int)threadIdx.x % L * V, a.N);
    const Matrix C(a.C + (int64_t)blockIdx.y * a.M * a.ldc, a.M, a.N, a.ldc, 4);
    const Matrix Y(static_cast<T *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, a.N, a.ldy, sizeof(T));
    const Matrix R(a.row, 1, a.M, a.M, 4), S(a.col ? a.col + (int64_t)blockIdx.y * a.N : nullptr, 1, a.N, a.N, 4);
    float col[V];
#pragma unroll
    for (int v = 0; v < V; ++v) col[v] = 1.0f;
    if (a.col) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float one[1];
            load<float, 1>(S, columns.any ? (uint32_t)(columns.first + v) * 4u : kNowhere, 0, one);
            col[v] = one[0];
        }
    }
    int32_t c[kDequantPasses][V];
    float r[kDequantPasses];
#pragma unroll
    for (int i = 0; i < kDequantPasses; ++i) {
        const int m = first + i * ROWS + row;
        load<int32_t, V>(C, m < a.M && columns.any ? ((uint32_t)m * (uint32_t)a.ldc + (uint32_t)columns.first) * 4u : kNowhere, 0, c[i]);
        float one[1] = {1.0f};
        if (a.row) load<float, 1>(R, m < a.M ? (uint32_t)m * 4u : kNowhere, 0, one);
        r[i] = one[0];
    }
#pragma unroll
    for (int i = 0; i < kDequantPasses; ++i) {
        const int m = first + i * ROWS + row;
        T y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] = (T)((float)c[i][v] * col[v] * r[i]);
        store<T, V>(Y, m < a.M && columns.any ? ((uint32_t)m * (uint32_t)a.ldy + (uint32_t)columns.first) * (uint32_t)sizeof(T) : kNowhere, 0,
                    columns.any ? columns.skip : 0, y);
    }
}

namespace {

template <typename T, int V> const void *dequantize_of(int lanes) {
    if constexpr (V > 1)   // (single columns are three at most)
        if (lanes > 4) return lanes == 64 ? (const void *)dequantize_kernel<T, V, 64> : (const void *)dequantize_kernel<T, V, 16>;
    return lanes == 4 ? (const void *)dequantize_kernel<T, V, 4> : (const void *)dequantize_kernel<T, V, 1>;
}

}  // namespace

int launch_dequantize(const DequantCall &c, std::string &err) {
    const sparsert_dequant &d = c.d;
    DequantArgs a{c.C, c.row, c.col, c.Y, d.M, d.N, d.ldc, d.ldy};
    const int V = d.N < 4 ? 1 : 4;   // 16 bytes of C to a lane
    const int vectors = (int)(((int64_t)d.N + V - 1) / V), lanes = vectors > 16 ? 64 : vectors > 4 ? 16 : vectors > 1 ? 4 : 1;
    const int64_t strips = (vectors + lanes - 1) / lanes, rows = kDequantThreads / lanes * kDequantPasses;
    const int64_t blocks = (d.M + rows - 1) / rows, tasks = strips * blocks;
    const bool half = d.dtype == SPARSERT_F16;
    const void *kernel = V == 1 ? half ? dequantize_of<_Float16, 1>(lanes) : dequantize_of<float, 1>(lanes)
                                : half ? dequantize_of<_Float16, 4>(lanes) : dequantize_of<float, 4>(lanes);
    return launch_operator(kernel, dim3((uint32_t)((tasks + 7) / 8 * 8), (uint32_t)d.batch), kDequantThreads, a, c.stream, err);
}

}  // namespace sparsert
