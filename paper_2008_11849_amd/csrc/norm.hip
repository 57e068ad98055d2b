// Root-mean-square norm over the features of every token, with the residual's addition and, for int8 products, quantisation.
//
// h = x + r,  v = h gamma,  f = 1 / sqrt(sum h^2 / K + eps),  y = v f.  int8: y = round(127 v / a) with a = max |v|, scale a f / 127: f drops out
// of the integers, so that the sum of squares and the maximum come from one pass.  A token is a column: its sums run down the rows, lanes of a wave
// lie along them, so that rows are read in runs, and columns meet in LDS.  Everything is held in binary32 and rounded once, at the stores; sums are
// added in one order, whatever the timing.
//
// Bounds: the wait for one read of memory and for two rounds through LDS in small calls (K = 1024, one token: 2.3 us, of which 1.7 are a kernel
// that does nothing), memory in large ones: 4096 x 4096 half with both residuals, 134 MB: 33.6 us, 4.0 TB/s, where two copies of as many bytes take
// 28.2 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "launch.h"
#include "operators.h"
#include "strips.h"
#include "wave_sums.h"

namespace sparsert {

struct NormArgs {
    const void *X, *R;
    const float *gamma;
    void *H, *Y;
    float *scale;
    int32_t K, N, ldx, ldh, ldy;
    float eps;
    float *sums;           // split norms: the parts' sums,
    int32_t parts, rows;   // parts of a column, and rows of each
};

// 1 / sqrt(m), rounded once: a root and a quotient are two roundings, 1.5 times as far off.  A step of Newton's from there, on what is left of m r^2
// to 1, exactly.
__device__ __forceinline__ float reciprocal_root(float m) {
    const float r = 1.0f / sqrtf(m), h = m * r, rest = __builtin_fmaf(-h, r, 1.0f) - __builtin_fmaf(m, r, -h) * r;
    return r > 0.0f ? __builtin_fmaf(0.5f * r, rest, r) : r;   // (of infinity it is 0)
}

// What a column's weighted sums are multiplied with, from the sum of its squares and its largest |h * gamma|.
template <bool QUANT> __device__ __forceinline__ float factor_of(float total, float most, const NormArgs &a, float &scale) {
    const float inv = reciprocal_root(total / (float)a.K + a.eps);
    if constexpr (!QUANT) return inv;
    const bool sound = total < INFINITY && most < INFINITY, some = most >= 0x1p-100f;
    scale = !sound ? NAN : some ? most * inv / 127.0f : 0.0f;
    return sound && some ? 127.0f / most : 0.0f;
}
template <typename Out> __device__ __forceinline__ Out result(float v, float f) {
    if constexpr (sizeof(Out) == 1) return f == 0.0f ? (int8_t)0 : (int8_t)(int)rintf(v * f);
    else return (Out)(v * f);
}

// Rows [first, end) of a strip of V * L columns: thread t has V columns in the rows first + t / L, first + t / L + THREADS / L, ...,
// a pass for each of them.
template <typename T, int V, int L, int THREADS> struct Rows {
    static constexpr int W = V * L, ROWS = THREADS / L;
    const NormArgs &a;
    int row, first, end;
    Columns<V> columns;
    Matrix X, R, G;
    __device__ __forceinline__ Rows(const NormArgs &a, int strip, int first, int end)
        : a(a), row((int)threadIdx.x / L), first(first), end(end), columns(strip * W + (int)threadIdx.x % L * V, a.N),
          X(static_cast<const T *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, a.N, a.ldx, sizeof(T)),
          R(a.R ? static_cast<const T *>(a.R) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr, a.K, a.N, a.ldh, sizeof(T)),
          G(a.gamma, 1, a.K, a.K, sizeof(float)) {}
    // This thread's byte in pass i of the rows from k0 on.
    __device__ __forceinline__ uint32_t place(int k0, int i, int ld, int size, uint32_t &common) const {
        const int at = k0 + i * ROWS;
        common = at < end ? (uint32_t)at * (uint32_t)ld * (uint32_t)size : 0;
        return at + row < end && columns.any ? ((uint32_t)row * (uint32_t)ld + (uint32_t)columns.first) * (uint32_t)size : kNowhere;
    }
    // The sums and weights of PASSES passes, every load before the first use.  Rows past the end are zeros.
    template <int PASSES> __device__ __forceinline__ void fetch(int k0, float (&h)[PASSES][V], float (&g)[PASSES]) const {
        T x[PASSES][V], r[PASSES][V];
        uint32_t common;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const uint32_t at = place(k0, i, a.ldx, sizeof(T), common);
            load<T, V>(X, at, common, x[i]);
        }
        if (a.R) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const uint32_t at = place(k0, i, a.ldh, sizeof(T), common);
                load<T, V>(R, at, common, r[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < PASSES; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v) r[i][v] = T(-0.0f);   // x + -0 is x
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int k = k0 + i * ROWS + row;
            g[i] = a.gamma ? __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(G.at, k < end ? (uint32_t)k * 4u : kNowhere, 0, 0))
                : 1.0f;
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) h[i][v] = (float)x[i][v] + (float)r[i][v];
    }
    template <typename Out, int PASSES, int AUX = 0, typename F>
    __device__ __forceinline__ void write(const Matrix &m, int k0, int ld, F value) const {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            Out out[V];
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = value(i, v);
            uint32_t common;
            const uint32_t at = place(k0, i, ld, sizeof(Out), common);
            store<Out, V, AUX>(m, at, common, columns.any ? columns.skip : 0, out);
        }
    }
};

template <typename T, bool QUANT> using out_t = typename std::conditional<QUANT, int8_t, T>::type;
template <typename T> __device__ __forceinline__ Matrix sum_of(const NormArgs &a) {
    return Matrix(a.H ? static_cast<T *>(a.H) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr, a.K, a.N, a.ldh, sizeof(T));
}
template <typename Out> __device__ __forceinline__ Matrix result_of(const NormArgs &a) {
    return Matrix(static_cast<Out *>(a.Y) + (int64_t)blockIdx.y * a.K * a.ldy, a.K, a.N, a.ldy, sizeof(Out));
}

// ---- One kernel: a workgroup of THREADS threads does a strip.  HELD: PASSES passes are all rows, and stay in registers between the
// sums and the results; otherwise the rows are fetched twice.  768 x 1024 half to int8: 5.0 us; 4096 x 16: 5.7 us.
template <typename T, bool QUANT, int V, int L, int PASSES, bool HELD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(const NormArgs a) {
    typedef out_t<T, QUANT> Out;
    typedef Rows<T, V, L, THREADS> Strip;
    constexpr int W = V * L, WAVES = THREADS / 64, ROWS = Strip::ROWS;
    __shared__ __align__(16) float sums[WAVES][W], tops[QUANT ? WAVES : 1][W], factors[W];
    const int strips = (a.N + W - 1) / W, strip = task_of(blockIdx.x, strips);
    if (strip >= strips) return;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const Strip rows(a, strip, 0, a.K);
    const Matrix H = sum_of<T>(a), Y = result_of<Out>(a);
    float h[PASSES][V], g[PASSES], s[V], top[V], f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = top[v] = 0.0f;
    auto weigh = [&](bool add) {   // h becomes h * gamma; `add`: and is added up
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (add) s[v] = __builtin_fmaf(h[i][v], h[i][v], s[v]);
                h[i][v] *= g[i];
                if constexpr (QUANT)
                    if (add) top[v] = larger(top[v], fabsf(h[i][v]));
            }
    };
    auto write_sum = [&](int k0) {
        if (a.H) rows.template write<T, PASSES>(H, k0, a.ldh, [&](int i, int v) { return (T)h[i][v]; });
    };
    auto write = [&](int k0) { rows.template write<Out, PASSES>(Y, k0, a.ldy, [&](int i, int v) { return result<Out>(h[i][v], f[v]); }); };

    if constexpr (HELD) {
        rows.fetch(0, h, g);
        write_sum(0);
        weigh(true);
    } else {
        for (int k0 = 0; k0 < a.K; k0 += PASSES * ROWS) {
            rows.fetch(k0, h, g);
            weigh(true);
        }
    }
    // The sums meet in LDS, in wave order.
    wave_sums<V, L, false>(s, lane, rows.columns.skip, sums[wave]);
    if constexpr (QUANT) wave_sums<V, L, true>(top, lane, rows.columns.skip, tops[wave]);
    __syncthreads();
    if (t < W && strip * W + t < a.N) {
        float total = sums[0][t], most = 0.0f, scale;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) total += sums[w][t];
        if constexpr (QUANT)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = larger(most, tops[w][t]);
        factors[t] = factor_of<QUANT>(total, most, a, scale);
        if constexpr (QUANT) a.scale[(size_t)blockIdx.y * a.N + strip * W + t] = scale;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = factors[max(0, t % L * V + v - rows.columns.skip)];   // (of skipped columns: not used)
    if constexpr (HELD) {
        write(0);
    } else {
        for (int k0 = 0; k0 < a.K; k0 += PASSES * ROWS) {
            rows.fetch(k0, h, g);
            write_sum(k0);
            weigh(false);
            write(k0);
        }
    }
}

// ---- Two kernels, for columns too few and too long to fill the GPU, and for calls beyond the caches: sums of every part of a strip, then the
// results.  A part is `rows` rows of a strip.  The second kernel reads the rows again, from the caches (of 4096 x 4096 half, 67 MB, from the one
// beside memory).  1027 x 771 of 784, binary32: 7.1 us.  The parts' sums and largest values lie in the caller's workspace, [batch][part][1 or
// 2][N].
constexpr int kPartThreads = 256, kWideLanes = 16;
constexpr int kPartPasses = 4;    // rows of a thread that are fetched at a time
constexpr int kPartsAtOnce = 8;   // sums that a thread of the second kernel fetches at a time

// Task -> strip and part, the same in both kernels, so that the second one finds in its L2 what the first one fetched.  Parts of a strip
// one after the other; in the wide strips that calls beyond the caches take, strips of a part, so that an XCD reads long runs of a row.
template <int L> __device__ __forceinline__ int strip_of(int task, int strips, int parts) { return L >= kWideLanes ? task % strips : task / parts; }
template <int L> __device__ __forceinline__ int part_of(int task, int strips, int parts) { return L >= kWideLanes ? task / strips : task % parts; }

template <typename T, bool QUANT, int V, int L> __global__ __launch_bounds__(kPartThreads) void norm_sums_kernel(const NormArgs a) {
    typedef Rows<T, V, L, kPartThreads> Part;
    constexpr int W = V * L, WAVES = kPartThreads / 64;
    __shared__ float sums[WAVES][W], tops[QUANT ? WAVES : 1][W];
    const int strips = (a.N + W - 1) / W, task = task_of(blockIdx.x, strips * a.parts);
    if (task >= strips * a.parts) return;
    const int strip = strip_of<L>(task, strips, a.parts), part = part_of<L>(task, strips, a.parts), t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const Part p(a, strip, part * a.rows, min(a.K, (part + 1) * a.rows));
    float s[V], top[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = top[v] = 0.0f;
    for (int k0 = p.first; k0 < p.end; k0 += kPartPasses * Part::ROWS) {
        float h[kPartPasses][V], g[kPartPasses];
        p.fetch(k0, h, g);
#pragma unroll
        for (int i = 0; i < kPartPasses; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[v] = __builtin_fmaf(h[i][v], h[i][v], s[v]);
                if constexpr (QUANT) top[v] = larger(top[v], fabsf(h[i][v] * g[i]));
            }
    }
    wave_sums<V, L, false>(s, lane, p.columns.skip, sums[wave]);
    if constexpr (QUANT) wave_sums<V, L, true>(top, lane, p.columns.skip, tops[wave]);
    __syncthreads();
    float *const to = a.sums + ((size_t)blockIdx.y * a.parts + part) * (QUANT ? 2 : 1) * a.N;
    const int n = strip * W + t;
    if (t < W && n < a.N) {
        float total = sums[0][t], most = 0.0f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) total += sums[w][t];
        to[n] = total;
        if constexpr (QUANT) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = larger(most, tops[w][t]);
            to[a.N + n] = most;
        }
    }
}

// FAR: H is not to be kept in the caches, so that it does not displace Y, which the next call reads first.
template <typename T, bool QUANT, int V, int L, bool FAR> __global__ __launch_bounds__(kPartThreads) void norm_results_kernel(const NormArgs a) {
    typedef out_t<T, QUANT> Out;
    typedef Rows<T, V, L, kPartThreads> Part;
    constexpr int W = V * L, GROUPS = kPartThreads / W;
    __shared__ float sums[GROUPS][W], tops[QUANT ? GROUPS : 1][W];
    __shared__ __align__(16) float factors[W];
    const int strips = (a.N + W - 1) / W, task = task_of(blockIdx.x, strips * a.parts);
    if (task >= strips * a.parts) return;
    const int strip = strip_of<L>(task, strips, a.parts), part = part_of<L>(task, strips, a.parts), t = threadIdx.x;
    const Part p(a, strip, part * a.rows, min(a.K, (part + 1) * a.rows));
    const Matrix H = sum_of<T>(a), Y = result_of<Out>(a);
    // The parts' sums of a column, dealt to GROUPS threads and joined in LDS: always in the same order.
    const float *const from = a.sums + (size_t)blockIdx.y * a.parts * (QUANT ? 2 : 1) * a.N;
    const int c = t % W, n = strip * W + c;
    float total = 0.0f, most = 0.0f;
    if (n < a.N)
        for (int of = t / W; of < a.parts; of += GROUPS * kPartsAtOnce) {
            float u[kPartsAtOnce], q[kPartsAtOnce];
#pragma unroll
            for (int j = 0; j < kPartsAtOnce; ++j) {
                const int which = of + j * GROUPS;
                u[j] = which < a.parts ? from[(size_t)which * (QUANT ? 2 : 1) * a.N + n] : 0.0f;
                if constexpr (QUANT) q[j] = which < a.parts ? from[((size_t)which * 2 + 1) * a.N + n] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < kPartsAtOnce; ++j) {
                total += u[j];
                if constexpr (QUANT) most = larger(most, q[j]);
            }
        }
    sums[t / W][c] = total;
    if constexpr (QUANT) tops[t / W][c] = most;
    __syncthreads();
    if (t < W) {
        float scale;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) {
            total += sums[i][c];
            if constexpr (QUANT) most = larger(most, tops[i][c]);
        }
        factors[t] = factor_of<QUANT>(total, most, a, scale);
        if constexpr (QUANT)
            if (part == 0 && n < a.N) a.scale[(size_t)blockIdx.y * a.N + n] = scale;
    }
    __syncthreads();
    float f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = factors[max(0, t % L * V + v - p.columns.skip)];   // (of skipped columns: not used)
    for (int k0 = p.first; k0 < p.end; k0 += kPartPasses * Part::ROWS) {
        float h[kPartPasses][V], g[kPartPasses];
        p.fetch(k0, h, g);
        if (a.H) p.template write<T, kPartPasses, FAR ? 2 : 0>(H, k0, a.ldh, [&](int i, int v) { return (T)h[i][v]; });
        p.template write<Out, kPartPasses>(Y, k0, a.ldy, [&](int i, int v) { return result<Out>(h[i][v] * g[i], f[v]); });
    }
}

namespace {

constexpr int kNormThreads = 1024;

template <typename T, bool QUANT, int V, int L> const void *norm_of(int K) {
    constexpr int ROWS = kNormThreads / L;
    const int passes = (K + ROWS - 1) / ROWS;
    if (passes <= 1) return (const void *)norm_kernel<T, QUANT, V, L, 1, true, kNormThreads>;
    if (passes <= 2) return (const void *)norm_kernel<T, QUANT, V, L, 2, true, kNormThreads>;
    if (passes <= 4) return (const void *)norm_kernel<T, QUANT, V, L, 4, true, kNormThreads>;
    if (passes <= 8) return (const void *)norm_kernel<T, QUANT, V, L, 8, true, kNormThreads>;
    return (const void *)norm_kernel<T, QUANT, V, L, 4, false, kNormThreads>;
}

// Columns of a lane and lanes of a strip: 16 bytes, and as many lanes as leave 256 workgroups; narrower than that, one column to a lane.  Where a
// lane is a strip and 128 columns or fewer are all, four columns in half, too.  Four and eight, in us, to int8: 4096 x 8 5.1 and 6.2, x 16 5.8 and
// 6.5, x 32 8.4 and 8.3; 1024 x 8 3.3 and 3.6, x 128 4.7 and 4.7, x 384 5.3 and 5.1, x 1024 6.5 and 5.7.  From 32 to 256 columns they are within 5
// % of each other in calls that are one kernel.
template <typename T> void strip_shape(const sparsert_norm &d, int &V, int &L) {
    V = 16 / sizeof(T);
    if (d.N < V) {
        V = 1;
        L = d.N > 4 ? 8 : d.N > 2 ? 4 : d.N;
        return;
    }
    const int64_t vectors = (int64_t)d.batch * ((d.N + V - 1) / V);
    L = vectors >= 8 * 256 ? 8 : vectors >= 4 * 256 ? 4 : vectors >= 2 * 256 ? 2 : 1;
    if (L == 1 && (int64_t)d.batch * d.N <= 128) V = 4;
}

template <typename T, bool QUANT> const void *norm_of(const sparsert_norm &d, int &columns) {
    int V, L;
    strip_shape<T>(d, V, L);
    columns = V * L;
    constexpr int W = 16 / sizeof(T);
    if constexpr (W > 4)   // (single columns are fewer than W)
        if (V == 1 && L == 8) return norm_of<T, QUANT, 1, 8>(d.K);
    if (V == 1) return L == 4 ? norm_of<T, QUANT, 1, 4>(d.K) : L == 2 ? norm_of<T, QUANT, 1, 2>(d.K) : norm_of<T, QUANT, 1, 1>(d.K);
    if (V == 4 && L == 1) return norm_of<T, QUANT, 4, 1>(d.K);
    return L == 8 ? norm_of<T, QUANT, W, 8>(d.K) : L == 4 ? norm_of<T, QUANT, W, 4>(d.K)
         : L == 2 ? norm_of<T, QUANT, W, 2>(d.K) : norm_of<T, QUANT, W, 1>(d.K);
}

// Estimate of a call as one kernel, fitted (with eight halves to a lane) to calls of one to 4096 tokens of 768 to 8192 rows: a turn of the loads
// costs its wait and what the strip's narrowness wastes of the lines that it touches.
template <typename T> double one_kernel_us(const sparsert_norm &d, double bytes) {
    int V, L;
    strip_shape<T>(d, V, L);
    const int passes = (d.K + kNormThreads / L - 1) / (kNormThreads / L);
    if (V == 1) return 2.2 + passes * (passes <= 8 ? 0.2 : 0.55);
    const double lines = std::min(1.0, d.ldx * (double)sizeof(T) / 128.0);   // that a lane's vector is alone in
    return 2.2 + passes * (0.35 + 1.9 * lines / L) * (passes <= 8 ? 1.0 : 2.0) + bytes / 5e6;
}

struct SplitNorm { int parts, rows, strips; const void *sums, *results; };

template <typename T, bool QUANT, int V, int L, bool FAR = false> SplitNorm split_with(const sparsert_norm &d, int workgroups) {
    constexpr int W = V * L, ROWS = kPartThreads / L;
    const int strips = (int)(((int64_t)d.N + W - 1) / W);
    // No more parts than a workgroup fetches the sums of at once.
    const int64_t most = std::min<int64_t>((d.K + ROWS - 1) / ROWS, kPartThreads / W * kPartsAtOnce);
    const int64_t parts = std::min(most, std::max<int64_t>(1, workgroups / ((int64_t)strips * d.batch)));
    const int rows = (int)((d.K + parts - 1) / parts);
    return {(d.K + rows - 1) / rows, rows, strips, (const void *)norm_sums_kernel<T, QUANT, V, L>,
            (const void *)norm_results_kernel<T, QUANT, V, L, FAR>};
}

template <typename T, bool QUANT> SplitNorm split_of(const sparsert_norm &d) {
    constexpr int V = 16 / sizeof(T);
    const double bytes = (double)d.K * d.N * d.batch * (3 * sizeof(T) + sizeof(out_t<T, QUANT>));
    // One kernel and two, measured in us (half): 1024 x 16 3.4 and 6.1, 768 x 1024 5.1 and 6.2, 2048 x 1024 10.3 and 7.7, 4096 x 128 12.9 and 6.5,
    // 8192 x 1024 37 and 20.  Over 232 sizes, of half and binary32 to themselves and to int8, the choices come to 0.4 % above the best of each,
    // with 13 % at most (4096 x 16 half 6.2 and 5.5).
    if (one_kernel_us<T>(d, bytes) <= (QUANT ? 6.2 : 5.3) + bytes / 4.4e6) return {};
    if constexpr (V > 4)
        if (d.N > 4 && d.N < V) return split_with<T, QUANT, 1, 8>(d, 256);
    if (d.N < V) return d.N > 2 ? split_with<T, QUANT, 1, 4>(d, 256) : split_with<T, QUANT, 1, 2>(d, 256);
    // Strips of 8 vectors and of 16 (wide): 4096 x 1024 half 12.0 and 14.9, binary32 (67 MB) 19.2 and 18.1, 8192 x 1024 binary32 41 and 33, 4096 x
    // 4096 half 44 and 34. H kept in the caches and not: 4096 x 4096 half 41.0 and 33.6, with a reader of Y and a later one of H behind it 72.5 and
    // 69.2; 2048 x 4096 (67 MB) with the readers 37.0 and 38.4.
    constexpr int64_t wide = V * kWideLanes;
    if (bytes > 40e6 && d.batch * (d.N / wide) * (kPartThreads / wide * kPartsAtOnce) >= 256)
        return bytes > 100e6 ? split_with<T, QUANT, V, kWideLanes, true>(d, 512) : split_with<T, QUANT, V, kWideLanes>(d, 512);
    return d.N > 4 * V ? split_with<T, QUANT, V, 8>(d, 256) : d.N > 2 * V ? split_with<T, QUANT, V, 4>(d, 256)
         : d.N > V ? split_with<T, QUANT, V, 2>(d, 256) : split_with<T, QUANT, V, 1>(d, 256);
}

SplitNorm split_norm(const sparsert_norm &d) {
    const bool half = d.dtype == SPARSERT_F16, quant = d.out_dtype == SPARSERT_I8;
    return half ? quant ? split_of<_Float16, true>(d) : split_of<_Float16, false>(d) : quant ? split_of<float, true>(d) : split_of<float, false>(d);
}

}  // namespace

size_t norm_workspace(const sparsert_norm &d) {
    const SplitNorm s = split_norm(d);
    return s.parts ? (size_t)d.batch * s.parts * (d.out_dtype == SPARSERT_I8 ? 2 : 1) * d.N * sizeof(float) : 0;
}

int launch_norm(const NormCall &c, std::string &err) {
    const sparsert_norm &d = c.d;
    NormArgs a{c.X, c.R, c.gamma, c.H, c.Y, c.scale, d.K, d.N, d.ldx, d.ldh, d.ldy, d.eps, c.workspace, 0, 0};
    if (c.workspace)
        if (const SplitNorm s = split_norm(d); s.parts) {
            a.parts = s.parts; a.rows = s.rows;
            const dim3 grid((uint32_t)((s.strips * s.parts + 7) / 8 * 8), (uint32_t)d.batch);
            if (int rc = launch_operator(s.sums, grid, kPartThreads, a, c.stream, err)) return rc;
            return launch_operator(s.results, grid, kPartThreads, a, c.stream, err);
        }
    int columns = 1;
    const bool half = d.dtype == SPARSERT_F16, quant = d.out_dtype == SPARSERT_I8;
    const void *kernel = half ? quant ? norm_of<_Float16, true>(d, columns) : norm_of<_Float16, false>(d, columns)
                              : quant ? norm_of<float, true>(d, columns) : norm_of<float, false>(d, columns);
    const int64_t strips = ((int64_t)d.N + columns - 1) / columns, workgroups = (strips + 7) / 8 * 8;
    if (int rc = check_launch(workgroups, kNormThreads, err)) return rc;
    return launch_operator(kernel, dim3((uint32_t)workgroups, (uint32_t)d.batch), kNormThreads, a, c.stream, err);
}

bool stream_of_current_device(void *stream) {
    if (reinterpret_cast<uintptr_t>(stream) <= 2) return true;   // the null stream and its per-thread form go by the current device
    hipDevice_t of = -1;
    int current = -1;
    if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &of) != hipSuccess || hipGetDevice(&current) != hipSuccess) return false;
    return of == current;
}

}  // namespace sparsert
