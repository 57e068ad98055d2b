// Root-mean-square norm over the features of every token, with the residual's addition and, for int8 products, quantisation.
#include <hip/hip_runtime.h>

#include <cmath>

#include "launch.h"
#include "operators.h"
#include "strips.h"

namespace sparsert {

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

template <int C> __device__ __forceinline__ float from_lane_xor(float v) {   // C: 1, 2, 4 or 8
    if constexpr (C == 8) return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));        // row_ror:8
    else if constexpr (C == 4) return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 4 << 10 | 0x1f));
    else return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), C == 2 ? 0x4e : 0xb1, 0xf, 0xf, false));           // quad_perm
}

// a of this lane's half with a of the other one, or b with b, whichever half this lane is in: two values become one.
template <bool MAX> __device__ __forceinline__ float join(float a, float b) { return MAX ? larger(a, b) : a + b; }
template <int C, bool MAX> __device__ __forceinline__ float halve(float a, float b, int lane) {
    if constexpr (C == 32 || C == 16) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        const auto s = C == 32 ? __builtin_amdgcn_permlane32_swap(x, y, false, false) : __builtin_amdgcn_permlane16_swap(x, y, false, false);
        return join<MAX>(__uint_as_float(s[0]), __uint_as_float(s[1]));
    } else {
        const bool upper = lane & C;
        return join<MAX>(upper ? b : a, from_lane_xor<C>(upper ? a : b));
    }
}

// Column sums (or largest values) of a wave whose lanes l, l + L, l + 2 L ... hold V columns each: the lanes give half of
// their columns away at every step, as long as they have more than one.  Returns that one; its number among the V: column_of.
template <int V, int L, bool MAX> __device__ __forceinline__ float over_rows(const float (&v)[V], int lane) {
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = v[i];
    constexpr int S1 = V >= 2 ? V / 2 : 0, S2 = V >= 4 ? V / 4 : 0, S3 = V >= 8 ? V / 8 : 0;
#pragma unroll
    for (int i = 0; i < S1; ++i) a[i] = halve<32, MAX>(a[i], a[i + S1], lane);
#pragma unroll
    for (int i = 0; i < S2; ++i) a[i] = halve<16, MAX>(a[i], a[i + S2], lane);
#pragma unroll
    for (int i = 0; i < S3; ++i) a[i] = halve<8, MAX>(a[i], a[i + S3], lane);
    float s = a[0];
    if constexpr (V < 2) s = halve<32, MAX>(s, s, lane);
    if constexpr (V < 4) s = halve<16, MAX>(s, s, lane);
    if constexpr (V < 8 && L <= 8) s = join<MAX>(s, from_lane_xor<8>(s));
    if constexpr (L <= 4) s = join<MAX>(s, from_lane_xor<4>(s));
    if constexpr (L <= 2) s = join<MAX>(s, from_lane_xor<2>(s));
    if constexpr (L <= 1) s = join<MAX>(s, from_lane_xor<1>(s));
    return s;
}
template <int V> __device__ __forceinline__ int column_of(int lane) { return V == 8 ? lane >> 3 & 7 : V == 4 ? lane >> 4 & 3 : V == 2 ? lane >> 5 : 0; }
// of the lanes with the same sum, the one that stores it
template <int V, int L> __device__ __forceinline__ bool stores(int lane) { return (lane & (64 / V - 1)) < L; }

// A workgroup of THREADS threads does a strip of V * L columns: thread t has the V columns of lane t % L in the rows t / L, t / L +
// THREADS / L, ...  PASSES of them are fetched at a time, all before the first is used.  HELD: they are all rows, and stay in
// registers; otherwise the rows are fetched twice, once for the sums and once for the results.
// WHOLE: every lane's V columns exist, as in all strips but a last one.
template <typename T, bool QUANT, int V, int L, int PASSES, bool HELD, int THREADS, bool WHOLE>
__device__ __forceinline__ void norm_strip(const NormArgs &a, int strip) {
    constexpr int W = V * L, WAVES = THREADS / 64, ROWS = THREADS / L;
    __shared__ __align__(16) float sums[WAVES][W], tops[QUANT ? WAVES : 1][W], factors[W];
    typedef typename std::conditional<QUANT, int8_t, T>::type Out;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, row = t / L, n = strip * W + t % L * V;
    const int valid = WHOLE ? V : a.N - n;   // columns of this lane; none (not positive) behind the last one
    const Matrix X(static_cast<const T *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, a.N, a.ldx, sizeof(T));
    const Matrix R(a.R ? static_cast<const T *>(a.R) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr, a.K, a.N, a.ldh, sizeof(T));
    const Matrix H(a.H ? static_cast<T *>(a.H) + (int64_t)blockIdx.y * a.K * a.ldh : nullptr, a.K, a.N, a.ldh, sizeof(T));
    const Matrix Y(static_cast<Out *>(a.Y) + (int64_t)blockIdx.y * a.K * a.ldy, a.K, a.N, a.ldy, sizeof(Out));
    const Matrix G(a.gamma, 1, a.K, a.K, sizeof(float));

    float h[PASSES][V], g[PASSES];
    auto place = [&](int k0, int i, int ld, int size, uint32_t &common) {   // this lane's byte in pass i of the rows from k0 on
        const int first = k0 + i * ROWS;
        common = first < a.K ? (uint32_t)first * (uint32_t)ld * (uint32_t)size : 0;
        return first + row < a.K && valid > 0 ? ((uint32_t)row * (uint32_t)ld + (uint32_t)n) * (uint32_t)size : kNowhere;
    };
    auto fetch = [&](int k0) {
        T x[PASSES][V], r[PASSES][V];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            uint32_t common;
            const uint32_t at = place(k0, i, a.ldx, sizeof(T), common);
            load<T, V>(X, at, common, valid, x[i]);
        }
        if (a.R) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                uint32_t common;
                const uint32_t at = place(k0, i, a.ldh, sizeof(T), common);
                load<T, V>(R, at, common, valid, r[i]);
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
            g[i] = a.gamma ? __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(G.at, k < a.K ? (uint32_t)k * 4u : kNowhere, 0, 0)) : 1.0f;
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) h[i][v] = (float)x[i][v] + (float)r[i][v];
    };
    auto write_sum = [&](int k0) {
        if (!a.H) return;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            T out[V];
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = (T)h[i][v];
            uint32_t common;
            const uint32_t at = place(k0, i, a.ldh, sizeof(T), common);
            store<T, V>(H, at, common, valid, out);
        }
    };
    float s[V], top[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = top[v] = 0.0f;
    auto add_up_and_weigh = [&]() {   // h becomes h * gamma
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[v] = __builtin_fmaf(h[i][v], h[i][v], s[v]);
                h[i][v] *= g[i];
                if constexpr (QUANT) top[v] = larger(top[v], fabsf(h[i][v]));
            }
    };
    float f[V];
    auto write = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            Out out[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (QUANT) out[v] = f[v] == 0.0f ? (int8_t)0 : (int8_t)(int)rintf(h[i][v] * f[v]);
                else out[v] = (T)(h[i][v] * f[v]);
            }
            uint32_t common;
            const uint32_t at = place(k0, i, a.ldy, sizeof(Out), common);
            store<Out, V>(Y, at, common, valid, out);
        }
    };

    if constexpr (HELD) {
        fetch(0);
        write_sum(0);
        add_up_and_weigh();
    } else {
        for (int k0 = 0; k0 < a.K; k0 += PASSES * ROWS) {
            fetch(k0);
            add_up_and_weigh();
        }
    }
    // Rows past K are zeros: they add nothing.  The sums meet in LDS, in wave order.
    const float mine = over_rows<V, L, false>(s, lane);
    float largest = 0.0f;
    if constexpr (QUANT) largest = over_rows<V, L, true>(top, lane);
    if (stores<V, L>(lane)) {
        sums[wave][lane % L * V + column_of<V>(lane)] = mine;
        if constexpr (QUANT) tops[wave][lane % L * V + column_of<V>(lane)] = largest;
    }
    __syncthreads();
    if (t < W) {
        float total = sums[0][t], most = 0.0f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) total += sums[w][t];
        const float inv = 1.0f / sqrtf(total / (float)a.K + a.eps);
        float factor = inv;
        if constexpr (QUANT) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = larger(most, tops[w][t]);
            const bool sound = total < INFINITY && most < INFINITY, some = most >= 0x1p-100f;
            factor = sound && some ? 127.0f / most : 0.0f;
            if (strip * W + t < a.N) a.scale[(size_t)blockIdx.y * a.N + strip * W + t] = !sound ? NAN : some ? most * inv / 127.0f : 0.0f;
        }
        factors[t] = factor;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = factors[t % L * V + v];
    if constexpr (HELD) {
        write(0);
    } else {
        for (int k0 = 0; k0 < a.K; k0 += PASSES * ROWS) {
            fetch(k0);
            write_sum(k0);
#pragma unroll
            for (int i = 0; i < PASSES; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v) h[i][v] *= g[i];
            write(k0);
        }
    }
}

template <typename T, bool QUANT, int V, int L, int PASSES, bool HELD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(const NormArgs a) {
    constexpr int W = V * L;
    const int strips = (a.N + W - 1) / W, strip = task_of(blockIdx.x, strips);
    if (strip >= strips) return;
    if (V == 1 || strip * W + W <= a.N) norm_strip<T, QUANT, V, L, PASSES, HELD, THREADS, V != 1>(a, strip);
    else if constexpr (V != 1) norm_strip<T, QUANT, V, L, PASSES, HELD, THREADS, false>(a, strip);
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

template <typename T, bool QUANT> const void *norm_of(const sparsert_norm &d, int &columns) {
    constexpr int V = 16 / sizeof(T);   // columns of a lane: 16 bytes
    if (d.N < V) {
        const int lanes = d.N > 4 ? 8 : d.N > 2 ? 4 : d.N;
        columns = lanes;
        return lanes == 8 ? norm_of<T, QUANT, 1, 8>(d.K) : lanes == 4 ? norm_of<T, QUANT, 1, 4>(d.K) : lanes == 2 ? norm_of<T, QUANT, 1, 2>(d.K) : norm_of<T, QUANT, 1, 1>(d.K);
    }
    const int64_t vectors = (int64_t)d.batch * ((d.N + V - 1) / V);
    const int lanes = vectors >= 8 * 256 ? 8 : vectors >= 4 * 256 ? 4 : vectors >= 2 * 256 ? 2 : 1;
    columns = lanes * V;
    return lanes == 8 ? norm_of<T, QUANT, V, 8>(d.K) : lanes == 4 ? norm_of<T, QUANT, V, 4>(d.K) : lanes == 2 ? norm_of<T, QUANT, V, 2>(d.K) : norm_of<T, QUANT, V, 1>(d.K);
}

}  // namespace

int launch_norm(const NormCall &c, std::string &err) {
    const sparsert_norm &d = c.d;
    NormArgs a{c.X, c.R, c.gamma, c.H, c.Y, c.scale, d.K, d.N, d.ldx, d.ldh, d.ldy, d.eps};
    int columns = 1;
    const bool half = d.dtype == SPARSERT_F16, quant = d.out_dtype == SPARSERT_I8;
    const void *kernel = half ? quant ? norm_of<_Float16, true>(d, columns) : norm_of<_Float16, false>(d, columns)
                              : quant ? norm_of<float, true>(d, columns) : norm_of<float, false>(d, columns);
    const int strips = (int)(((int64_t)d.N + columns - 1) / columns);
    return launch_operator(kernel, dim3((uint32_t)((strips + 7) / 8 * 8), (uint32_t)d.batch), kNormThreads, a, c.stream, err);
}

bool stream_of_current_device(void *stream) {
    if (reinterpret_cast<uintptr_t>(stream) <= 2) return true;   // the null stream and its per-thread form go by the current device
    hipDevice_t of = -1;
    int current = -1;
    if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &of) != hipSuccess || hipGetDevice(&current) != hipSuccess) return false;
    return of == current;
}

}  // namespace sparsert
