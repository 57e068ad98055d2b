// Low-rank adapters of many requests beside a projection that they share, in two kernels:
//   shrink  t[n, j] = sum_k down[a][j, k] x[k, n]         for the adapter a of every token, over a part of the rows k
//   expand  Y[m, n] = c[m, n] + alpha[a] sum_j up[a][m, j] t[n, j]
// t lies in the caller's workspace, [batch * N][part][ranks, rounded up to 16], in binary32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "launch.h"
#include "operators.h"
#include "strips.h"
#include "wave_sums.h"

namespace sparsert {

struct ShrinkArgs {
    const void *X, *down;
    const int32_t *index;
    float *t;
    int32_t K, N, ldx, rank, count;
    int32_t parts, rows;   // parts of K, rows of each
};

struct ExpandArgs {
    const void *C, *up;
    const int32_t *index;
    const float *alpha, *row, *col, *t;
    void *Y;
    int32_t M, N, ldc, ldy, rank, count, parts;
    int32_t tokens;   // of a workgroup
};

__device__ __forceinline__ int ranks16(int rank) { return (rank + 15) & ~15; }

// V adjacent weights of a row from element `at` of it on: all in range if `whole`, else those before `end` and zeros.  (What lies behind a row is the
// next one, and may be infinite: it has to be left out, not multiplied by zero.)
template <typename W, int V> __device__ __forceinline__ void weights(const Matrix &m, uint32_t row_at, int at, int end, bool whole, W (&to)[V]) {
    constexpr int PIECE = 16 / sizeof(W);
    if (whole) {
#pragma unroll
        for (int p = 0; p < V / PIECE; ++p) {
            W piece[PIECE];
            load<W, PIECE>(m, row_at + (uint32_t)(at + p * PIECE) * (uint32_t)sizeof(W), 0, piece);
#pragma unroll
            for (int i = 0; i < PIECE; ++i) to[p * PIECE + i] = piece[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            W one[1];
            load<W, 1>(m, at + i < end ? row_at + (uint32_t)(at + i) * (uint32_t)sizeof(W) : kNowhere, 0, one);
            to[i] = one[0];
        }
    }
}

// ---- Few tokens: every token on its own.

constexpr int kTokenGroup = 8, kTokenRows = 512, kTokenThreads = 512;   // tokens and rows of x of a workgroup; a wave for each token

// The group's x goes to LDS once, whole rows of eight tokens at a time (V = 8; 1: fewer than eight tokens); then wave w has token w, and its lane l the rows 8 l ... 8 l + 7,
// which it multiplies with 16 rows of `down` at a time.
template <typename X, typename W, int V> __global__ __launch_bounds__(kTokenThreads) void shrink_tokens_kernel(const ShrinkArgs a) {
    __shared__ __align__(16) float xs[kTokenGroup][kTokenRows + 4];
    const int groups = (a.N + kTokenGroup - 1) / kTokenGroup;
    const int group = blockIdx.x % groups, part = blockIdx.x / groups, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int n0 = group * kTokenGroup, k0 = part * kTokenRows, n = n0 + wave;
    const int id = n < a.N ? a.index[(size_t)blockIdx.y * a.N + n] : -1;
    {
        const Matrix x(static_cast<const X *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, a.N, a.ldx, sizeof(X));
        const int k = k0 + t;
        if constexpr (V == kTokenGroup) {
            const Columns<V> columns(n0, a.N);
            constexpr int PIECE = sizeof(X) * V > 16 ? 16 / (int)sizeof(X) : V;
#pragma unroll
            for (int p = 0; p < V / PIECE; ++p) {
                X v[PIECE];
                load<X, PIECE>(x, k < a.K ? ((uint32_t)k * (uint32_t)a.ldx + (uint32_t)(columns.first + p * PIECE)) * (uint32_t)sizeof(X) : kNowhere, 0, v);
#pragma unroll
                for (int i = 0; i < PIECE; ++i)
                    if (p * PIECE + i >= columns.skip) xs[p * PIECE + i - columns.skip][t] = (float)v[i];
            }
        } else {
            for (int c = 0; c < a.N; ++c) {
                X v[1];
                load<X, 1>(x, k < a.K ? ((uint32_t)k * (uint32_t)a.ldx + (uint32_t)c) * (uint32_t)sizeof(X) : kNowhere, 0, v);
                xs[c][t] = (float)v[0];
            }
        }
    }
    __syncthreads();
    if (id < 0 || id >= a.count) return;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = xs[wave][lane * 8 + i];
    const int ranks = ranks16(a.rank), k = k0 + lane * 8;
    const bool whole = k0 + kTokenRows <= a.K || a.K % 8 == 0;   // no lane's eight rows end before it does
    const Matrix down(static_cast<const W *>(a.down) + (size_t)id * a.rank * a.K, a.rank, a.K, a.K, sizeof(W));
    float *const to = a.t + (((size_t)blockIdx.y * a.N + n) * a.parts + part) * ranks;
    for (int j0 = 0; j0 < ranks; j0 += 16) {
        W w[16][8];
        float s[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) weights<W, 8>(down, j0 + j < a.rank && k < a.K ? (uint32_t)(j0 + j) * (uint32_t)a.K * (uint32_t)sizeof(W) : kNowhere, k, a.K, whole, w[j]);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j] = __builtin_fmaf((float)w[j][i], x[i], s[j]);
        }
        float sum[1];
        over_rows<16, 1, false>(s, lane, sum);
        if (stores<16, 1>(lane)) to[j0 + column_of<16, 1>(lane)] = sum[0];
    }
}

// t of `tokens` tokens from n0 on, its parts added up in order, times everything that does not depend on the row, to LDS; zeros for tokens without adapter.
template <bool SCALED> __device__ __forceinline__ void gather_t(const ExpandArgs &a, int n0, int tokens, int threads, float *ts, int pitch) {
    const int ranks = ranks16(a.rank);
    for (int i = threadIdx.x; i < tokens * ranks; i += threads) {
        const int c = i / ranks, j = i - c * ranks, n = n0 + c;
        float s = 0.0f;
        const int id = n < a.N ? a.index[(size_t)blockIdx.y * a.N + n] : -1;
        if (id >= 0 && id < a.count) {
            const float *from = a.t + ((size_t)blockIdx.y * a.N + n) * a.parts * ranks + j;
            for (int p0 = 0; p0 < a.parts; p0 += 8) {
                float u[8];
#pragma unroll
                for (int p = 0; p < 8; ++p) u[p] = p0 + p < a.parts ? from[(size_t)(p0 + p) * ranks] : 0.0f;
#pragma unroll
                for (int p = 0; p < 8; ++p) s += u[p];
            }
            if (a.alpha) s *= a.alpha[id];
            if (SCALED && a.col) s *= a.col[(size_t)blockIdx.y * a.N + n];
        }
        ts[c * pitch + j] = s;
    }
}

// Y of V tokens of a row: the projection's result, scaled, and what the adapter adds.
template <typename C, typename W, int V> __device__ __forceinline__ void finish(const float (&c)[V], const float (&col)[V], float row, const float (&add)[V], W (&y)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = (W)((std::is_same<C, int32_t>::value ? c[v] * col[v] * row : c[v]) + add[v]);
}

// A workgroup does 64 rows of Y for up to 64 tokens: a wave takes a token, its lane l row l; the sums meet the rows of C through LDS, so that both are read and written along the rows.
constexpr int kExpandTokens = 64, kExpandRows = 64, kExpandThreads = 1024;

template <typename C, typename W> __global__ __launch_bounds__(kExpandThreads) void expand_tokens_kernel(const ExpandArgs a) {
    constexpr bool SCALED = std::is_same<C, int32_t>::value;
    extern __shared__ __align__(16) float lds[];
    float *const ys = lds;                                                  // [row][token], rows 65 apart
    const int ranks = ranks16(a.rank);
    float *const ts = lds + kExpandRows * (kExpandTokens + 1) + 16 - (kExpandRows * (kExpandTokens + 1)) % 16;   // [token][rank]
    const int blocks = (a.M + kExpandRows - 1) / kExpandRows, m0 = (int)(blockIdx.x % blocks) * kExpandRows, n0 = (int)(blockIdx.x / blocks) * a.tokens;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), tokens = min(a.tokens, a.N - n0);
    gather_t<SCALED>(a, n0, tokens, kExpandThreads, ts, ranks);
    __syncthreads();
    for (int c = wave; c < tokens; c += kExpandThreads / 64) {
        const int id = __builtin_amdgcn_readfirstlane(a.index[(size_t)blockIdx.y * a.N + n0 + c]);
        float s = -0.0f;   // (what is added to nothing leaves it as it is)
        if (id >= 0 && id < a.count) {
            const Matrix up(static_cast<const W *>(a.up) + (size_t)id * a.M * a.rank, a.M, a.rank, a.rank, sizeof(W));
            const uint32_t row_at = m0 + lane < a.M ? (uint32_t)(m0 + lane) * (uint32_t)a.rank * (uint32_t)sizeof(W) : kNowhere;
            s = 0.0f;
            for (int j0 = 0; j0 < a.rank; j0 += 16) {
                W u[2][8];
                weights<W, 8>(up, row_at, j0, a.rank, j0 + 8 <= a.rank, u[0]);
                weights<W, 8>(up, row_at, j0 + 8, a.rank, j0 + 16 <= a.rank, u[1]);
#pragma unroll
                for (int i = 0; i < 16; ++i) s = __builtin_fmaf((float)u[i / 8][i % 8], ts[c * ranks + j0 + i], s);
            }
        }
        ys[lane * (kExpandTokens + 1) + c] = s;
    }
    __syncthreads();
    const Matrix from(static_cast<const C *>(a.C) + (int64_t)blockIdx.y * a.M * a.ldc, a.M, a.N, a.ldc, sizeof(C));
    const Matrix Y(static_cast<W *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, a.N, a.ldy, sizeof(W));
    for (int i = t; i < kExpandRows * tokens; i += kExpandThreads) {
        const int r = i / tokens, c = i - r * tokens, m = m0 + r;
        if (m >= a.M) continue;
        C had[1];
        load<C, 1>(from, ((uint32_t)m * (uint32_t)a.ldc + (uint32_t)(n0 + c)) * (uint32_t)sizeof(C), 0, had);
        const float c1[1] = {(float)had[0]}, col[1] = {SCALED && a.col ? a.col[(size_t)blockIdx.y * a.N + n0 + c] : 1.0f};
        const float add[1] = {ys[r * (kExpandTokens + 1) + c]};
        W y[1];
        finish<C, W, 1>(c1, col, SCALED && a.row ? a.row[m] : 1.0f, add, y);
        store<W, 1>(Y, ((uint32_t)m * (uint32_t)a.ldy + (uint32_t)(n0 + c)) * (uint32_t)sizeof(W), 0, 0, y);
    }
}

namespace {

struct Kernels { const void *shrink, *expand; };

template <typename X, typename C, typename W> Kernels token_kernels(bool few) {
    return {few ? (const void *)shrink_tokens_kernel<X, W, 1> : (const void *)shrink_tokens_kernel<X, W, kTokenGroup>, (const void *)expand_tokens_kernel<C, W>};
}

int parts_of(const sparsert_adapter_set &d) { return (d.K + kTokenRows - 1) / kTokenRows; }

}  // namespace

size_t adapters_workspace(const sparsert_adapter_set &d) { return (size_t)d.batch * d.N * parts_of(d) * ((d.rank + 15) / 16 * 16) * sizeof(float); }

int launch_adapters(const AdaptersCall &c, std::string &err) {
    const sparsert_adapter_set &d = c.d;
    const bool half = d.dtype == SPARSERT_F16, i8 = d.x_dtype == SPARSERT_I8, few = d.N < kTokenGroup;
    const Kernels k = i8 ? half ? token_kernels<int8_t, int32_t, _Float16>(few) : token_kernels<int8_t, int32_t, float>(few)
                         : half ? token_kernels<_Float16, _Float16, _Float16>(few) : token_kernels<float, float, float>(few);
    const int parts = parts_of(d), ranks = (d.rank + 15) / 16 * 16, tokens = std::min(kExpandTokens, 8192 / ranks);   // t of 32 KiB at most in LDS
    const int64_t groups = ((int64_t)d.N + kTokenGroup - 1) / kTokenGroup, tiles = ((int64_t)d.N + tokens - 1) / tokens;
    const int64_t blocks = ((int64_t)d.M + kExpandRows - 1) / kExpandRows;
    if (groups * parts >= 1ll << 31 || tiles * blocks >= 1ll << 31) { err = "too many workgroups"; return SPARSERT_EUNSUPPORTED; }
    ShrinkArgs s{c.X, c.down, c.index, static_cast<float *>(c.workspace), d.K, d.N, d.ldx, d.rank, d.count, parts, kTokenRows};
    if (int rc = launch_operator(k.shrink, dim3((uint32_t)(groups * parts), (uint32_t)d.batch), kTokenThreads, s, c.stream, err)) return rc;
    ExpandArgs e{c.C, c.up, c.index, c.alpha, c.row, c.col, static_cast<float *>(c.workspace), c.Y, d.M, d.N, d.ldc, d.ldy, d.rank, d.count, parts, tokens};
    const int bytes = (kExpandRows * (kExpandTokens + 1) + 16 + tokens * ranks) * (int)sizeof(float);
    return launch_operator(k.expand, dim3((uint32_t)(tiles * blocks), (uint32_t)d.batch), kExpandThreads, e, c.stream, err, bytes);
}

}  // namespace sparsert
