// Low-rank adapters of many requests beside a projection that they share, in two kernels:
//   shrink  t[n, j] = sum_k down[a][j, k] x[k, n]         for the adapter a of every token, over a part of the rows k
//   expand  Y[m, n] = c[m, n] + alpha[a] sum_j up[a][m, j] t[n, j]
// t lies in the caller's workspace, [batch * N][part][ranks, rounded up to 16], in binary32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>

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
    int32_t parts, slots;   // parts of K; workgroups that share the adapters of a tile of tokens
};

struct ExpandArgs {
    const void *C, *up;
    const int32_t *index;
    const float *alpha, *row, *col, *t;
    void *Y;
    int32_t M, N, ldc, ldy, count, parts;
    int32_t rows;          // of a workgroup,
    int16_t tokens, rank;  // and its tokens
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
    if ((int)blockIdx.x >= groups * a.parts) return;
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
    if (n0 >= a.N) return;
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

// ---- Many tokens: tiles of 64 on the matrix cores.
//
// A lane has four adjacent tokens, one of each of four 16-wide tiles, so that x, C and Y are read and written 4 tokens at a time.  An adapter's weights meet
// all tokens of a tile, of which only those that are its own take the result: nothing of another token or adapter reaches them.  Tokens of
// a request lie side by side, so that a tile meets one adapter or two; a tile of 64 requests takes 64 turns.

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;

// The tokens of a lane, and which adapter each of them has (-1: none).
struct TileTokens {
    Columns<4> columns;
    int id[4];
    __device__ __forceinline__ TileTokens(const int32_t *index, int count, int n0, int N, int lane) : columns(n0 + (lane & 15) * 4, N) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            id[c] = columns.any && c >= columns.skip ? index[(size_t)blockIdx.y * N + columns.first + c] : -1;
            if (id[c] >= count) id[c] = -1;
        }
    }
    // The adapters of the tile one after the other, each once: the next one, with its tokens taken out of `left`, or -1.  Uniform.
    static __device__ __forceinline__ int next(int (&left)[4]) {
        int a = -1;
#pragma unroll
        for (int c = 3; c >= 0; --c)
            if (const uint64_t have = __ballot(left[c] >= 0)) a = __builtin_amdgcn_readlane(left[c], __builtin_ctzll(have));
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (left[c] == a) left[c] = -1;
        return a;
    }
};

// Operands of the matrix cores.  half: 32 rows of K a step, eight adjacent ones in a lane.  float: 16 rows a step in four instructions, lane group g
// has rows 4 g ... 4 g + 3.
template <typename W> struct Step;
template <> struct Step<_Float16> {
    static constexpr int ROWS = 32, LANE = 8;
    typedef half8 frag;
    static __device__ __forceinline__ float4v mma(const frag &w, const frag &x, const float4v &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, c, 0, 0, 0); }
};
template <> struct Step<float> {
    static constexpr int ROWS = 16, LANE = 4;
    typedef float4v frag;
    static __device__ __forceinline__ float4v mma(const frag &w, const frag &x, float4v c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
        return c;
    }
};

constexpr int kShrinkWaves = 8;

// A workgroup does 64 tokens and a part of 8 * STEPS steps of K: wave w keeps its STEPS steps of x in registers and multiplies them with 16 ranks of an
// adapter at a time; the waves' sums meet in LDS.
template <typename X, typename W, int STEPS> __global__ __launch_bounds__(kShrinkWaves * 64, 2) void shrink_tiles_kernel(const ShrinkArgs a) {
    typedef Step<W> Q;
    typedef typename Q::frag frag;
    constexpr int WAVE_ROWS = STEPS * Q::ROWS, PART = kShrinkWaves * WAVE_ROWS;
    __shared__ __align__(16) float4v sums[2][kShrinkWaves][4][64];
    __shared__ int ids[kTile];
    const int tiles = (a.N + kTile - 1) / kTile, task = task_of(blockIdx.x, tiles * a.parts * a.slots);
    if (task >= tiles * a.parts * a.slots) return;
    const int slot = task % a.slots, part = task / a.slots % a.parts, n0 = task / a.slots / a.parts * kTile;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, i = lane & 15;
    const TileTokens tokens(a.index, a.count, n0, a.N, lane);
    int left[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) left[c] = tokens.id[c];
    auto next = [&]() {   // of this workgroup's adapters: every slots-th, from the slot-th on
        return TileTokens::next(left);
    };
    int id = -1;
    for (int skip = slot; skip >= 0; --skip) {
        id = next();
        if (id < 0) return;
    }
    if (wave == 0 && g == 0)
#pragma unroll
        for (int c = 0; c < 4; ++c) ids[i * 4 + c] = tokens.id[c];
    const int k0 = part * PART + wave * WAVE_ROWS;
    frag x[STEPS][4];
    {
        const Matrix from(static_cast<const X *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, a.N, a.ldx, sizeof(X));
        X v[STEPS][Q::LANE][4];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < Q::LANE; ++e) {
                const int k = k0 + s * Q::ROWS + g * Q::LANE + e;
                load<X, 4>(from, k < a.K && tokens.columns.any ? ((uint32_t)k * (uint32_t)a.ldx + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(X) : kNowhere, 0, v[s][e]);
            }
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < Q::LANE; ++e) x[s][c][e] = (W)v[s][e][c];
    }
    const int ranks = ranks16(a.rank);
    const bool whole = k0 + WAVE_ROWS <= a.K || a.K % Q::LANE == 0;   // no lane's rows end before they do
    auto fetch = [&](int id, int j0, frag (&w)[STEPS]) {
        const Matrix down(static_cast<const W *>(a.down) + (size_t)id * a.rank * a.K, a.rank, a.K, a.K, sizeof(W));
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int k = k0 + s * Q::ROWS + g * Q::LANE;
            W v[Q::LANE];
            weights<W, Q::LANE>(down, j0 + i < a.rank && k < a.K ? (uint32_t)(j0 + i) * (uint32_t)a.K * (uint32_t)sizeof(W) : kNowhere, k, a.K, whole, v);
#pragma unroll
            for (int e = 0; e < Q::LANE; ++e) w[s][e] = v[e];
        }
    };
    frag w[STEPS];
    fetch(id, 0, w);
    for (int turn = 0, j0 = 0; id >= 0; ++turn) {
        float4v acc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            acc[c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) acc[c] = Q::mma(w[s], x[s][c], acc[c]);
        }
        const int of = id, at = j0;
        j0 += 16;
        if (j0 >= ranks) {
            j0 = 0;
            for (int skip = a.slots; skip > 0 && id >= 0; --skip) id = next();
        }
        if (id >= 0) fetch(id, j0, w);   // the next turn's weights are on their way while the sums meet
        float4v(*const mine)[4][64] = sums[turn & 1];
#pragma unroll
        for (int c = 0; c < 4; ++c) mine[wave][c][lane] = acc[c];
        __syncthreads();   // (the buffer of the turn before last was read before the last turn's barrier)
        // Thread t: two ranks of a token, the waves' sums in their order.
        const int item = t >> 1, c = item >> 6, l = item & 63, n = min(n0 + (l & 15) * 4, a.N - 4) + c;
        if (ids[(l & 15) * 4 + c] == of) {
            float2 sum = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < kShrinkWaves; ++v) {
                const float2 u = *(reinterpret_cast<const float2 *>(&mine[v][c][l]) + (t & 1));
                sum.x += u.x;
                sum.y += u.y;
            }
            float *const to = a.t + (((size_t)blockIdx.y * a.N + n) * a.parts + part) * ranks + at + (l >> 4) * 4 + (t & 1) * 2;
            *reinterpret_cast<float2 *>(to) = sum;
        }
    }
}

constexpr int kExpandTileThreads = 256;

// A workgroup does 64 tokens and `rows` rows of Y, its waves 16 of them at a time.
// half: t is split into two halves, t = hi + lo, which the instruction's 32 steps take side by side for 16 ranks, beside the same 16 weights
// twice: 22 bits of t, at a sixteenth of what binary32 instructions cost.  Every token's t is scaled by a power of two first, its largest
// to 2^14 ... 2^15, so that neither half leaves its range: what lo loses below 2^-24 is 2^-39 of that largest.
template <typename C, typename W, int RB> __global__ __launch_bounds__(kExpandTileThreads) void expand_tiles_kernel(const ExpandArgs a) {
    constexpr bool SCALED = std::is_same<C, int32_t>::value, HALF = std::is_same<W, _Float16>::value;
    typedef Step<W> Q;
    typedef typename Q::frag frag;
    constexpr int PITCH = RB * 16 + 4;
    __shared__ __align__(16) float ts[kTile * PITCH];
    __shared__ int exponents[kTile], list[kTile];
    const int tiles = (a.N + kTile - 1) / kTile, chunks = (a.M + a.rows - 1) / a.rows, task = task_of(blockIdx.x, tiles * chunks);
    if (task >= tiles * chunks) return;
    const int n0 = task % tiles * kTile, m0 = task / tiles * a.rows, end = min(a.M, m0 + a.rows);
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, i = lane & 15;
    const TileTokens tokens(a.index, a.count, n0, a.N, lane);
    int count = 0;
    {
        int left[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) left[c] = tokens.id[c];
        for (int id = TileTokens::next(left); id >= 0; id = TileTokens::next(left)) {
            if (t == 0) list[count] = id;
            ++count;
        }
    }
    // ts[token]: by the tokens' order in the lanes, which a last tile's shifted columns change nothing about
    gather_t<SCALED>(a, n0, min(kTile, a.N - n0), kExpandTileThreads, ts, PITCH);
    __syncthreads();
    if constexpr (HALF) {   // the tokens' exponents: four threads to a token
        float top = 0.0f;
        for (int j = t & 3; j < RB * 16; j += 4)
            if (j < ranks16(a.rank) && n0 + (t >> 2) < a.N) top = larger(top, fabsf(ts[(t >> 2) * PITCH + j]));
        top = larger(top, from_lane_xor<1>(top));
        top = larger(top, from_lane_xor<2>(top));
        if ((t & 3) == 0) exponents[t >> 2] = top > 0.0f && top < INFINITY ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
        __syncthreads();
    }
    frag x[RB][4];
    int down[4];   // the tokens' scaling, to be undone
    const int ranks = ranks16(a.rank);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int of = tokens.columns.first + c - n0;   // its row in ts: before the tile where a lane's first columns are not its own
        const bool have = tokens.id[c] >= 0;
        down[c] = HALF && have ? -exponents[of] : 0;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int e = 0; e < Q::LANE; ++e) {
                const int j = b * 16 + (HALF ? (g & 1) * 8 : g * 4) + e;
                const float v = have && j < ranks ? ts[of * PITCH + j] : 0.0f;
                if constexpr (HALF) {
                    const float scaled = __builtin_ldexpf(v, -down[c]);
                    const _Float16 hi = (_Float16)scaled;
                    const float rest = scaled - (float)hi;
                    x[b][c][e] = g < 2 ? hi : rest - rest == 0.0f ? (_Float16)rest : (_Float16)0.0f;   // (an infinity has no rest)
                } else {
                    x[b][c][e] = v;
                }
            }
    }
    float col[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) col[c] = SCALED && a.col && tokens.columns.any ? a.col[(size_t)blockIdx.y * a.N + tokens.columns.first + c] : 1.0f;
    const Matrix from(static_cast<const C *>(a.C) + (int64_t)blockIdx.y * a.M * a.ldc, a.M, a.N, a.ldc, sizeof(C));
    const Matrix Y(static_cast<W *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, a.N, a.ldy, sizeof(W));
    const Matrix rows(a.row, 1, a.M, a.M, 4);
    const bool whole = a.rank % Q::LANE == 0;
    for (int m = m0 + wave * 16; m < end; m += kExpandTileThreads / 64 * 16) {
        C had[4][4];
        float row[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at = m + g * 4 + q;
            load<C, 4>(from, at < end && tokens.columns.any ? ((uint32_t)at * (uint32_t)a.ldc + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(C) : kNowhere, 0, had[q]);
            float one[1] = {1.0f};
            if (SCALED && a.row) load<float, 1>(rows, at < end ? (uint32_t)at * 4u : kNowhere, 0, one);
            row[q] = one[0];
        }
        float add[4][4];   // [row][token]
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c) add[q][c] = -0.0f;   // (what is added to nothing leaves it as it is)
        for (int o = 0; o < count; ++o) {
            const int id = __builtin_amdgcn_readfirstlane(list[o]);
            const Matrix up(static_cast<const W *>(a.up) + (size_t)id * a.M * a.rank, a.M, a.rank, a.rank, sizeof(W));
            frag w[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int j = b * 16 + (HALF ? (g & 1) * 8 : g * 4);
                W v[Q::LANE];
                weights<W, Q::LANE>(up, m + i < a.M && j < a.rank ? (uint32_t)(m + i) * (uint32_t)a.rank * (uint32_t)sizeof(W) : kNowhere, j, a.rank, whole, v);
#pragma unroll
                for (int e = 0; e < Q::LANE; ++e) w[b][e] = v[e];
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int b = 0; b < RB; ++b) acc = Q::mma(w[b], x[b][c], acc);
                if (tokens.id[c] == id)
#pragma unroll
                    for (int q = 0; q < 4; ++q) add[q][c] = HALF ? __builtin_ldexpf(acc[q], down[c]) : acc[q];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at = m + g * 4 + q;
            float c4[4];
            W y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) c4[c] = (float)had[q][c];
            finish<C, W, 4>(c4, col, row[q], add[q], y);
            store<W, 4>(Y, at < end && tokens.columns.any ? ((uint32_t)at * (uint32_t)a.ldy + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(W) : kNowhere, 0,
                        tokens.columns.any ? tokens.columns.skip : 0, y);
        }
    }
}

namespace {

struct Plan {   // the kernels of a call, and what they go by
    const void *shrink, *expand;
    int parts, slots, tokens, rows;
    int64_t shrink_grid, expand_grid;
    int shrink_threads, expand_threads, expand_lds;
};

template <typename X, typename C, typename W> Plan plan_of(const sparsert_adapter_set &d) {
    Plan p{};
    const int ranks = (d.rank + 15) / 16 * 16;
    static const int mode = getenv("AD_MODE") ? atoi(getenv("AD_MODE")) : 0;
    static const int want = getenv("AD_WG") ? atoi(getenv("AD_WG")) : 128;
    static const int ewant = getenv("AD_EWG") ? atoi(getenv("AD_EWG")) : 512;
    if (d.N >= 4 && d.rank <= 64 && (mode == 2 || (mode == 0 && (int64_t)d.N * d.batch > 64))) {
        const int64_t tiles = ((int64_t)d.N + kTile - 1) / kTile;
        constexpr int unit = kShrinkWaves * Step<W>::ROWS;
        int steps = 4;
        auto parts = [&]() { return (d.K + unit * steps - 1) / (unit * steps); };
        while (steps > 1 && tiles * d.batch * parts() < want) steps /= 2;
        p.parts = parts();
        p.slots = (int)std::min<int64_t>({8, d.count, std::max<int64_t>(1, 2 * want / (tiles * d.batch * p.parts))});
        p.shrink = steps == 4 ? (const void *)shrink_tiles_kernel<X, W, 4> : steps == 2 ? (const void *)shrink_tiles_kernel<X, W, 2> : (const void *)shrink_tiles_kernel<X, W, 1>;
        p.shrink_grid = tiles * p.parts * p.slots; p.shrink_threads = kShrinkWaves * 64;
        p.expand = ranks <= 16 ? (const void *)expand_tiles_kernel<C, W, 1> : ranks <= 32 ? (const void *)expand_tiles_kernel<C, W, 2> : (const void *)expand_tiles_kernel<C, W, 4>;
        p.tokens = kTile;
        const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>((d.M + 63) / 64, ewant / (tiles * d.batch)));
        p.rows = (int)(((d.M + chunks - 1) / chunks + 63) / 64 * 64);
        p.expand_grid = tiles * ((d.M + p.rows - 1) / p.rows); p.expand_threads = kExpandTileThreads;
        return p;
    }
    p.parts = (d.K + kTokenRows - 1) / kTokenRows;
    p.tokens = std::min(kExpandTokens, 8192 / ranks);   // t of 32 KiB at most in LDS
    p.rows = kExpandRows;
    p.shrink = d.N < kTokenGroup ? (const void *)shrink_tokens_kernel<X, W, 1> : (const void *)shrink_tokens_kernel<X, W, kTokenGroup>;
    p.expand = (const void *)expand_tokens_kernel<C, W>;
    p.shrink_grid = ((int64_t)d.N + kTokenGroup - 1) / kTokenGroup * p.parts; p.shrink_threads = kTokenThreads;
    p.expand_grid = ((int64_t)d.N + p.tokens - 1) / p.tokens * ((d.M + p.rows - 1) / p.rows); p.expand_threads = kExpandThreads;
    p.expand_lds = (kExpandRows * (kExpandTokens + 1) + 16 + p.tokens * ranks) * (int)sizeof(float);
    return p;
}

Plan plan_of(const sparsert_adapter_set &d) {
    const bool half = d.dtype == SPARSERT_F16;
    if (d.x_dtype == SPARSERT_I8) return half ? plan_of<int8_t, int32_t, _Float16>(d) : plan_of<int8_t, int32_t, float>(d);
    return half ? plan_of<_Float16, _Float16, _Float16>(d) : plan_of<float, float, float>(d);
}

}  // namespace

size_t adapters_workspace(const sparsert_adapter_set &d) { return (size_t)d.batch * d.N * plan_of(d).parts * ((d.rank + 15) / 16 * 16) * sizeof(float); }

int launch_adapters(const AdaptersCall &c, std::string &err) {
    const sparsert_adapter_set &d = c.d;
    const Plan p = plan_of(d);
    if (p.shrink_grid >= 1ll << 30 || p.expand_grid >= 1ll << 30) { err = "too many workgroups"; return SPARSERT_EUNSUPPORTED; }
    float *const t = static_cast<float *>(c.workspace);
    ShrinkArgs s{c.X, c.down, c.index, t, d.K, d.N, d.ldx, d.rank, d.count, p.parts, p.slots};
    const auto grid = [&](int64_t n) { return dim3((uint32_t)((n + 7) / 8 * 8), (uint32_t)d.batch); };
    if (int rc = launch_operator(p.shrink, grid(p.shrink_grid), p.shrink_threads, s, c.stream, err)) return rc;
    ExpandArgs e{c.C, c.up, c.index, c.alpha, c.row, c.col, t, c.Y, d.M, d.N, d.ldc, d.ldy, d.count, p.parts, p.rows, (int16_t)p.tokens, (int16_t)d.rank};
    return launch_operator(p.expand, grid(p.expand_grid), p.expand_threads, e, c.stream, err, p.expand_lds);
}

}  // namespace sparsert
