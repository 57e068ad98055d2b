// Low-rank adapters of many requests beside a projection that they share, in two kernels:
//   shrink  t[n, j] = alpha[a] sum_k down[a][j, k] x[k, n]     for the adapter a of every token, over a part of the rows k
//   expand  Y[m, n] = c[m, n] + sum_j up[a][m, j] t[n, j]
// t lies in the caller's workspace, [batch * N][part][ranks, rounded up to 16], in binary32.  (The factors are in t, so that the second kernel
// fetches everything but `up` without waiting for an index.)
//
// Bounds: 2 rank (M + K) operations a token are little beside C and Y of a prompt, or beside the adapters' weights of a few tokens; small calls are
// the wait for memory, twice in each kernel.  One token, 1024 x 1024, rank 8: 3.5 us; 48 requests of 32 adapters, 4096 x 4096, rank 16: 8.6 us;
// 1024 tokens of prompts, 1024 -> 4096, rank 16: 11.2 us; 2048 tokens of int8, 4096 x 4096, rank 64: 37 us, 2.0 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "operators.h"
#include "strips.h"
#include "wave_sums.h"

namespace sparsert {

struct ShrinkArgs {
    const void *X, *down;
    const int32_t *index;
    const float *alpha, *col;
    float *t;
    int32_t K, N, ldx, rank, count;
    int32_t parts, turns, slots;   // parts of K, turns of a part; workgroups that share the adapters of a tile of tokens
};

struct ExpandArgs {
    const void *C, *up;
    const int32_t *index;
    const float *row, *col, *t;
    void *Y;
    int32_t M, N, ldc, ldy, count, parts;
    int32_t rows;          // of a workgroup
    int32_t rank;
};

__device__ __forceinline__ int ranks16(int rank) { return (rank + 15) & ~15; }

// 16 bytes of weights of a row of `end` elements, from element `at` on; zeros for those behind the row's end.  (There lies the next row, which may
// hold infinities: it has to be left out, not multiplied by zero.)  `whole`: no piece is cut short by the end.  A piece that is reads the row's
// last 16 bytes and moves them down.  A row shorter than that is read over its end, so it has an even number of halves: a range is checked in steps
// of four bytes.
template <typename W> struct Piece { W v[16 / sizeof(W)]; };
template <typename W> __device__ __forceinline__ Piece<W> piece(const Matrix &m, uint32_t row_at, uint32_t common, int at, int end, bool whole) {
    constexpr int LANE = 16 / sizeof(W), BITS = 8 * sizeof(W);
    Piece<W> p;
    if (whole) {
        load<W, LANE>(m, at < end ? row_at + (uint32_t)at * (uint32_t)sizeof(W) : kNowhere, common, p.v);
        return p;
    }
    const int from = max(min(at, end - LANE), 0);
    load<W, LANE>(m, at < end ? row_at + (uint32_t)from * (uint32_t)sizeof(W) : kNowhere, common, p.v);
    uint64_t u[2];
    __builtin_memcpy(u, p.v, 16);
    const int down = (at - from) * BITS, keep = (end - at) * BITS;   // (of lanes behind the end: nothing is there)
    if (end < LANE) {
        u[1] &= keep > 64 ? ~0ull >> (128 - keep & 63) : 0;
        u[0] &= keep >= 64 ? ~0ull : ~0ull >> (64 - keep & 63);
    } else if (at < end) {
        const uint64_t low = u[0], high = u[1];
        u[0] = down == 0 ? low : down < 64 ? low >> (down & 63) | high << (64 - down & 63) : high >> (down - 64 & 63);
        u[1] = down < 64 ? high >> (down & 63) : 0;
    }
    __builtin_memcpy(p.v, u, 16);
    return p;
}
// Can rows of `end` elements be read so?
template <typename W> bool pieces_fit(int end) { return end >= 16 / (int)sizeof(W) || end * sizeof(W) % 4 == 0; }

// The same for the kernels that multiply a lane's piece of many rows with numbers of its own: a piece that the end cuts short is the row's last 16
// bytes as they lie, without what belongs to the lane before, and the lane moves its numbers instead (2.6 us less than moving the weights, for 16
// rows of half weights).
template <typename W, bool WHOLE> struct Cut {
    static constexpr int LANE = 16 / sizeof(W), EACH = 4 / sizeof(W);
    int from, end;
    bool any;
    uint32_t keep[4];
    __device__ __forceinline__ Cut(int at, int end) : from(WHOLE ? at : max(min(at, end - LANE), 0)), end(end), any(at < end) {
        if constexpr (!WHOLE)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                keep[d] = 0;
#pragma unroll
                for (int h = 0; h < EACH; ++h)
                    if (from + d * EACH + h >= at && from + d * EACH + h < end) keep[d] |= EACH == 1 ? ~0u : 0xffffu << (h * 16);
            }
    }
    __device__ __forceinline__ bool keeps(int i) const { return WHOLE ? any : (keep[i / EACH] >> (i % EACH * 16) & 1) != 0; }
    __device__ __forceinline__ void load(const Matrix &m, uint32_t row_at, W (&to)[LANE]) const {
        const uint32_t at = any ? row_at + (uint32_t)from * (uint32_t)sizeof(W) : kNowhere;
        if (WHOLE || end >= LANE) {
            sparsert::load<W, LANE>(m, at, 0, to);
        } else {   // (ranges are checked in steps of four bytes, so that 16 bytes may leave out the last half of a matrix)
#pragma unroll
            for (int i = 0; i < LANE; ++i) {
                W one[1];
                sparsert::load<W, 1>(m, any && i < end ? at + (uint32_t)i * (uint32_t)sizeof(W) : kNowhere, 0, one);
                to[i] = one[0];
            }
        }
        if constexpr (!WHOLE) mask(to);
    }
    __device__ __forceinline__ void mask(W (&to)[LANE]) const {
        uint32_t u[4];
        __builtin_memcpy(u, to, 16);
#pragma unroll
        for (int d = 0; d < 4; ++d) u[d] &= keep[d];
        __builtin_memcpy(to, u, 16);
    }
};

// ---- Few tokens: every token on its own.

constexpr int kTokenGroup = 8, kTokenRows = 512, kTokenThreads = 512;   // tokens and rows of x of a workgroup; a wave for each token

// The group's x goes to LDS once, whole rows of eight tokens at a time (V = 8; 1: fewer than eight tokens); then wave w has token w, and its lane l
// the rows 8 l ... 8 l + 7, which it multiplies with 16 rows of `down`; other workgroups have the others.
template <typename X, typename W, int V, bool WHOLE> __global__ __launch_bounds__(kTokenThreads) void shrink_tokens_kernel(const ShrinkArgs a) {
    __shared__ __align__(16) float xs[kTokenGroup][kTokenRows + 4];
    const int groups = (a.N + kTokenGroup - 1) / kTokenGroup, ranks = ranks16(a.rank), blocks = ranks / 16;
    if ((int)blockIdx.x >= groups * a.parts * blocks) return;
    const int group = blockIdx.x % groups, part = blockIdx.x / groups % a.parts, j0 = blockIdx.x / groups / a.parts * 16, t = threadIdx.x,
        lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
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
                load<X, PIECE>(x, k < a.K ? ((uint32_t)k * (uint32_t)a.ldx + (uint32_t)(columns.first + p * PIECE)) * (uint32_t)sizeof(X) : kNowhere,
                               0, v);
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
    constexpr int LANE = 16 / (int)sizeof(W), PIECES = 8 / LANE;
    const Matrix down(static_cast<const W *>(a.down) + (size_t)id * a.rank * a.K, a.rank, a.K, a.K, sizeof(W));
    const float alpha = a.alpha ? a.alpha[id] : 1.0f, col = a.col ? a.col[(size_t)blockIdx.y * a.N + n] : 1.0f;
    float s[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = 0.0f;
    auto dots = [&](auto whole) {
        W w[PIECES][16][LANE];
        float x[PIECES][LANE];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const Cut<W, decltype(whole)::value> cut(k0 + lane * 8 + p * LANE, a.K);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                cut.load(down, j0 + j < a.rank ? (uint32_t)(j0 + j) * (uint32_t)a.K * (uint32_t)sizeof(W) : kNowhere, w[p][j]);
#pragma unroll
            for (int i = 0; i < LANE; ++i) x[p][i] = cut.keeps(i) ? xs[wave][cut.from - k0 + i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
#pragma unroll
                for (int i = 0; i < LANE; ++i) s[j] = __builtin_fmaf((float)w[p][j][i], x[p][i], s[j]);
    };
    if (WHOLE || k0 + kTokenRows <= a.K) dots(std::true_type{});
    else dots(std::false_type{});
    float sum[1];
    over_rows<16, 1, false>(s, lane, sum);
    if (stores<16, 1>(lane)) a.t[(((size_t)blockIdx.y * a.N + n) * a.parts + part) * ranks + j0 + column_of<16, 1>(lane)] = sum[0] * alpha * col;
}

// t of up to TOKENS tokens from n0 on to LDS, rows of `pitch`: the parts added up in order.  THREADS / TOKENS threads share a token, each of them
// with four adjacent ranks at a time, RANKS ranks in a turn.  Tokens without adapter get what happens to lie there.  Returns the largest finite |t|
// of this thread's.
template <int THREADS, int RANKS, int TOKENS = 64> struct GatherT {
    static constexpr int SHARE = THREADS / TOKENS, AT_ONCE = 4, OWN = RANKS / (SHARE * 4);
    static_assert(RANKS % (SHARE * 4) == 0 && OWN >= 1, "whole turns");
    const float4 *from;
    float4 u[AT_ONCE][OWN];
    int parts, ranks, c, share;
    bool mine;
    __device__ __forceinline__ void fetch(int j0, int p0) {
#pragma unroll
        for (int p = 0; p < AT_ONCE; ++p)
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int j = j0 + (share + i * SHARE) * 4;
                u[p][i] = mine && p0 + p < parts && j < ranks ? from[((p0 + p) * ranks + j) / 4] : float4{0.0f, 0.0f, 0.0f, 0.0f};
            }
    }
    static __device__ __forceinline__ float finite(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; }
    // Sends for the first of it.
    __device__ __forceinline__ GatherT(const ExpandArgs &a, int n0, int tokens)
        : parts(a.parts), ranks(ranks16(a.rank)), c((int)threadIdx.x / SHARE), share((int)threadIdx.x % SHARE), mine(c < tokens) {
        from = reinterpret_cast<const float4 *>(a.t + ((size_t)blockIdx.y * a.N + n0 + c) * parts * ranks);
        fetch(0, 0);
    }
    __device__ __forceinline__ float finish(float *ts, int pitch, int row) {   // row: of this thread's token
        float top = 0.0f;
        for (int j0 = 0; j0 < ranks; j0 += RANKS) {
            float4 s[OWN];
#pragma unroll
            for (int i = 0; i < OWN; ++i) s[i] = float4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int p0 = 0; p0 < parts; p0 += AT_ONCE) {
                if (j0 > 0 || p0 > 0) fetch(j0, p0);
#pragma unroll
                for (int p = 0; p < AT_ONCE; ++p)
#pragma unroll
                    for (int i = 0; i < OWN; ++i) s[i].x += u[p][i].x, s[i].y += u[p][i].y, s[i].z += u[p][i].z, s[i].w += u[p][i].w;
            }
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int j = j0 + (share + i * SHARE) * 4;
                if (mine && j < ranks) *reinterpret_cast<float4 *>(ts + row * pitch + j) = s[i];
                top = fmaxf(fmaxf(fmaxf(finite(s[i].x), finite(s[i].y)), fmaxf(finite(s[i].z), finite(s[i].w))), top);
            }
        }
        return top;
    }
};

// Y of V tokens of a row: the projection's result, scaled, and what the adapter adds.
template <typename C, typename W, int V>
__device__ __forceinline__ void finish(const float (&c)[V], const float (&col)[V], float row, const float (&add)[V], W (&y)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = (W)((std::is_same<C, int32_t>::value ? c[v] * col[v] * row : c[v]) + add[v]);
}

// A workgroup does 64 rows of Y for 16 * EACH tokens: a wave takes EACH of them, its lane l row l; the sums meet the rows of C through LDS, so that
// both are read and written along the rows.
constexpr int kExpandRows = 64, kExpandThreads = 1024, kExpandWaves = kExpandThreads / 64;

template <typename C, typename W, int EACH, bool WHOLE> __global__ __launch_bounds__(kExpandThreads) void expand_tokens_kernel(const ExpandArgs a) {
    constexpr int TOKENS = EACH * kExpandWaves, LANE = 16 / (int)sizeof(W), PIECES = 16 / LANE;
    constexpr bool SCALED = std::is_same<C, int32_t>::value;
    extern __shared__ __align__(16) float ts[];           // [token][rank]
    __shared__ float ys[kExpandRows * (TOKENS + 1)];      // [row][token]
    const int ranks = ranks16(a.rank);
    const int blocks = (a.M + kExpandRows - 1) / kExpandRows, m0 = (int)(blockIdx.x % blocks) * kExpandRows, n0 = (int)(blockIdx.x / blocks) * TOKENS;
    if (n0 >= a.N) return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), tokens = min(TOKENS, a.N - n0);
    // Everything that waits for nothing is on its way first: this thread's elements of C, the indices of its wave's tokens, t.
    constexpr int OWN = kExpandRows * TOKENS / kExpandThreads;   // elements of a thread
    const Matrix from(static_cast<const C *>(a.C) + (int64_t)blockIdx.y * a.M * a.ldc, a.M, a.N, a.ldc, sizeof(C));
    C had[OWN];
    int row[OWN], token[OWN], id[EACH];
#pragma unroll
    for (int q = 0; q < EACH; ++q) id[q] = wave + q * kExpandWaves < tokens ? a.index[(size_t)blockIdx.y * a.N + n0 + wave + q * kExpandWaves] : -1;
    constexpr int TURN = 4 * kExpandThreads / TOKENS;   // ranks
    GatherT<kExpandThreads, TURN, TOKENS> gather(a, n0, tokens);
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = t + o * kExpandThreads;
        row[o] = i / tokens;
        token[o] = i - row[o] * tokens;
        C one[1];
        load<C, 1>(from, row[o] < kExpandRows && m0 + row[o] < a.M
                       ? ((uint32_t)(m0 + row[o]) * (uint32_t)a.ldc + (uint32_t)(n0 + token[o])) * (uint32_t)sizeof(C) : kNowhere, 0, one);
        had[o] = one[0];
    }
    float s[EACH];
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        id[q] = __builtin_amdgcn_readfirstlane(id[q]);
        if (id[q] >= a.count) id[q] = -1;
        s[q] = id[q] >= 0 ? 0.0f : -0.0f;   // (what is added to nothing leaves it as it is)
    }
    for (int j0 = 0; j0 < a.rank; j0 += 16) {
        W u[EACH][PIECES][LANE];
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (id[q] >= 0) {
                const Matrix up(static_cast<const W *>(a.up) + (size_t)id[q] * a.M * a.rank, a.M, a.rank, a.rank, sizeof(W));
                const uint32_t row_at = m0 + lane < a.M ? (uint32_t)(m0 + lane) * (uint32_t)a.rank * (uint32_t)sizeof(W) : kNowhere;
#pragma unroll
                for (int p = 0; p < PIECES; ++p) Cut<W, WHOLE>(j0 + p * LANE, a.rank).load(up, row_at, u[q][p]);
            }
        if (j0 == 0) {
            gather.finish(ts, ranks, gather.c);
            __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (id[q] >= 0)
#pragma unroll
                for (int p = 0; p < PIECES; ++p) {
                    const Cut<W, WHOLE> cut(j0 + p * LANE, a.rank);
                    if (!cut.any) continue;
#pragma unroll
                    for (int i = 0; i < LANE; ++i)
                        if (cut.keeps(i)) s[q] = __builtin_fmaf((float)u[q][p][i], ts[(wave + q * kExpandWaves) * ranks + cut.from + i], s[q]);
                }
    }
#pragma unroll
    for (int q = 0; q < EACH; ++q) ys[lane * (TOKENS + 1) + wave + q * kExpandWaves] = s[q];
    __syncthreads();
    const Matrix Y(static_cast<W *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, a.N, a.ldy, sizeof(W));
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (row[o] < kExpandRows && m0 + row[o] < a.M) {
            const float c1[1] = {(float)had[o]}, col[1] = {SCALED && a.col ? a.col[(size_t)blockIdx.y * a.N + n0 + token[o]] : 1.0f};
            const float add[1] = {ys[row[o] * (TOKENS + 1) + token[o]]};
            W y[1];
            finish<C, W, 1>(c1, col, SCALED && a.row ? a.row[m0 + row[o]] : 1.0f, add, y);
            store<W, 1>(Y, ((uint32_t)(m0 + row[o]) * (uint32_t)a.ldy + (uint32_t)(n0 + token[o])) * (uint32_t)sizeof(W), 0, 0, y);
        }
}

// ---- One token: one kernel.  Every workgroup works t out for itself, as that is a few reads of `down` from L2, and less than a second kernel has
// to wait.

constexpr int kOneRank = 64, kOneSize = 1 << 16;   // most ranks; most elements of `down`
constexpr int kOneRows = 64, kOneThreads = 1024, kOneShare = kOneThreads / kOneRows;   // kOneShare: threads of a row of Y

struct OneArgs {
    const void *X, *down, *up;
    const int32_t *index;
    const float *alpha;
    const void *C;
    void *Y;
    const float *row, *col;
    int32_t M, K, ldx, ldc, ldy, rank, count;
};

// x goes to LDS; then a wave does a row of `down` at a time, and 16 threads a row of `up`.
template <typename X, typename C, typename W, bool WHOLE> __global__ __launch_bounds__(kOneThreads) void one_token_kernel(const OneArgs a) {
    constexpr bool SCALED = std::is_same<C, int32_t>::value;
    // PIECE: elements of a wave's load; AT_ONCE: loads on their way at a time
    constexpr int LANE = 16 / (int)sizeof(W), WAVES = kOneThreads / 64, PIECE = 64 * LANE, AT_ONCE = 8;
    extern __shared__ __align__(16) float xs[];   // K, rounded up
    __shared__ __align__(16) float ts[kOneRank];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int id = a.index[blockIdx.y];
    const bool some = (uint32_t)id < (uint32_t)a.count;
    const Matrix x(static_cast<const X *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, 1, a.ldx, sizeof(X));
    const Matrix from(static_cast<const C *>(a.C) + (int64_t)blockIdx.y * a.M * a.ldc, a.M, 1, a.ldc, sizeof(C));
    const int row = t / kOneShare, p = t % kOneShare, m = (int)blockIdx.x * kOneRows + row;
    C had[1];
    load<C, 1>(from, m < a.M && p == 0 ? (uint32_t)m * (uint32_t)a.ldc * (uint32_t)sizeof(C) : kNowhere, 0, had);
    float s = -0.0f;   // (what is added to nothing leaves it as it is)
    if (some) {
        for (int k = t; k < ((a.K + 7) & ~7); k += kOneThreads) {
            X v[1];
            load<X, 1>(x, k < a.K ? (uint32_t)k * (uint32_t)a.ldx * (uint32_t)sizeof(X) : kNowhere, 0, v);
            xs[k] = (float)v[0];
        }
        const Matrix up(static_cast<const W *>(a.up) + (size_t)id * a.M * a.rank, a.M, a.rank, a.rank, sizeof(W));
        const Matrix down(static_cast<const W *>(a.down) + (size_t)id * a.rank * a.K, a.rank, a.K, a.K, sizeof(W));
        auto at_ranks = [&](auto what) {
            if (a.rank % LANE == 0) what(Cut<W, true>(p * LANE, a.rank));
            else what(Cut<W, false>(p * LANE, a.rank));
        };
        W u[LANE];
        at_ranks([&](auto cut) { cut.load(up, m < a.M ? (uint32_t)m * (uint32_t)a.rank * (uint32_t)sizeof(W) : kNowhere, u); });
        const float alpha = a.alpha ? a.alpha[id] : 1.0f;
        auto at_piece = [&](int k, auto what) {   // (all but the last one of a row are whole)
            if (WHOLE || k + PIECE <= a.K) what(Cut<W, true>(k + lane * LANE, a.K));
            else what(Cut<W, false>(k + lane * LANE, a.K));
        };
        for (int j0 = 0; j0 < a.rank; j0 += WAVES) {
            const int j = j0 + wave;
            float dot = 0.0f;
            for (int k0 = 0; k0 < a.K; k0 += PIECE * AT_ONCE) {
                W w[AT_ONCE][LANE];
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q)
                    if (k0 + q * PIECE < a.K)
                        at_piece(k0 + q * PIECE, [&](auto cut) {
                            cut.load(down, j < a.rank ? (uint32_t)j * (uint32_t)a.K * (uint32_t)sizeof(W) : kNowhere, w[q]);
                        });
                if (j0 == 0 && k0 == 0) __syncthreads();   // x is in LDS
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q)
                    if (k0 + q * PIECE < a.K)
                        at_piece(k0 + q * PIECE, [&](auto cut) {
                            if (cut.any)
#pragma unroll
                                for (int i = 0; i < LANE; ++i) dot = __builtin_fmaf((float)w[q][i], cut.keeps(i) ? xs[cut.from + i] : 0.0f, dot);
                        });
            }
            const float each[1] = {dot};
            float sum[1];
            over_rows<1, 1, false>(each, lane, sum);
            if (lane == 0 && j < a.rank) ts[j] = sum[0] * alpha;
        }
        __syncthreads();
        s = 0.0f;
        at_ranks([&](auto cut) {
            if (cut.any)
#pragma unroll
                for (int i = 0; i < LANE; ++i)
                    if (cut.keeps(i)) s = __builtin_fmaf((float)u[i], ts[cut.from + i], s);
        });
        s += from_lane_xor<8>(s);
        s += from_lane_xor<4>(s);
        s += from_lane_xor<2>(s);
        s += from_lane_xor<1>(s);
    }
    if (m >= a.M || p > 0) return;
    float col[1] = {1.0f}, scale = 1.0f;
    if constexpr (SCALED) {
        if (a.col) col[0] = a.col[blockIdx.y];
        if (a.row) scale = a.row[m];
        if (some) s *= col[0];
    }
    const Matrix Y(static_cast<W *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, 1, a.ldy, sizeof(W));
    const float c1[1] = {(float)had[0]}, add[1] = {s};
    W y[1];
    finish<C, W, 1>(c1, col, scale, add, y);
    store<W, 1>(Y, (uint32_t)m * (uint32_t)a.ldy * (uint32_t)sizeof(W), 0, 0, y);
}

// ---- Many tokens: tiles of 64 on the matrix cores.
//
// A lane has four adjacent tokens, one of each of four 16-wide tiles, so that x, C and Y are read and written 4 tokens at a time.  An adapter's
// weights meet all tokens of a tile, of which only those that are its own take the result: nothing of another token or adapter reaches them.
// Tokens of a request lie side by side, so that a tile meets one adapter or two; a tile of 64 requests takes 64 turns.

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;

// The tokens of a lane, and which adapter each of them has (-1: none).
struct TileTokens {
    Columns<4> columns;
    int id[4];
    __device__ __forceinline__ TileTokens(const int32_t *index, int count, int n0, int N, int lane) : columns(n0 + (lane & 15) * 4, N) {
        const Matrix m(index + (size_t)blockIdx.y * N, 1, N, N, 4);
        load<int32_t, 4>(m, columns.any ? (uint32_t)columns.first * 4u : kNowhere, 0, id);
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (!columns.any || c < columns.skip || (uint32_t)id[c] >= (uint32_t)count) id[c] = -1;
    }
    // The adapters of the tile one after the other, each once: the next one, with its tokens taken out of `left`, or -1.  Uniform.
    static __device__ __forceinline__ int next(int (&left)[4]) {
        const uint32_t any = min(min((uint32_t)left[0], (uint32_t)left[1]), min((uint32_t)left[2], (uint32_t)left[3]));   // (-1 is the largest)
        const uint64_t lanes = __ballot(any != 0xffffffffu);
        if (lanes == 0) return -1;
        const int a = __builtin_amdgcn_readlane((int)any, __builtin_ctzll(lanes));
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
    static __device__ __forceinline__ float4v mma(const frag &w, const frag &x, const float4v &c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, c, 0, 0, 0);
    }
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

// 2048 tokens of int8, K = 4096, rank 64: 13.6 us, a turn 1.2 (two parts of eight turns; four parts lengthen the second kernel by more).
// A workgroup does 64 tokens and a part of K, its eight waves a step each at a time (256 rows of half weights, 128 of binary32); what a turn needs
// from memory is fetched while the one before it is computed.  When an adapter's last turn is done, the waves' sums meet in LDS.
template <typename X, typename W, int RB, bool WHOLE>
__global__ __launch_bounds__(kShrinkWaves * 64, 2) void shrink_tiles_kernel(const ShrinkArgs a) {
    typedef Step<W> Q;
    typedef typename Q::frag frag;
    constexpr int TURN = kShrinkWaves * Q::ROWS;
    __shared__ __align__(16) float4v sums[RB][kShrinkWaves][4][64];
    __shared__ int ids[kTile];
    const int tiles = (a.N + kTile - 1) / kTile, task = task_of(blockIdx.x, tiles * a.parts * a.slots);
    if (task >= tiles * a.parts * a.slots) return;
    const int slot = task % a.slots, part = task / a.slots % a.parts, n0 = task / a.slots / a.parts * kTile;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, i = lane & 15;
    const TileTokens tokens(a.index, a.count, n0, a.N, lane);
    const int ranks = ranks16(a.rank), first = part * a.turns, last = min(first + a.turns, (a.K + TURN - 1) / TURN);   // turns of this part
    const Matrix from(static_cast<const X *>(a.X) + (int64_t)blockIdx.y * a.K * a.ldx, a.K, a.N, a.ldx, sizeof(X));
    struct Loads { X v[Q::LANE][4]; frag w[RB]; };
    Loads even, odd;
    // Offsets of a lane in a turn.  Rows of x past K lie outside of it.  (What the lanes share, the turn's first row, does not: a range is checked
    // after it has been taken off.)
    const int lane_row = wave * Q::ROWS + g * Q::LANE;
    uint32_t x_at[Q::LANE];
#pragma unroll
    for (int e = 0; e < Q::LANE; ++e)
        x_at[e] = tokens.columns.any ? ((uint32_t)(lane_row + e) * (uint32_t)a.ldx + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(X) : kNowhere;
    // (Every fetch is made, if of nothing: where one might be left out, the compiler has to wait for the whole of the one before it.)
    // !WHOLE: how many rows up the piece begins that the end of K cuts short.
    const int turns = (a.K + TURN - 1) / TURN, end_at = (turns - 1) * TURN + lane_row;
    const int up = !WHOLE && end_at < a.K ? max(0, end_at + Q::LANE - a.K) : 0;
    auto fetch_x = [&](bool any, int turn, Loads &l) {
        if constexpr (!WHOLE) {   // (a first row of the turn, less those rows, may lie before it)
            const uint32_t to = ((uint32_t)turn * (uint32_t)TURN - (turn + 1 == turns ? (uint32_t)up : 0u)) * (uint32_t)a.ldx * (uint32_t)sizeof(X);
#pragma unroll
            for (int e = 0; e < Q::LANE; ++e) load<X, 4>(from, any && tokens.columns.any ? x_at[e] + to : kNowhere, 0, l.v[e]);
            return;
        }
#pragma unroll
        for (int e = 0; e < Q::LANE; ++e)
            load<X, 4>(from, any ? x_at[e] : kNowhere, (uint32_t)turn * (uint32_t)TURN * (uint32_t)a.ldx * (uint32_t)sizeof(X), l.v[e]);
    };
    auto fetch_w = [&](int id, int turn, Loads &l) {
        const Matrix down(id >= 0 ? static_cast<const W *>(a.down) + (size_t)id * a.rank * a.K : nullptr, a.rank, a.K, a.K, sizeof(W));
        const int k = turn * TURN + lane_row;
        if constexpr (WHOLE) {
            // (Ranks past the last lie outside, too.)
            const uint32_t at = k < a.K ? ((uint32_t)i * (uint32_t)a.K + (uint32_t)lane_row) * (uint32_t)sizeof(W) : kNowhere;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                W v[Q::LANE];
                load<W, Q::LANE>(down, at + (k < a.K ? (uint32_t)(b * 16) * (uint32_t)a.K * (uint32_t)sizeof(W) : 0),
                                 id >= 0 ? (uint32_t)turn * (uint32_t)TURN * (uint32_t)sizeof(W) : 0, v);
                __builtin_memcpy(&l.w[b], v, 16);
            }
        } else {
            const Cut<W, false> cut(k, a.K);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                W v[Q::LANE];
                load<W, Q::LANE>(down, cut.any && b * 16 + i < a.rank
                                     ? ((uint32_t)(b * 16 + i) * (uint32_t)a.K + (uint32_t)cut.from) * (uint32_t)sizeof(W) : kNowhere, 0, v);
                cut.mask(v);
                __builtin_memcpy(&l.w[b], v, 16);
            }
        }
    };
    fetch_x(true, first, even);
    int left[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) left[c] = tokens.id[c];
    auto next = [&](int n) {   // the n-th adapter from here, or -1
        int id;
        do id = TileTokens::next(left);
        while (id >= 0 && --n > 0);
        return id;
    };
    int id = next(slot + 1);   // of this workgroup's adapters: every slots-th, from the slot-th on
    if (id < 0) return;
    fetch_w(id, first, even);
    if (wave == 0 && g == 0)
#pragma unroll
        for (int c = 0; c < 4; ++c) ids[i * 4 + c] = tokens.id[c];
    // Thread t: two ranks of a token, the waves' sums in their order.
    const int item = t >> 1, of_c = item >> 6, of_lane = item & 63, n = min(n0 + (of_lane & 15) * 4, a.N - 4) + of_c;
    const int of_j = (of_lane >> 4) * 4 + (t & 1) * 2;
    float *const to = a.t + (((size_t)blockIdx.y * a.N + n) * a.parts + part) * ranks + of_j;
    const float col = a.col ? a.col[(size_t)blockIdx.y * a.N + n] : 1.0f;
    float4v acc[RB][4];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    frag x[4];
    int turn = first, then = next(a.slots);   // then: the adapter after this one
    bool fresh = true, met = false;           // is x of this turn still to be made; have sums met already?
    // One turn; false when it was the last one.
    auto step = [&](Loads &now, Loads &ahead) {
        const bool done = turn + 1 == last;
        const int of = done ? then : id, at = done ? first : turn + 1;
        fetch_x(of >= 0 && last - first > 1, at, ahead);
        fetch_w(of, at, ahead);
        if (fresh)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < Q::LANE; ++e) x[c][e] = !WHOLE && e < up && turn + 1 == turns ? (W)0 : (W)now.v[e][c];
        fresh = last - first > 1;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[b][c] = Q::mma(now.w[b], x[c], acc[b][c]);
        if (!done) {
            ++turn;
            return true;
        }
        const float alpha = a.alpha ? a.alpha[id] : 1.0f;
        if (met) __syncthreads();   // the last adapter's sums have been read
        met = true;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                sums[b][wave][c][lane] = acc[b][c];
                acc[b][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            }
        __syncthreads();
        if (ids[(of_lane & 15) * 4 + of_c] == id) {
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                float2 sum = {0.0f, 0.0f};
#pragma unroll
                for (int v = 0; v < kShrinkWaves; ++v) {
                    const float2 u = *(reinterpret_cast<const float2 *>(&sums[b][v][of_c][of_lane]) + (t & 1));
                    sum.x += u.x;
                    sum.y += u.y;
                }
                sum.x = sum.x * alpha * col;
                sum.y = sum.y * alpha * col;
                if constexpr (std::is_same<W, float>::value) {
                    // Ranks behind the last one are zeros, not what zeros for weights make of an infinite x: the second kernel multiplies them.
                    // (For half it makes sums that are not finite again, of the ranks there are.)
                    if (b * 16 + of_j >= a.rank) sum.x = 0.0f;
                    if (b * 16 + of_j + 1 >= a.rank) sum.y = 0.0f;
                }
                if (b * 16 < ranks) *reinterpret_cast<float2 *>(to + b * 16) = sum;
            }
        }
        id = then;
        turn = first;
        if (id < 0) return false;
        then = next(a.slots);
        return true;
    };
    while (step(even, odd) && step(odd, even)) {}
}

// 2048 tokens, 4096 rows, rank 64, int32 to half, 50 MB: 15 us where every tile meets one adapter, 19 with two, 23 with runs of random lengths,
// whose longest tile ends last; of it about 6 us before the first block, in which t is gathered and made into operands.
// Waves of a workgroup: the more ranks, the more of them share what is made of t first.
template <int RB> constexpr int kExpandTileWaves = RB < 4 ? 4 : 8;

// A workgroup does 64 tokens and `rows` rows of Y (a multiple of 64), its waves 16 of them at a time; what such a block needs from memory is
// fetched while the one before it is computed.
// half: t is split into two halves, t = hi + lo, which the instruction's 32 steps take side by side
// for 16 ranks, beside the same 16 weights twice: 22 bits of t, at a sixteenth of what binary32 instructions cost.  Every token's t is scaled by a
// power of two first, its largest finite one to 2^14 ... 2^15, so that neither half leaves its range: what lo loses below 2^-24 is 2^-39 of that
// largest.  (An infinite t stays one, and has no lo.)
template <typename C, typename W, int RB, bool WHOLE>
__global__ __launch_bounds__(kExpandTileWaves<RB> * 64, RB < 2 ? 3 : 2) void expand_tiles_kernel(const ExpandArgs a) {
    constexpr bool SCALED = std::is_same<C, int32_t>::value, HALF = std::is_same<W, _Float16>::value;
    typedef Step<W> Q;
    typedef typename Q::frag frag;
    constexpr int WAVES = kExpandTileWaves<RB>, PITCH = RB * 16 + 4, SHARE = WAVES * 64 / kTile;   // SHARE: threads of a token
    __shared__ __align__(16) float ts[kTile * PITCH];
    __shared__ __align__(16) frag operands[RB * 4][64];
    __shared__ int exponents[kTile];
    const int tiles = (a.N + kTile - 1) / kTile, chunks = (a.M + a.rows - 1) / a.rows, task = task_of(blockIdx.x, tiles * chunks);
    if (task >= tiles * chunks) return;
    const int n0 = task % tiles * kTile, m0 = task / tiles * a.rows, end = min(a.M, m0 + a.rows);
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, i = lane & 15;
    // Everything that waits for nothing is on its way first.
    const TileTokens tokens(a.index, a.count, n0, a.N, lane);
    GatherT<WAVES * 64, RB * 16> gather(a, n0, min(kTile, a.N - n0));
    const Matrix from(static_cast<const C *>(a.C) + (int64_t)blockIdx.y * a.M * a.ldc, a.M, a.N, a.ldc, sizeof(C));
    const Matrix Y(static_cast<W *>(a.Y) + (int64_t)blockIdx.y * a.M * a.ldy, a.M, a.N, a.ldy, sizeof(W));
    const Matrix rows(a.row, 1, a.M, a.M, 4);
    // Offsets of a lane in a block; rows past M lie outside the matrices.  (What the lanes share, the block's first row, does not: a range is
    // checked after it has been taken off.)
    const bool any = tokens.columns.any;
    uint32_t c_at[4], y_at[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        c_at[q] = any ? ((uint32_t)(g * 4 + q) * (uint32_t)a.ldc + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(C) : kNowhere;
        y_at[q] = any ? ((uint32_t)(g * 4 + q) * (uint32_t)a.ldy + (uint32_t)tokens.columns.first) * (uint32_t)sizeof(W) : kNowhere;
    }
    constexpr bool TWO = RB < 4;   // (there are no registers for more)
    struct Block { C had[4][4]; float row[4]; frag w[RB], w2[TWO ? RB : 1]; };   // weights of the first adapter of the tile; of the second one
    // (Every fetch is made, if of nothing: where one might be left out, the compiler has to wait for the whole of the one before it.)
    auto fetch_c = [&](int m, Block &b) {
        const bool some = m < end;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            load<C, 4>(from, some ? c_at[q] : kNowhere, some ? (uint32_t)m * (uint32_t)a.ldc * (uint32_t)sizeof(C) : 0, b.had[q]);
        if constexpr (SCALED) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float one[1];
                load<float, 1>(rows, some ? (uint32_t)(m + g * 4 + q) * 4u : kNowhere, 0, one);   // (0 where there are no scales)
                b.row[q] = one[0];
            }
        }
    };
    auto up_of = [&](int m, int id, frag (&w)[RB]) {
        const bool some = id >= 0 && m < end;
        const Matrix up(some ? static_cast<const W *>(a.up) + (size_t)id * a.M * a.rank : nullptr, a.M, a.rank, a.rank, sizeof(W));
        const uint32_t block_at = some ? (uint32_t)m * (uint32_t)a.rank * (uint32_t)sizeof(W) : 0;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int j = b * 16 + (HALF ? (g & 1) * 8 : g * 4);
            const Piece<W> p = piece<W>(up, (uint32_t)i * (uint32_t)a.rank * (uint32_t)sizeof(W), block_at, j, a.rank, WHOLE);
            __builtin_memcpy(&w[b], p.v, 16);
        }
    };
    Block even, odd;
    const int mine = m0 + wave * 16;
    fetch_c(mine, even);
    int left[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) left[c] = tokens.id[c];
    const int first = TileTokens::next(left), second = TileTokens::next(left);
    bool all = true;   // have all tokens the first one?
#pragma unroll
    for (int c = 0; c < 4; ++c) all &= tokens.id[c] == first || !any || c < tokens.columns.skip;
    all = __all(all);
    auto fetch = [&](int m, Block &b) {
        fetch_c(m, b);
        up_of(m, first, b.w);
        if constexpr (TWO) up_of(m, second, b.w2);
    };
    up_of(mine, first, even.w);
    if constexpr (TWO) up_of(mine, second, even.w2);
    // Row (n % 4) * 16 + n / 4 of ts is token n of the tile: the lanes of a quarter read rows that follow each other.
    auto row_of = [](int n) { return (n & 3) * 16 + (n >> 2); };
    float top = gather.finish(ts, PITCH, row_of(gather.c));
    if constexpr (HALF) {
        top = fmaxf(top, from_lane_xor<1>(top));
        top = fmaxf(top, from_lane_xor<2>(top));
        if constexpr (SHARE == 8) top = fmaxf(top, from_lane_xor<4>(top));
        if (t % SHARE == 0) exponents[t / SHARE] = top > 0.0f ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
    }
    __syncthreads();
    // The second operand of every instruction, one for each 16 ranks and each quarter of the tokens: a wave makes some of a quarter.
    int down[4];   // the tokens' scaling, to be undone
#pragma unroll
    for (int c = 0; c < 4; ++c) down[c] = HALF && tokens.id[c] >= 0 ? -exponents[tokens.columns.first + c - n0] : 0;
    {
        const int q = wave & 3, id = q == 0 ? tokens.id[0] : q == 1 ? tokens.id[1] : q == 2 ? tokens.id[2] : tokens.id[3];
        const int shift = q == 0 ? down[0] : q == 1 ? down[1] : q == 2 ? down[2] : down[3];
        const int of = id >= 0 ? tokens.columns.first + q - n0 : 0;   // (a last lane's first columns may lie before the tile: they have no adapter)
        const int ranks = ranks16(a.rank);
#pragma unroll
        for (int o = 0; o < RB * 4 / WAVES; ++o) {
            const int b = o * (WAVES / 4) + (wave >> 2), j0 = b * 16 + (HALF ? (g & 1) * 8 : g * 4);
            const float *const from = ts + row_of(of) * PITCH + j0;
            float4v v[Q::LANE / 4];
#pragma unroll
            for (int p = 0; p < Q::LANE / 4; ++p)
                v[p] = id >= 0 && b * 16 < ranks ? *reinterpret_cast<const float4v *>(from + p * 4) : float4v{0.0f, 0.0f, 0.0f, 0.0f};
            frag f;
#pragma unroll
            for (int e = 0; e < Q::LANE; ++e) {
                if constexpr (HALF) {
                    const float scaled = __builtin_ldexpf(v[e / 4][e % 4], -shift);
                    const _Float16 hi = (_Float16)scaled;
                    const float rest = scaled - (float)hi;
                    f[e] = g < 2 ? hi : fabsf(rest) < INFINITY ? (_Float16)rest : (_Float16)0.0f;   // (an infinity has no rest)
                } else {
                    f[e] = v[e / 4][e % 4];
                }
            }
            operands[b * 4 + q][lane] = f;
        }
    }
    __syncthreads();
    frag x[RB][4];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[b][c] = operands[b * 4 + c][lane];
    const uint32_t ones = a.row ? 0u : __float_as_uint(1.0f);   // of rows without scales
    float col[4];
    if constexpr (SCALED) {
#pragma unroll
        for (int c = 0; c < 4; ++c) col[c] = a.col && any ? a.col[(size_t)blockIdx.y * a.N + tokens.columns.first + c] : 1.0f;
    }
    auto block = [&](int m, const Block &b) {
        float add[4][4];   // [row][token]
        // What an adapter adds to the tokens that are its own (alone: all are).
        auto one = [&](int id, const frag (&w)[RB], auto alone) {
            float4v acc[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    // (In binary32 a product is worth a branch around it: 512 requests of a token each, 4096 rows, rank 16: 19 us for 25.  In half
                    // it is not.)
                    if (!HALF && !decltype(alone)::value && !__any(tokens.id[c] == id)) continue;
                    acc[c] = Q::mma(w[r], x[r][c], acc[c]);
                }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v = HALF ? __builtin_ldexpf(acc[c][q], down[c]) : acc[c][q];
                    add[q][c] = decltype(alone)::value || tokens.id[c] == id ? v : add[q][c];
                }
        };
        if (all && first >= 0) {
            one(first, b.w, std::true_type{});
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int c = 0; c < 4; ++c) add[q][c] = -0.0f;   // (what is added to nothing leaves it as it is)
            // (The next adapter's weights are on their way while one is multiplied.)
            int rest[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) rest[c] = left[c];
            int id = TWO ? TileTokens::next(rest) : second;
            frag w[RB];
            up_of(m, id, w);
            if (first >= 0) one(first, b.w, std::false_type{});
            if constexpr (TWO)
                if (second >= 0) one(second, b.w2, std::false_type{});
            while (id >= 0) {
                const int then = TileTokens::next(rest);
                frag ahead[RB];
                up_of(m, then, ahead);
                one(id, w, std::false_type{});
                id = then;
                if (id < 0) break;
                const int last = TileTokens::next(rest);
                up_of(m, last, w);
                one(id, ahead, std::false_type{});
                id = last;
            }
        }
        if constexpr (HALF) {
            // Halves of t say nothing about infinities: an infinite weight times lo is undefined or of any sign.  Sums that are not finite are made
            // again from t itself.
            // (It costs 0.1 us of 11.1 for 1024 tokens of prompts, 1024 -> 4096, rank 16; looking for infinite weights before
            // every product 0.3, and 0.8 of 37 at rank 64.)
            float most = 0.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int c = 0; c < 4; ++c) most = __builtin_elementwise_maximum(most, fabsf(add[q][c]));   // (undefined if one is)
            if (__builtin_expect(__any(!(most < INFINITY)), 0)) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!(fabsf(add[q][c]) < INFINITY)) {
                            int of = tokens.id[c], n = tokens.columns.first + c - n0, at = m + g * 4 + q;
                            // (or the addresses of all sixteen are reckoned ahead and fill the registers)
                            asm volatile("" : "+v"(of), "+v"(n), "+v"(at));
                            if (of < 0 || at >= a.M) continue;
                            const W *const up = static_cast<const W *>(a.up) + ((size_t)of * a.M + at) * a.rank;
                            const float *const from = ts + row_of(n) * PITCH;
                            float s = 0.0f;
#pragma unroll 1
                            for (int j = 0; j < a.rank; ++j) s = __builtin_fmaf((float)up[j], from[j], s);
                            add[q][c] = s;
                        }
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            W y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float had = (float)b.had[q][c];
                if constexpr (SCALED) had = had * col[c] * __uint_as_float(__float_as_uint(b.row[q]) | ones);
                y[c] = (W)(had + add[q][c]);
            }
            store<W, 4>(Y, y_at[q], (uint32_t)m * (uint32_t)a.ldy * (uint32_t)sizeof(W), any ? tokens.columns.skip : 0, y);
        }
    };
    constexpr int NEXT = WAVES * 16;
    for (int m = mine; m < end; m += 2 * NEXT) {
        fetch(m + NEXT, odd);
        block(m, even);
        if (m + NEXT >= end) break;
        fetch(m + 2 * NEXT, even);
        block(m + NEXT, odd);
    }
}

namespace {

struct Plan {   // the kernels of a call, and what they go by
    const void *one;   // one kernel, or
    const void *shrink, *expand;
    int parts, turns, slots, rows;
    int64_t shrink_grid, expand_grid;
    int shrink_threads, expand_threads, lds;
};

template <typename X, typename W, int RB> const void *shrink_tiles(bool whole) {
    return whole ? (const void *)shrink_tiles_kernel<X, W, RB, true> : (const void *)shrink_tiles_kernel<X, W, RB, false>;
}
template <typename C, typename W, int RB> const void *expand_tiles(bool whole) {
    return whole ? (const void *)expand_tiles_kernel<C, W, RB, true> : (const void *)expand_tiles_kernel<C, W, RB, false>;
}
template <typename C, typename W, int EACH> const void *expand_tokens(bool whole) {
    return whole ? (const void *)expand_tokens_kernel<C, W, EACH, true> : (const void *)expand_tokens_kernel<C, W, EACH, false>;
}
template <typename X, typename W, int V> const void *shrink_tokens(bool whole) {
    return whole ? (const void *)shrink_tokens_kernel<X, W, V, true> : (const void *)shrink_tokens_kernel<X, W, V, false>;
}
template <typename X, typename C, typename W> const void *one_token(bool whole) {
    return whole ? (const void *)one_token_kernel<X, C, W, true> : (const void *)one_token_kernel<X, C, W, false>;
}

template <typename X, typename C, typename W> Plan plan_of(const sparsert_adapter_set &d) {
    Plan p{};
    constexpr int LANE = 16 / (int)sizeof(W);
    const bool whole_k = d.K % LANE == 0, whole_rank = d.rank % LANE == 0;
    const int ranks = (d.rank + 15) / 16 * 16;
    // One token.  Measured as one kernel and as two, in us: K = 1024, ranks 8, 32, 64: half 3.6, 4.2, 5.7 and 5.6, 5.8, 6.3, binary32 3.6, 4.5, 6.0
    // and 5.7, 6.0, 6.6; K = 4096, rank 16: 4.7 and 6.0, 5.6 and 6.1, rank 32: 6.4 and 6.1, 7.9 and 6.4.  Odd K = 771, ranks 8, 32, 64: half 4.5,
    // 6.0, 8.9 and 6.0, 6.2, 6.7, binary32 4.9, 7.1, 11.5 and 6.4, 6.7, 7.3.
    if (d.N == 1 && d.rank <= kOneRank && (int64_t)ranks * d.K <= (whole_k ? kOneSize : kOneSize / 4)) {
        p.one = one_token<X, C, W>(whole_k);
        p.expand_grid = (d.M + kOneRows - 1) / kOneRows;
        p.lds = (d.K + 7) / 8 * 8 * (int)sizeof(float);
        return p;
    }
    // Bytes of weights that the tokens read if every one reads its own: what the first kind of kernels spends its time on.  The other kind spends
    // it on the adapters that a tile meets, which only the device knows, so the limit grows with their number.  4096 x 4096, rank 16, half, 24
    // adapters, tokens and tiles, us: 64 tokens in runs 8.2 and 9.2, 256 13.3 and 9.8, 512 21 and 11; 64 requests of a token each 9.5 and 18, 512
    // 23 and 29.  Over 405 calls of 8 to 512 tokens, with 2 and 24 adapters, the choices come to 3 % above the best of each.  What they miss is a
    // batch that meets few of many adapters, or many of few: 1024 -> 4096, 1024 tokens, rank 16 in half, tokens and tiles: in runs with 32 adapters
    // 25.9 and 11.5 (tiles), with 64 25.6 and 11.9 (tokens); requests of a token each with 24 26.1 and 32.5 (tiles), with 64 27.0 and 49.7
    // (tokens); 4096 x 4096, 2048 requests, 64 adapters 73 and 128 (tiles).
    // Tiles are built for ranks up to 64, and for rows of weights that are
    // read in pieces (pieces_fit).  Beyond them tokens take what is left: 4096 x 4096, 2048 tokens, half, rank 64 37 us in tiles, 65 601, 96 245,
    // 128 404, 256 716; 1024 -> 4096, rank 8 14.8, 6 17.0, 7 102.
    const double own = (double)d.N * d.batch * ((double)d.M + d.K) * ranks * (int)sizeof(W);
    const double limit = (30e6 + 4e6 * std::min(d.count, kTile)) * (sizeof(W) == 4 ? 2 : 1);
    // (The tiles' lanes reckon with offsets of some rows on from any one.)
    const bool near = (int64_t)(kShrinkWaves * Step<W>::ROWS) * d.ldx * (int)sizeof(X) < 1ll << 31 &&
        16ll * std::max((int64_t)d.ldc * (int)sizeof(C), (int64_t)d.ldy * (int)sizeof(W)) < 1ll << 31 &&
                      64ll * d.K * (int)sizeof(W) < 1ll << 31 && 16ll * d.rank * (int)sizeof(W) < 1ll << 31;
    if (near && d.N >= 4 && d.rank <= 64 && pieces_fit<W>(d.rank) && d.K >= LANE && own > limit) {
        const int64_t tiles = ((int64_t)d.N + kTile - 1) / kTile;
        constexpr int TURN = kShrinkWaves * Step<W>::ROWS;
        const int turns = (d.K + TURN - 1) / TURN;
        p.parts = (int)std::min<int64_t>(turns, std::max<int64_t>(1, 64 / (tiles * d.batch)));
        p.turns = (turns + p.parts - 1) / p.parts;
        p.parts = (turns + p.turns - 1) / p.turns;
        p.slots = (int)std::min<int64_t>({8, d.count, std::max<int64_t>(1, 256 / (tiles * d.batch * p.parts))});
        p.shrink = ranks <= 16 ? shrink_tiles<X, W, 1>(whole_k) : ranks <= 32 ? shrink_tiles<X, W, 2>(whole_k) : shrink_tiles<X, W, 4>(whole_k);
        p.shrink_grid = tiles * p.parts * p.slots; p.shrink_threads = kShrinkWaves * 64;
        p.expand = ranks <= 16 ? expand_tiles<C, W, 1>(whole_rank)
                 : ranks <= 32 ? expand_tiles<C, W, 2>(whole_rank) : expand_tiles<C, W, 4>(whole_rank);
        const int step = ranks <= 32 ? kExpandTileWaves<2> * 16 : kExpandTileWaves<4> * 16;
        const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>((d.M + step - 1) / step, (ranks <= 32 ? 512 : 256) / (tiles * d.batch)));
        p.rows = (int)(((d.M + chunks - 1) / chunks + step - 1) / step * step);
        p.expand_grid = tiles * ((d.M + p.rows - 1) / p.rows); p.expand_threads = step * 4;
        return p;
    }
    p.parts = (d.K + kTokenRows - 1) / kTokenRows;
    p.shrink = d.N < kTokenGroup ? shrink_tokens<X, W, 1>(d.K % 8 == 0) : shrink_tokens<X, W, kTokenGroup>(d.K % 8 == 0);
    p.shrink_grid = ((int64_t)d.N + kTokenGroup - 1) / kTokenGroup * p.parts * (ranks / 16); p.shrink_threads = kTokenThreads;
    const int64_t blocks = (d.M + kExpandRows - 1) / kExpandRows;
    int each = 4;
    // (No more tokens than make t 32 KiB in LDS.)
    while (each > 1 && (blocks * (((int64_t)d.N + each * kExpandWaves - 1) / (each * kExpandWaves)) * d.batch < 256 ||
        each * kExpandWaves * ranks > 8192)) each /= 2;
    p.expand = each == 4 ? expand_tokens<C, W, 4>(whole_rank) : each == 2 ? expand_tokens<C, W, 2>(whole_rank) : expand_tokens<C, W, 1>(whole_rank);
    p.expand_grid = ((int64_t)d.N + each * kExpandWaves - 1) / (each * kExpandWaves) * blocks; p.expand_threads = kExpandThreads;
    p.lds = each * kExpandWaves * ranks * (int)sizeof(float);
    return p;
}

Plan plan_of(const sparsert_adapter_set &d) {
    const bool half = d.dtype == SPARSERT_F16;
    if (d.x_dtype == SPARSERT_I8) return half ? plan_of<int8_t, int32_t, _Float16>(d) : plan_of<int8_t, int32_t, float>(d);
    return half ? plan_of<_Float16, _Float16, _Float16>(d) : plan_of<float, float, float>(d);
}

}  // namespace

size_t adapters_workspace(const sparsert_adapter_set &d) {
    return (size_t)d.batch * d.N * plan_of(d).parts * ((d.rank + 15) / 16 * 16) * sizeof(float);
}

int launch_adapters(const AdaptersCall &c, std::string &err) {
    const sparsert_adapter_set &d = c.d;
    const Plan p = plan_of(d);
    if (p.one) {
        if (int rc = check_launch(p.expand_grid, kOneThreads, err)) return rc;
        OneArgs a{c.X, c.down, c.up, c.index, c.alpha, c.C, c.Y, c.row, c.col, d.M, d.K, d.ldx, d.ldc, d.ldy, d.rank, d.count};
        return launch_operator(p.one, dim3((uint32_t)p.expand_grid, (uint32_t)d.batch), kOneThreads, a, c.stream, err, p.lds);
    }
    const auto whole = [](int64_t n) { return (n + 7) / 8 * 8; };
    if (int rc = check_launch(whole(p.shrink_grid), p.shrink_threads, err)) return rc;
    if (int rc = check_launch(whole(p.expand_grid), p.expand_threads, err)) return rc;
    float *const t = static_cast<float *>(c.workspace);
    ShrinkArgs s{c.X, c.down, c.index, c.alpha, c.col, t, d.K, d.N, d.ldx, d.rank, d.count, p.parts, p.turns, p.slots};
    const auto grid = [&](int64_t n) { return dim3((uint32_t)whole(n), (uint32_t)d.batch); };
    if (int rc = launch_operator(p.shrink, grid(p.shrink_grid), p.shrink_threads, s, c.stream, err)) return rc;
    ExpandArgs e{c.C, c.up, c.index, c.row, c.col, t, c.Y, d.M, d.N, d.ldc, d.ldy, d.count, p.parts, p.rows, d.rank};
    return launch_operator(p.expand, grid(p.expand_grid), p.expand_threads, e, c.stream, err, p.lds);
}

}  // namespace sparsert
