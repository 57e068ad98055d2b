// Sums and largest values over the lanes of a wave, of several numbers at once.  Device code.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sparsert {

// The larger of two sizes by their bits: as numbers, and above them infinity and what is undefined.
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }

template <int C> __device__ __forceinline__ float from_lane_xor(float v) {   // C: 1, 2, 4 or 8
    if constexpr (C == 8) return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));        // row_ror:8
    else if constexpr (C == 4) return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 4 << 10 | 0x1f));
    else return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), C == 2 ? 0x4e : 0xb1, 0xf, 0xf, false));           // quad_perm
}

// a of this lane and the lane C away in the lanes without bit C, b of both in the others: two numbers become one.
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

// V numbers of every lane, over the lanes l, l + L, l + 2 L ... (L of them remain).  At every step the lanes give
// half of their numbers away, as long as they have more than one; kLeft of them are left, the first of them column_of: V - 1
// exchanges and the last steps in place of V times six.
template <int V, int L> constexpr int kLeft = V * L > 64 ? V * L / 64 : 1;
template <int V, int L, bool MAX> __device__ __forceinline__ void over_rows(const float (&v)[V], int lane, float (&left)[kLeft<V, L>]) {
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = v[i];
    constexpr int S1 = L <= 32 ? V / 2 : 0, S2 = L <= 16 ? V / 4 : 0, S3 = L <= 8 ? V / 8 : 0, S4 = L <= 4 ? V / 16 : 0;
#pragma unroll
    for (int i = 0; i < S1; ++i) a[i] = halve<32, MAX>(a[i], a[i + S1], lane);
#pragma unroll
    for (int i = 0; i < S2; ++i) a[i] = halve<16, MAX>(a[i], a[i + S2], lane);
#pragma unroll
    for (int i = 0; i < S3; ++i) a[i] = halve<8, MAX>(a[i], a[i + S3], lane);
#pragma unroll
    for (int i = 0; i < S4; ++i) a[i] = halve<4, MAX>(a[i], a[i + S4], lane);
    if constexpr (V < 2 && L <= 32) a[0] = halve<32, MAX>(a[0], a[0], lane);
    if constexpr (V < 4 && L <= 16) a[0] = halve<16, MAX>(a[0], a[0], lane);
    if constexpr (V < 8 && L <= 8) a[0] = join<MAX>(a[0], from_lane_xor<8>(a[0]));
    if constexpr (V < 16 && L <= 4) a[0] = join<MAX>(a[0], from_lane_xor<4>(a[0]));
    if constexpr (L <= 2) a[0] = join<MAX>(a[0], from_lane_xor<2>(a[0]));
    if constexpr (L <= 1) a[0] = join<MAX>(a[0], from_lane_xor<1>(a[0]));
#pragma unroll
    for (int i = 0; i < kLeft<V, L>; ++i) left[i] = a[i];
}
template <int V, int L> __device__ __forceinline__ int column_of(int lane) {
    int c = 0;
    if (V >= 2 && L <= 32) c += (lane >> 5 & 1) * (V / 2);
    if (V >= 4 && L <= 16) c += (lane >> 4 & 1) * (V / 4);
    if (V >= 8 && L <= 8) c += (lane >> 3 & 1) * (V / 8);
    if (V >= 16 && L <= 4) c += (lane >> 2 & 1) * (V / 16);
    return c;
}
// of the lanes with the same sums, the one that stores them
template <int V, int L> __device__ __forceinline__ bool stores(int lane) { return V * L >= 64 || (lane & (64 / V - 1)) < L; }
// The sums of a wave's lanes into its row of `to`, one for each column of a strip of V * L columns; a lane's first `skip` are not its own.
template <int V, int L, bool MAX> __device__ __forceinline__ void wave_sums(const float (&v)[V], int lane, int skip, float *to) {
    float left[kLeft<V, L>];
    over_rows<V, L, MAX>(v, lane, left);
    if (stores<V, L>(lane))
#pragma unroll
        for (int i = 0; i < kLeft<V, L>; ++i) {
            const int c = column_of<V, L>(lane) + i;
            if (c >= skip) to[lane % L * V + c - skip] = left[i];
        }
}

}  // namespace sparsert
