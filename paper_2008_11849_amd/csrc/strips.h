// Access to a strip of columns of feature-major activations: a lane owns V adjacent columns and walks the rows.
// Device code.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sparsert {

constexpr uint32_t kNowhere = 0x80000000u;   // a byte offset that every descriptor refuses: matrices are under 2 GiB

template <int BYTES> struct Raw;
template <> struct Raw<1> { typedef uint8_t type; };
template <> struct Raw<2> { typedef uint16_t type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Raw<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

// One problem's matrix.  What lies outside it is neither read (zeros instead) nor written.
struct Matrix {
    __amdgpu_buffer_rsrc_t at;
    __device__ __forceinline__ Matrix(const void *p, int rows, int N, int ld, int size)
        : at(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, p ? (int)(((uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)N) * (uint32_t)size) : 0, 0x00020000)) {}
};

// The columns of a lane whose share of the N columns begins at `from`: V of them from `first` on.  The last lane of a row begins
// earlier where its share is cut short, and `skip` says how many of its columns are the lane's before it: those it reads, as
// vectors are the fast way to read, but leaves alone (they may change under it: results in place).  Needs N >= V.
template <int V> struct Columns {
    int first, skip;
    bool any;   // has the lane a share?
    __device__ __forceinline__ Columns(int from, int N) : first(min(from, N - V)), skip(from < N ? from - first : V), any(from < N) {}
};

// V adjacent elements at byte `lane` + `common` (the part that all lanes share).
template <typename T, int V> __device__ __forceinline__ void load(const Matrix &m, uint32_t lane, uint32_t common, T (&to)[V]) {
    typedef typename Raw<(int)sizeof(T) * V>::type raw;
    raw r;
    if constexpr (sizeof(raw) == 16) r = __builtin_amdgcn_raw_buffer_load_b128(m.at, lane, common, 0);
    else if constexpr (sizeof(raw) == 8) r = __builtin_amdgcn_raw_buffer_load_b64(m.at, lane, common, 0);
    else if constexpr (sizeof(raw) == 4) r = __builtin_amdgcn_raw_buffer_load_b32(m.at, lane, common, 0);
    else if constexpr (sizeof(raw) == 2) r = __builtin_amdgcn_raw_buffer_load_b16(m.at, lane, common, 0);
    else r = __builtin_amdgcn_raw_buffer_load_b8(m.at, lane, common, 0);
    __builtin_memcpy(to, &r, sizeof(raw));
}

// The same for results; the first `skip` of them belong to another lane.
// The offset of a store is one register: behind a store of 16 bytes with a scalar offset the compiler lets the next instruction overwrite
// the data at once, and of the first four bytes the last lanes of every sixteen then stored the new ones.  With none it keeps a clock between.
// AUX: cache policy (2: not to be kept).
template <typename T, int V, int AUX = 0> __device__ __forceinline__ void store(const Matrix &m, uint32_t lane, uint32_t common, int skip, const T (&from)[V]) {
    typedef typename Raw<(int)sizeof(T) * V>::type raw;
    const uint32_t at = lane + common;   // (kNowhere plus a part under 2 GiB stays out of every range)
    if (skip == 0) {
        raw r;
        __builtin_memcpy(&r, from, sizeof(raw));
        if constexpr (sizeof(raw) == 16) __builtin_amdgcn_raw_buffer_store_b128(r, m.at, at, 0, AUX);
        else if constexpr (sizeof(raw) == 8) __builtin_amdgcn_raw_buffer_store_b64(r, m.at, at, 0, AUX);
        else if constexpr (sizeof(raw) == 4) __builtin_amdgcn_raw_buffer_store_b32(r, m.at, at, 0, AUX);
        else if constexpr (sizeof(raw) == 2) __builtin_amdgcn_raw_buffer_store_b16(r, m.at, at, 0, AUX);
        else __builtin_amdgcn_raw_buffer_store_b8(r, m.at, at, 0, AUX);
    } else if constexpr (V > 1) {
#pragma unroll
        for (int v = 1; v < V; ++v) {
            const T one[1] = {from[v]};
            store<T, 1, AUX>(m, v >= skip ? lane + (uint32_t)v * (uint32_t)sizeof(T) : kNowhere, common, 0, one);
        }
    }
}

// Workgroup -> task, so that neighbouring tasks, whose columns share lines of memory, run on one XCD (workgroups are dealt
// to the eight of them in turn).  Of `tasks` tasks; at least `tasks` for a workgroup without one.
__device__ __forceinline__ int task_of(int workgroup, int tasks) { return (workgroup & 7) * ((tasks + 7) >> 3) + (workgroup >> 3); }

}  // namespace sparsert
