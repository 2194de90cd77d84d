// Rows of learnt values in the storage types of X: loads and stores of several coordinates at once, always through
// float32, and the host side that the operators on them share (status codes, workspaces).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/rnnd.h"
#include "dist.h"
#include "grid.h"

template <int DT> struct RowType;
template <> struct RowType<DT_F32> { typedef float T; };
template <> struct RowType<DT_F16> { typedef _Float16 T; };
template <> struct RowType<DT_BF16> { typedef __bf16 T; };

// VEC coordinates that lie next to each other; one access of up to 16 bytes, so VEC = 8 of float32 are two
template <int DT, int VEC> struct alignas(VEC * sizeof(typename RowType<DT>::T) > 16 ? 16 : VEC * sizeof(typename RowType<DT>::T)) Pack {
    typename RowType<DT>::T v[VEC];
};

template <int DT, int VEC>
__device__ __forceinline__ void unpack(const Pack<DT, VEC> &p, float (&x)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)p.v[i];
}
// one rounding, to nearest even (float32: none)
template <int DT, int VEC>
__device__ __forceinline__ void store_pack(void *base, size_t at, const float (&x)[VEC])
{
    Pack<DT, VEC> p;
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.v[i] = (typename RowType<DT>::T)x[i];
    *(Pack<DT, VEC> *)((typename RowType<DT>::T *)base + at) = p;
}
template <int DT, int VEC>
__device__ __forceinline__ Pack<DT, VEC> load_pack(const void *base, size_t at)
{
    return *(const Pack<DT, VEC> *)((const typename RowType<DT>::T *)base + at);
}

// splitmix64's output function and increment, as RandomGraph uses them
__host__ __device__ inline u64 row_mix64(u64 z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
#define ROW_MIX_G 0x9E3779B97F4A7C15ull

// ---- host side
int report_hip_error(const char *what, hipError_t e);      // notes the message for rnnd_strerror; the status

static inline bool row_type(int dtype) { return dtype == RNND_F32 || dtype == RNND_F16 || dtype == RNND_BF16; }
static inline size_t ws_align(size_t x) { return (x + 255) & ~(size_t)255; }

// launch errors of the kernels just enqueued
static inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? RNND_OK : report_hip_error(what, e);
}

// Largest number of coordinates (8, 4, 2 or 1) that divides a row of d and that both sides can move in aligned
// accesses: p, q are rows of size_p, size_q bytes a coordinate.
static inline int row_vec(int d, const void *p, int size_p, const void *q, int size_q)
{
    for (int v = 8; v > 1; v >>= 1) {
        const int ap = v * size_p > 16 ? 16 : v * size_p, aq = v * size_q > 16 ? 16 : v * size_q;
        if (d % v == 0 && (uintptr_t)p % ap == 0 && (uintptr_t)q % aq == 0) return v;
    }
    return 1;
}
