// Element types of floating arrays (QRNNT_F32, _F16, _BF16) as the kernels read and write them: vectors of 16 bytes that
// may start at any element (the vector memory path takes any alignment), values in fp32 in between.
#pragma once

#include "qrnnt_common.h"

static inline bool qr_is_dtype(int dtype) { return dtype == QRNNT_F32 || dtype == QRNNT_F16 || dtype == QRNNT_BF16; }
static inline size_t qr_dtype_size(int dtype) { return dtype == QRNNT_F32 ? 4 : 2; }

// Whether [p, p + pn) and [q, q + qn) have a byte in common.
static inline bool qr_overlap(const void *p, size_t pn, const void *q, size_t qn)
{
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + qn && b < a + pn;
}
// Rows, columns and pitches whose products and sums stay far from the ends of 64 and, for the counts, 32 bits.
static inline bool qr_counts_ok(int64_t rows, int64_t cols) { return rows <= INT32_MAX && cols <= 1 << 30; }
static inline bool qr_pitch_ok(int64_t rows, int64_t ld) { return ld <= ((int64_t)1 << 60) / (rows > 0 ? rows : 1); }
// Bytes from the first to behind the last element of a matrix.
static inline size_t qr_matrix_bytes(int64_t rows, int64_t cols, int64_t ld, size_t size)
{
    return (size_t)((rows - 1) * ld + cols) * size;
}
// Whether two matrices of rows have a byte in common (sizes, rows and pitches in bytes); columns of one matrix have none.
static inline bool qr_rows_overlap(const void *p, size_t pn, int64_t p_row, int64_t p_pitch, const void *q, size_t qn, int64_t q_row, int64_t q_pitch)
{
    if (!qr_overlap(p, pn, q, qn)) return false;
    if (p_pitch != q_pitch) return true;
    const int64_t pitch = p_pitch, d = (((intptr_t)q - (intptr_t)p) % pitch + pitch) % pitch;
    return d < p_row || d + q_row > pitch;
}

template <class T>
struct QrVec {
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef type any __attribute__((aligned(sizeof(T))));   // at any element
};

template <class T>
__device__ __forceinline__ void qr_load_vec(const T *p, float (&v)[QrVec<T>::N])
{
    const typename QrVec<T>::type u = *(const typename QrVec<T>::any *)p;
#pragma unroll
    for (int i = 0; i < QrVec<T>::N; ++i) v[i] = (float)u[i];
}
// (past the caches: what is written is as a rule not read again soon)
template <class T>
__device__ __forceinline__ void qr_store_vec(T *p, const float (&v)[QrVec<T>::N])
{
    typename QrVec<T>::type u;
#pragma unroll
    for (int i = 0; i < QrVec<T>::N; ++i) u[i] = (T)v[i];
    __builtin_nontemporal_store(u, (typename QrVec<T>::any *)p);
}
// The same for the first n elements; the others read as `fill`.
template <class T>
__device__ __forceinline__ void qr_load_vec(const T *p, int n, float fill, float (&v)[QrVec<T>::N])
{
    if (n >= QrVec<T>::N) {
        qr_load_vec(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < QrVec<T>::N; ++i) v[i] = i < n ? (float)p[i] : fill;
    }
}
template <class T>
__device__ __forceinline__ void qr_store_vec(T *p, int n, const float (&v)[QrVec<T>::N])
{
    if (n >= QrVec<T>::N) {
        qr_store_vec(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < QrVec<T>::N; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}
