// Element types and 16-byte accesses shared by the operators on rows of vectors (layer norm, dropout, the gated
// feed-forward block).
#pragma once

#include "common.h"

namespace gmpgr {

template <int KIND> struct ElemOf;
template <> struct ElemOf<ANN_F32> { using type = float; };
template <> struct ElemOf<ANN_BF16> { using type = __bf16; };
template <> struct ElemOf<ANN_F16> { using type = _Float16; };

// 16 bytes of elements.  The type promises the element's own alignment only: gfx950 serves a 16-byte access at any
// such address, so rows of odd widths and sliced tensors need no code of their own.
template <typename T> constexpr int VEC = 16 / sizeof(T);
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Pack16 {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    type v;
};

template <typename T> __device__ __forceinline__ typename Pack16<T>::type load16(const T *p) {
    return reinterpret_cast<const Pack16<T> *>(p)->v;
}
template <typename T> __device__ __forceinline__ void store16(T *p, typename Pack16<T>::type v) {
    reinterpret_cast<Pack16<T> *>(p)->v = v;
}

// The VEC<T> elements from p on, the first `left` of them only (zeros behind).
template <typename T> __device__ __forceinline__ void load_floats(const T *p, int left, float *out) {
    if (left >= VEC<T>) {
        const typename Pack16<T>::type v = load16(p);
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i) out[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i) out[i] = i < left ? (float)p[i] : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store_floats(T *p, int left, const float *in) {
    if (left >= VEC<T>) {
        typename Pack16<T>::type v;
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i) v[i] = (T)in[i];
        store16(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i)
            if (i < left) p[i] = (T)in[i];
    }
}

inline bool row_dtype(int32_t dtype) { return dtype == ANN_F32 || dtype == ANN_BF16 || dtype == ANN_F16; }
inline size_t elem_bytes(int32_t dtype) { return dtype == ANN_F32 ? 4 : 2; }

// Whether two arrays of M rows share an element: their extents do, and they are not columns side by side of one array.
inline bool rows_overlap(const void *a, int64_t ld_a, int64_t width_a, const void *b, int64_t ld_b, int64_t width_b, int64_t M,
                         size_t e) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    const uintptr_t a1 = a0 + (size_t)((M - 1) * ld_a + width_a) * e, b1 = b0 + (size_t)((M - 1) * ld_b + width_b) * e;
    if (a0 >= b1 || b0 >= a1) return false;
    if (ld_a != ld_b) return true;
    const uintptr_t line = (uintptr_t)ld_a * e, from = (b0 + (a0 / line + 1) * line - a0) % line;  // b's column, from a's
    return !(from >= (uintptr_t)width_a * e && from + (uintptr_t)width_b * e <= line);
}

// rows.hip: first[c] (c < n) and second[c - n] = sum over P of part[p][c], in the order of p, rounded once to dtype; part
// [P][2 n] fp32, either result may be null
int launch_sum_two(const float *part, int64_t P, int64_t n, void *first, void *second, int dtype, hipStream_t stream);
// rows.hip: n elements of zeros
int launch_zero(void *out, int64_t n, int dtype, hipStream_t stream);
// rows.hip: column sums, deterministic, of one or two arrays: of [M][n] values of `dtype` by way of `parts` sums over slices of
// rows in part [parts][n], or (in = null) of parts that are there already.  The results are rounded once to dtype.
struct ColumnSums {
    struct Item {
        const void *in;
        int64_t n, ld;
        void *out;
        float *part;
        int64_t parts;
    } item[2];
    int n;
};
int64_t column_sum_parts(int64_t M, int64_t n);
int launch_column_sums(const ColumnSums &sums, int64_t M, int dtype, hipStream_t stream);

}  // namespace gmpgr
