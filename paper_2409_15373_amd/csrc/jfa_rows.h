// Pieces shared by the operators on rows of any length (jfa_layer_norm.hip, jfa_embedding.hip).  Not part of the C ABI.
#pragma once
#include "jfa_common.h"

namespace jfa {

template <typename T, int VEC> struct RowVec { typedef T Type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct RowVec<T, 1> { typedef T Type; };

template <typename T, int VEC> __device__ inline void load_vec(const T *p, float (&x)[VEC]) {
    const typename RowVec<T, VEC>::Type v = *reinterpret_cast<const typename RowVec<T, VEC>::Type *>(p);
    if constexpr (VEC == 1) x[0] = (float)v;
    else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = (float)v[e];
    }
}
template <typename T, int VEC, bool PAST = false> __device__ inline void store_vec(T *p, const float (&x)[VEC]) {
    typename RowVec<T, VEC>::Type v;
    if constexpr (VEC == 1) v = (T)x[0];
    else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = (T)x[e];
    }
    store_streaming<PAST>(reinterpret_cast<typename RowVec<T, VEC>::Type *>(p), v);
}

// Rows of the jagged tensor that there are: offsets[B], if given, at most the buffer's.
__device__ inline int64_t rows_there(const int64_t *offsets, int64_t B, int64_t rows) {
    if (!offsets) return rows;
    const int64_t have = offsets[B];
    return have < 0 ? 0 : have < rows ? have : rows;
}

}  // namespace jfa
