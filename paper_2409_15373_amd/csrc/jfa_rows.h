// Pieces shared by the operators on rows of any length (jfa_layer_norm.hip, jfa_embedding.hip).  Not part of the C ABI.
#pragma once
#include "jfa_common.h"

namespace jfa {

// Rows are moved 16 bytes of T at a time (kRowVec elements).  EVEN: every row starts on 16 bytes and has whole vectors.  Otherwise vectors start wherever the
// rows do, which the memory instructions allow (a vector that crosses a 64-byte boundary is two requests).  (Layer norm of 1001 bf16 a row,
// forward: element by element 1.1 TB/s, by vectors but the last of a row element by element 3.4, as here 4.4.)
template <typename T> constexpr int kRowVec = 16 / (int)sizeof(T);
template <typename T, int VEC, bool EVEN> struct RowVec { typedef T Type __attribute__((ext_vector_type(VEC))); };
template <typename T, int VEC> struct RowVec<T, VEC, false> { typedef T Type __attribute__((ext_vector_type(VEC), aligned(sizeof(T)))); };
template <typename T, int VEC> using RowRaw = typename RowVec<T, VEC, true>::Type;   // as it is held in registers

// What is not the row's is zero.
template <typename T, int VEC, bool EVEN> __device__ inline RowRaw<T, VEC> read_vec(const T *p, int64_t left) {
    if (EVEN || left >= VEC) return *reinterpret_cast<const typename RowVec<T, VEC, EVEN>::Type *>(p);
    RowRaw<T, VEC> v = {};
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (e < left) v[e] = p[e];
    return v;
}
template <typename T, int VEC> __device__ inline void widen_vec(const RowRaw<T, VEC> &v, float (&x)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = (float)v[e];
}
template <typename T, int VEC, bool EVEN> __device__ inline void load_vec(const T *p, int64_t left, float (&x)[VEC]) { widen_vec<T, VEC>(read_vec<T, VEC, EVEN>(p, left), x); }
template <typename T, int VEC, bool EVEN, bool PAST = false> __device__ inline void store_vec(T *p, int64_t left, const float (&x)[VEC]) {
    typename RowVec<T, VEC, EVEN>::Type v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (T)x[e];
    if (EVEN || left >= VEC) {
        auto *const dst = reinterpret_cast<typename RowVec<T, VEC, EVEN>::Type *>(p);
        if constexpr (PAST) __builtin_nontemporal_store(v, dst);
        else *dst = v;
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < left) p[e] = v[e];
    }
}

// Where the vector at `c` of a row of N elements is moved: the last one of a row that has no whole number of them ends with the row, over elements that
// the one before it has as well (both store the same values).  A row of less than a vector goes element by element.
template <int VEC, bool EVEN, typename I> __device__ inline I vec_at(I c, I N) { return EVEN || N < VEC || c + VEC <= N ? c : N - VEC; }

// Rows of the jagged tensor that there are: offsets[B], if given, at most the buffer's.
__device__ inline int64_t rows_there(const int64_t *offsets, int64_t B, int64_t rows) {
    if (!offsets) return rows;
    const int64_t have = offsets[B];
    return have < 0 ? 0 : have < rows ? have : rows;
}

}  // namespace jfa
