// Element types of the model operators (fp32, binary16, bfloat16) and 16-byte
// accesses to their rows at any element alignment.
#pragma once
#include "kkm_internal.h"

namespace kkm {

typedef __bf16 bf16_t;

// Vector of 16 bytes of T whose address need only suit T: gfx950 takes global
// loads and stores of any width at any address.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T>
using raw_vec = T __attribute__((ext_vector_type(kVec<T>)));
template <typename T>
using any_vec = raw_vec<T> __attribute__((aligned(alignof(T))));

// N elements from element i of a row of d, zero from d on.
template <int N, typename T>
using raw_n = T __attribute__((ext_vector_type(N)));
template <int N, typename T>
using any_n = raw_n<N, T> __attribute__((aligned(alignof(T))));
template <int N, typename T>
__device__ inline raw_n<N, T> load_n(const T* row, int i, int d) {
  if (i + N <= d) return *(const any_n<N, T>*)(row + i);
  raw_n<N, T> r;
#pragma unroll
  for (int e = 0; e < N; ++e) r[e] = i + e < d ? row[i + e] : (T)0.f;
  return r;
}

template <typename T>
__device__ inline void to_floats(const raw_vec<T>& r, float (&v)[kVec<T>]) {
#pragma unroll
  for (int e = 0; e < kVec<T>; ++e) v[e] = (float)r[e];
}

template <typename T>
__device__ inline raw_vec<T> load_raw(const T* row, int i, int d) {
  return load_n<kVec<T>>(row, i, d);
}
template <typename T>
__device__ inline void load_part(const T* row, int i, int d, float (&v)[kVec<T>]) {
  to_floats<T>(load_raw(row, i, d), v);
}

// One rounding to T, to nearest even.
template <typename T>
__device__ inline void store_part(T* row, int i, int d, const float (&v)[kVec<T>]) {
  if (i + kVec<T> <= d) {
    raw_vec<T> r;
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) r[e] = (T)v[e];
    *(any_vec<T>*)(row + i) = r;
  } else {
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e)
      if (i + e < d) row[i + e] = (T)v[e];
  }
}

// Elements i .. i + N - 1 of a vector of WT beside a vector of another type;
// `none` past d and where there is no vector.
template <int N, typename WT>
__device__ inline void load_beside(const WT* w, int i, int d, float none, float (&v)[N]) {
  typedef WT raw __attribute__((ext_vector_type(N)));
  typedef raw any __attribute__((aligned(alignof(WT))));
  if (w && i + N <= d) {
    const raw r = *(const any*)(w + i);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)r[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = w && i + e < d ? (float)w[i + e] : none;
  }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

}  // namespace kkm
