// Eight neighbouring values of a row at a time, as fp32 (internal).
#pragma once

#include "common.h"

namespace moe {

// As they lie in memory: loads can be requested together and widened where they are used.
template <typename T>
struct Raw8 {
    typename Store<T>::vec_t v[8 / Store<T>::VEC];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int q = 0; q < 8 / Store<T>::VEC; ++q) r.v[q] = reinterpret_cast<const typename Store<T>::vec_t*>(p)[q];
    return r;
}
template <typename T>
__device__ __forceinline__ float at8(const Raw8<T>& r, int i) {
    return Store<T>::get(r.v[i / Store<T>::VEC], i % Store<T>::VEC);
}
template <typename T>
__device__ __forceinline__ Raw8<T> round8(const float (&f)[8]) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i / Store<T>::VEC][i % Store<T>::VEC] = Store<T>::from_f32(f[i]);
    return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r) {
#pragma unroll
    for (int q = 0; q < 8 / Store<T>::VEC; ++q) reinterpret_cast<typename Store<T>::vec_t*>(p)[q] = r.v[q];
}

}  // namespace moe
