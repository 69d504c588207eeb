// Loads and stores of float, bfloat16 and half data for the training operators, 16 bytes at a time and at any element
// alignment, with all arithmetic in binary32.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace amq {

typedef __bf16 bf16;
typedef _Float16 f16;

template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);  // elements in 16 bytes

// 16 bytes from any address that is aligned to an element: the target's vector loads and stores take unaligned
// addresses, so rows of odd length or stride need no scalar path of their own.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 {
  T v[kPer16<T>];
};

// `valid` of the V elements at p as they are, the others as 0.  (A piece that ends early repeats its last element in place of
// those past it and drops them again: loads side by side, without a branch for each.)
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Elements {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Elements<T, V> fetch(const T* p, int valid) {
  if (valid >= V) return *reinterpret_cast<const Elements<T, V>*>(p);
  Elements<T, V> b;
  if (valid <= 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) b.v[i] = (T)0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) b.v[i] = p[i < valid ? i : valid - 1];
#pragma unroll
    for (int i = 0; i < V; ++i) b.v[i] = i < valid ? b.v[i] : (T)0.0f;
  }
  return b;
}
template <typename T>
__device__ __forceinline__ Bytes16<T> fetch16(const T* p, int valid) {
  return __builtin_bit_cast(Bytes16<T>, fetch<T, kPer16<T>>(p, valid));
}

template <typename T>
__device__ __forceinline__ void load16(const T* p, int valid, float (&out)[kPer16<T>]) {
  const Bytes16<T> b = fetch16(p, valid);
#pragma unroll
  for (int i = 0; i < kPer16<T>; ++i) out[i] = (float)b.v[i];
}

template <typename T, int V>
__device__ __forceinline__ void store(T* p, int valid, const float (&in)[V]) {
  Elements<T, V> b;
#pragma unroll
  for (int i = 0; i < V; ++i) b.v[i] = (T)in[i];
  if (valid >= V) {
    *reinterpret_cast<Elements<T, V>*>(p) = b;
    return;
  }
  // half of it, half of the rest, ...
  int at = 0;
#pragma unroll
  for (int n = V / 2; n > 0; n /= 2)
    if (valid & n) {
#pragma unroll
      for (int i = 0; i < n; ++i) p[at + i] = b.v[i];
#pragma unroll
      for (int i = 0; i + n < V; ++i) b.v[i] = b.v[i + n];
      at += n;
    }
}
// All V of them in one store, which the compiler makes of single elements only at times.
template <typename T, int V>
__device__ __forceinline__ void store_whole(T* p, const float (&in)[V]) {
  Elements<T, V> b;
#pragma unroll
  for (int i = 0; i < V; ++i) b.v[i] = (T)in[i];
  constexpr int kBytes = V * (int)sizeof(T);
  if constexpr (kBytes % 4 == 0) {
    typedef uint32_t Words __attribute__((ext_vector_type(kBytes / 4)));
    struct __attribute__((packed, aligned(sizeof(T)))) Unaligned {
      Words w;
    };
    reinterpret_cast<Unaligned*>(p)->w = __builtin_bit_cast(Words, b);
  } else {
    *reinterpret_cast<Elements<T, V>*>(p) = b;
  }
}
// The same past the caches: results that are not read again soon.
template <typename T, int V>
__device__ __forceinline__ void store_streaming(T* p, const float (&in)[V]) {
  Elements<T, V> b;
#pragma unroll
  for (int i = 0; i < V; ++i) b.v[i] = (T)in[i];
  typedef uint32_t Words __attribute__((ext_vector_type(V * sizeof(T) / 4), aligned(sizeof(T))));
  __builtin_nontemporal_store(__builtin_bit_cast(Words, b), reinterpret_cast<Words*>(p));
}
template <typename T>
__device__ __forceinline__ void store16(T* p, int valid, const float (&in)[kPer16<T>]) {
  if (valid > 0) store<T, kPer16<T>>(p, valid, in);
}

// V consecutive parameters of type P (V need not be kPer16<P>), absent ones (null) as `absent`.
template <typename P, int V>
__device__ __forceinline__ void load_params(const P* p, int64_t at, int valid, float absent, float (&out)[V]) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = absent;
  } else {
    const Elements<P, V> b = fetch<P, V>(p + at, valid);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = (float)b.v[i];
  }
}

}  // namespace amq
