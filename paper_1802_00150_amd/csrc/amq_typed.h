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

// `valid` of the V = kPer16<T> elements at p, the others as 0.
template <typename T>
__device__ __forceinline__ void load16(const T* p, int valid, float (&out)[kPer16<T>]) {
  constexpr int V = kPer16<T>;
  if (valid >= V) {
    const Bytes16<T> b = *reinterpret_cast<const Bytes16<T>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = (float)b.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = i < valid ? (float)p[i] : 0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void store16(T* p, int valid, const float (&in)[kPer16<T>]) {
  constexpr int V = kPer16<T>;
  if (valid >= V) {
    Bytes16<T> b;
#pragma unroll
    for (int i = 0; i < V; ++i) b.v[i] = (T)in[i];
    *reinterpret_cast<Bytes16<T>*>(p) = b;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < valid) p[i] = (T)in[i];
  }
}

// V consecutive parameters of type P (V need not be kPer16<P>), absent ones (null) as `absent`.
template <typename P, int V>
__device__ __forceinline__ void load_params(const P* p, int64_t at, int valid, float absent, float (&out)[V]) {
  struct __attribute__((packed, aligned(sizeof(P)))) Group {
    P v[V];
  };
  if (!p) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = absent;
  } else if (valid >= V) {
    const Group b = *reinterpret_cast<const Group*>(p + at);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = (float)b.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = i < valid ? (float)p[at + i] : 0.0f;
  }
}

}  // namespace amq
