// Vectors of 1 to 8 elements of float, bfloat16 or half in registers: loads, stores, widening to float and rounding back.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace sae {

template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef unsigned short type; };
template <> struct Bits<4> { typedef unsigned int type; };
template <> struct Bits<8> { typedef uint2 type; };
template <> struct Bits<16> { typedef uint4 type; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// Two 16-bit elements of one word; a bfloat16 is the upper half of its float.
__device__ __forceinline__ float2 widen2(unsigned int w, const __nv_bfloat16*) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 widen2(unsigned int w, const __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ unsigned int round2(float a, float b, const __nv_bfloat16*) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned int*>(&v);
}
__device__ __forceinline__ unsigned int round2(float a, float b, const __half*) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned int*>(&v);
}

// Copies to shared memory that a thread waits for itself.  Two bytes have no asynchronous form.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const unsigned int s = (unsigned int)__cvta_generic_to_shared(to);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(s), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// V elements as they lie in memory; V * sizeof(T) is 2, 4, 8 or 16 bytes and the address a multiple of it.
template <typename T, int V>
struct Raw {
  typedef typename Bits<V * (int)sizeof(T)>::type B;
  B b;
  __device__ __forceinline__ void load(const T* p) { b = __ldg(reinterpret_cast<const B*>(p)); }          // nobody writes there while the kernel lives
  __device__ __forceinline__ void load_written(const T* p) { b = __ldcg(reinterpret_cast<const B*>(p)); } // another kernel of the call may
  __device__ __forceinline__ void clear() { b = B{}; }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<B*>(p) = b; }
  __device__ __forceinline__ void store_stream(T* p) const { __stcs(reinterpret_cast<B*>(p), b); }
  __device__ __forceinline__ void widen(float (&v)[V]) const {
    if constexpr (sizeof(T) == 4 || V == 1) {
      const T* e = reinterpret_cast<const T*>(&b);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = to_f(e[i]);
    } else {
      const unsigned int* w = reinterpret_cast<const unsigned int*>(&b);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) { const float2 f = widen2(w[i], (const T*)nullptr); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
    }
  }
  __device__ __forceinline__ void round(const float (&v)[V]) {
    if constexpr (sizeof(T) == 4 || V == 1) {
      T* e = reinterpret_cast<T*>(&b);
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = from_f<T>(v[i]);
    } else {
      unsigned int* w = reinterpret_cast<unsigned int*>(&b);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) w[i] = round2(v[2 * i], v[2 * i + 1], (const T*)nullptr);
    }
  }
};

// Lane-wise arithmetic on V floats, two at a time where V is even: sm_100a adds, multiplies and fuses pairs of floats in one
// instruction, each half rounded as the single operation rounds.  But a packed product that goes into a packed sum comes out as one
// fused operation, rounded once, .rn and --fmad=false notwithstanding (measured: 5.9 M of 25.7 M values of x * w + b were the
// fused ones; single operations are left apart).  Where both roundings are wanted, vmul_add has them.
__device__ __forceinline__ unsigned long long pair(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(unsigned long long r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }

template <int V>
__device__ __forceinline__ void vadd(float (&o)[V], const float (&a)[V], const float (&b)[V]) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      unsigned long long r;
      asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])));
      unpair(r, o[i], o[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = __fadd_rn(a[i], b[i]);
  }
}
template <int V>
__device__ __forceinline__ void vmul(float (&o)[V], const float (&a)[V], const float (&b)[V]) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      unsigned long long r;
      asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])));
      unpair(r, o[i], o[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = __fmul_rn(a[i], b[i]);
  }
}
// o = a * b + c, the product rounded before the sum: sums of single floats, which nothing fuses
template <int V>
__device__ __forceinline__ void vmul_add(float (&o)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
  vmul<V>(o, a, b);
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = __fadd_rn(o[i], c[i]);
}
// o = a * b + c, rounded once
template <int V>
__device__ __forceinline__ void vfma(float (&o)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      unsigned long long r;
      asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])), "l"(pair(c[i], c[i + 1])));
      unpair(r, o[i], o[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = __fmaf_rn(a[i], b[i], c[i]);
  }
}
// The same value in all lanes: a group's statistic where the V channels lie in one group, else one value a channel.
template <int V, bool WHOLE> struct Per;
template <int V> struct Per<V, true> {
  float v;
  template <typename F> __device__ __forceinline__ void set(F f) { v = f(0); }
  __device__ __forceinline__ float at(int) const { return v; }
  __device__ __forceinline__ void all(float (&o)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = v;
  }
};
template <int V> struct Per<V, false> {
  float v[V];
  template <typename F> __device__ __forceinline__ void set(F f) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = f(i);
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ void all(float (&o)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = v[i];
  }
};

}  // namespace sae
