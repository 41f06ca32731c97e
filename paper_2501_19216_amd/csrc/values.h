// Neighbouring float or bfloat16 values as loads and stores move them
// (block_norm.hip, layer_norm.hip, embedding.hip): up to 16 bytes at an
// element's alignment, taken apart into floats and joined again with one
// rounding to nearest even.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>
#include <utility>

namespace e2f {

// f(k) for k = 0 .. N - 1, each k a constant: what k indexes stays in registers
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}
// V channels as they are stored, in registers; the address needs no more than
// an element's alignment
template <typename T, int V>
struct Raw;
#define E2F_RAW(T, V, R)                                                                     \
  template <>                                                                                \
  struct Raw<T, V> {                                                                         \
    typedef R type;                                                                          \
    typedef R __attribute__((aligned(sizeof(T)))) any;                                       \
    static __device__ __forceinline__ type load(const char* p) { return *(const any*)p; }   \
    static __device__ __forceinline__ void store(char* p, type v) { *(any*)p = v; }          \
  };
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
struct bf16_t {
  unsigned short bits;
};
E2F_RAW(float, 1, float)
E2F_RAW(float, 2, f2)
E2F_RAW(float, 4, f4)
E2F_RAW(bf16_t, 1, unsigned short)
E2F_RAW(bf16_t, 2, unsigned)
E2F_RAW(bf16_t, 4, u2)
E2F_RAW(bf16_t, 8, u4)
#undef E2F_RAW

__device__ __forceinline__ float part(float v, int) { return v; }
__device__ __forceinline__ float part(f2 v, int u) { return v[u]; }
__device__ __forceinline__ float part(f4 v, int u) { return v[u]; }
__device__ __forceinline__ float part(unsigned v, int u) { return __uint_as_float(u ? v & 0xffff0000u : v << 16); }
__device__ __forceinline__ float part(unsigned short v, int) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ float part(u2 v, int u) { return part(v[u >> 1], u & 1); }
__device__ __forceinline__ float part(u4 v, int u) { return part(v[u >> 1], u & 1); }
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned pair(float x, float y) {  // round to nearest even
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f2){x, y}, b2));
}
__device__ __forceinline__ void join(const float* f, float& v) { v = f[0]; }
__device__ __forceinline__ void join(const float* f, f2& v) { v = (f2){f[0], f[1]}; }
__device__ __forceinline__ void join(const float* f, f4& v) { v = (f4){f[0], f[1], f[2], f[3]}; }
__device__ __forceinline__ void join(const float* f, unsigned& v) { v = pair(f[0], f[1]); }
__device__ __forceinline__ void join(const float* f, unsigned short& v) { v = __builtin_bit_cast(unsigned short, (__bf16)f[0]); }
__device__ __forceinline__ void join(const float* f, u4& v) {
  v = (u4){pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7])};
}
__device__ __forceinline__ void join(const float* f, u2& v) { v = (u2){pair(f[0], f[1]), pair(f[2], f[3])}; }

// An address as the workgroup's part, the same for its threads (the array's first row of the workgroup, and the
// component in it), and a thread's own 32 bits: one register addresses every component of every array
template <typename T, int V>
__device__ __forceinline__ void store(void* base, int64_t uniform, unsigned own, const float (&f)[V]) {
  typename Raw<T, V>::type v;
  join(f, v);
  Raw<T, V>::store((char*)base + uniform * (int)sizeof(T) + own, v);
}

}  // namespace e2f
