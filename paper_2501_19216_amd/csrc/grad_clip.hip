// The norm over all gradients of a training step and the gradients clipped by it:
//   norm = sqrt(sum over every tensor of g^2),   out = g min(1, max_norm / (norm + 1e-6)).
// Both passes stream: the norm reads every value once, the clipping reads and
// writes it once, and nothing else bounds them but memory.  The tensors'
// pointers and sizes travel in the kernel arguments (128 tensors a launch), so
// that no table has to be copied to the device and a captured graph keeps its
// own.  A tensor is cut into chunks of one size, a workgroup each; a chunk's
// values are squared and summed in float64, in which no float's square
// overflows and 10^9 of them lose nothing that a float result shows; its sum
// goes to a place of its own, and one workgroup adds those in a fixed order:
// no atomics, the same bits every time.
#include <hip/hip_runtime.h>

#include "e2f_launch.h"

namespace e2f {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned short v8s __attribute__((ext_vector_type(8)));
typedef float v4fu __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short v8su __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float bf16_float(unsigned short u) { return __uint_as_float((unsigned)u << 16); }
__device__ __forceinline__ unsigned short float_bf16(float x) {
  return __builtin_bit_cast(unsigned short, (__bf16)x);  // round to nearest even
}

// tensor of this workgroup, and its chunk
__device__ __forceinline__ int find_tensor(const TensorTable& t, int b) {
  int lo = 0, hi = t.count - 1;  // the last whose first block is <= b (tensors of no values have none)
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= b)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

__global__ __launch_bounds__(256) void k_grad_sumsq(TensorTable t, int64_t chunk, double* __restrict__ part) {
  const int b = blockIdx.x, k = find_tensor(t, b);
  const int64_t lo = (int64_t)(b - t.first[k]) * chunk, hi = min(lo + chunk, t.n[k]);
  double s = 0.0;
  if (t.bf16[k >> 5] >> (k & 31) & 1) {
    const unsigned short* g = (const unsigned short*)t.in[k];
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
      const double x = bf16_float(g[i]);
      s += x * x;
    }
  } else {
    const float* g = (const float*)t.in[k];
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
      const double x = g[i];
      s += x * x;
    }
  }
  __shared__ double w[4];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[b] = w[0] + w[1] + w[2] + w[3];
}

__global__ __launch_bounds__(1024) void k_grad_norm(const double* __restrict__ part, int count,
                                                    double* __restrict__ sumsq, float* __restrict__ norm) {
  double s = 0.0;
  for (int i = threadIdx.x; i < count; i += 1024) s += part[i];
  __shared__ double w[16];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int i = 0; i < 16; ++i) v += w[i];
    if (sumsq) *sumsq = v;
    if (norm) *norm = (float)sqrt(v);
  }
}

__global__ __launch_bounds__(256) void k_grad_clip(TensorTable t, int64_t chunk, const double* __restrict__ sumsq,
                                                   float max_norm) {
  const double c = (double)max_norm / (sqrt(*sumsq) + 1e-6);
  const float coef = c > 1.0 ? 1.0f : (float)c;  // (a NaN stays one)
  const int b = blockIdx.x, k = find_tensor(t, b);
  const int64_t lo = (int64_t)(b - t.first[k]) * chunk, hi = min(lo + chunk, t.n[k]);
  if (coef == 1.0f && t.in[k] == t.out[k]) return;
  if (t.bf16[k >> 5] >> (k & 31) & 1) {
    const unsigned short* g = (const unsigned short*)t.in[k];
    unsigned short* o = (unsigned short*)t.out[k];
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) o[i] = float_bf16(bf16_float(g[i]) * coef);
  } else {
    const float* g = (const float*)t.in[k];
    float* o = (float*)t.out[k];
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) o[i] = g[i] * coef;
  }
}

// Calls f(table, blocks) for every kTableMax tensors, with the launch's first
// block in `at`.
template <typename F>
hipError_t each_table(int count, const void* const* in, void* const* out, const int64_t* n, const int32_t* dtype,
                      int64_t chunk, F f) {
  TensorTable t;
  for (int i = 0; i < count;) {
    t.count = 0;
    for (int w = 0; w < kTableMax / 32; ++w) t.bf16[w] = 0;
    int64_t blocks = 0;
    for (; i < count && t.count < kTableMax; ++i) {
      if (n[i] == 0) continue;
      const int64_t b = (n[i] + chunk - 1) / chunk;
      if (t.count && blocks + b > 0x7fffffff) break;
      const int k = t.count++;
      t.in[k] = in[i];
      t.out[k] = out ? out[i] : nullptr;
      t.n[k] = n[i];
      t.first[k] = (int)blocks;
      if (dtype[i]) t.bf16[k >> 5] |= 1u << (k & 31);
      blocks += b;
    }
    if (t.count == 0) continue;
    f(t, (unsigned)blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

int64_t grad_chunk(int64_t total) {
  const int64_t c = (total / 2048 + 1023) / 1024 * 1024;
  return c < 4096 ? 4096 : c > 65536 ? 65536 : c;
}

hipError_t launch_grad_norm(int count, const void* const* in, const int64_t* n, const int32_t* dtype, int64_t total,
                            double* part, double* sumsq, float* norm, hipStream_t s) {
  const int64_t chunk = grad_chunk(total);
  int64_t at = 0;
  hipError_t e = each_table(count, in, nullptr, n, dtype, chunk, [&](const TensorTable& t, unsigned blocks) {
    k_grad_sumsq<<<blocks, 256, 0, s>>>(t, chunk, part + at);
    at += blocks;
  });
  if (e != hipSuccess) return e;
  k_grad_norm<<<1, 1024, 0, s>>>(part, (int)at, sumsq, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(int count, const void* const* in, void* const* out, const int64_t* n,
                            const int32_t* dtype, int64_t total, const double* sumsq, float max_norm, hipStream_t s) {
  const int64_t chunk = grad_chunk(total);
  return each_table(count, in, out, n, dtype, chunk, [&](const TensorTable& t, unsigned blocks) {
    k_grad_clip<<<blocks, 256, 0, s>>>(t, chunk, sumsq, max_norm);
  });
}

}  // namespace e2f
