// The norm over all gradients of a training step and the gradients clipped by it:
//   norm = sqrt(sum over every tensor of g^2),   out = g min(1, max_norm / (norm + 1e-6)).
// Both passes stream: the norm reads every value once, the clipping reads and
// writes it once, and nothing else bounds them but memory and, for lists of many small
// tensors, the host (33 million values in 300 tensors of float32 and bfloat16: 40 and 58 us).  The tensors'
// pointers and sizes travel in the kernel arguments (128 tensors a launch to clip,
// 192 to read, below 4 KB), so
// that no table has to be copied to the device and a captured graph keeps its
// own.  A tensor is cut into chunks of one size, a workgroup each; a chunk's
// values are squared and summed in float64, in which no float's square
// overflows and 10^9 of them lose nothing that a float result shows; its sum
// goes to a place of its own, and one workgroup adds those in a fixed order:
// no atomics, the same bits every time.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "e2f_launch.h"

namespace e2f {
namespace {

constexpr int64_t kMostBlocks = 0xffffffff / 256;  // of one launch, which holds below 2^32 threads

// the tensors of one launch
template <int N>
struct Table {
  static constexpr int MAX = N;
  const void* in[N];
  int64_t n[N];
  int first[N];  // first workgroup
  unsigned bf16[N / 32];
  int count;
};
typedef Table<192> ReadTable;
struct WriteTable : Table<128> {
  void* out[MAX];
};
static_assert(sizeof(ReadTable) <= 4064 && sizeof(WriteTable) <= 4064, "kernel arguments of 4 KB");

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void scaled(float& to, float x, float c) { to = x * c; }
__device__ __forceinline__ void scaled(unsigned short& to, unsigned short x, float c) {
  to = __builtin_bit_cast(unsigned short, (__bf16)(to_float(x) * c));  // round to nearest even
}

// 16 bytes of values, at an address of an element's alignment
template <typename T>
struct Pack {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};
template <typename T>
__device__ __forceinline__ Pack<T> load(const T* p) {
  Pack<T> r;
  __builtin_memcpy(&r, p, 16);
  return r;
}

// The values lo .. hi - 1 of an array: four(i) for every 16 bytes from i on of four in flight, 64 lanes side by
// side, from the first 16-byte boundary on; one(i) for those before it and behind
template <typename T, typename F, typename G>
__device__ __forceinline__ void each_value(const T* p, int64_t lo, int64_t hi, F four, G one) {
  constexpr int N = Pack<T>::N;
  const int64_t skew = (int64_t)((16 - (uintptr_t)(p + lo) % 16) % 16 / sizeof(T)), v0 = min(lo + skew, hi);
  const int64_t v1 = v0 + (hi - v0) / (N * 1024) * (N * 1024);  // whole rounds of 256 threads and four packs
  for (int64_t i = v0 + threadIdx.x * N; i < v1; i += N * 1024) four(i);
  for (int64_t i = lo + threadIdx.x; i < v0; i += 256) one(i);
  for (int64_t i = v1 + threadIdx.x; i < hi; i += 256) one(i);
}

// tensor of this workgroup, and its chunk
template <typename Table>
__device__ __forceinline__ int find_tensor(const Table& t, int b) {
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

__global__ __launch_bounds__(256) void k_grad_sumsq(ReadTable t, int64_t chunk, double* __restrict__ part) {
  const int b = blockIdx.x, k = find_tensor(t, b);
  const int64_t lo = (int64_t)(b - t.first[k]) * chunk, hi = min(lo + chunk, t.n[k]);
  double s = 0.0;
  auto sum = [&](const auto* g) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(g)>>;
    each_value(
        g, lo, hi,
        [&](int64_t i) {
          Pack<T> r[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) r[u] = load(g + i + u * 256 * Pack<T>::N);
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int x = 0; x < Pack<T>::N; ++x) {
              const double v = to_float(r[u].v[x]);
              s += v * v;
            }
        },
        [&](int64_t i) {
          const double v = to_float(g[i]);
          s += v * v;
        });
  };
  if (t.bf16[k >> 5] >> (k & 31) & 1)
    sum((const unsigned short*)t.in[k]);
  else
    sum((const float*)t.in[k]);
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

__global__ __launch_bounds__(256) void k_grad_clip(WriteTable t, int64_t chunk, const double* __restrict__ sumsq,
                                                   float max_norm) {
  const double c = (double)max_norm / (sqrt(*sumsq) + 1e-6);
  const float coef = c > 1.0 ? 1.0f : (float)c;  // (a NaN stays one)
  const int b = blockIdx.x, k = find_tensor(t, b);
  const int64_t lo = (int64_t)(b - t.first[k]) * chunk, hi = min(lo + chunk, t.n[k]);
  if (coef == 1.0f && t.in[k] == t.out[k]) return;
  auto scale = [&](const auto* g, auto* o) {
    using T = std::remove_pointer_t<decltype(o)>;
    each_value(
        g, lo, hi,
        [&](int64_t i) {
          Pack<T> r[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) r[u] = load(g + i + u * 256 * Pack<T>::N);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int x = 0; x < Pack<T>::N; ++x) scaled(r[u].v[x], r[u].v[x], coef);
            __builtin_memcpy(o + i + u * 256 * Pack<T>::N, &r[u], 16);
          }
        },
        [&](int64_t i) { scaled(o[i], g[i], coef); });
  };
  if (t.bf16[k >> 5] >> (k & 31) & 1)
    scale((const unsigned short*)t.in[k], (unsigned short*)t.out[k]);
  else
    scale((const float*)t.in[k], (float*)t.out[k]);
}

// Calls f(table, blocks) for as many tensors as a table holds after each other
template <typename Table, typename F>
hipError_t each_table(int count, const void* const* in, void* const* out, const int64_t* n, const int32_t* dtype,
                      int64_t chunk, F f) {
  Table t;
  for (int i = 0; i < count;) {
    t.count = 0;
    for (auto& w : t.bf16) w = 0;
    int64_t blocks = 0;
    for (; i < count && t.count < Table::MAX; ++i) {
      if (n[i] == 0) continue;
      const int64_t b = (n[i] + chunk - 1) / chunk;
      if (t.count && blocks + b > kMostBlocks) break;
      const int k = t.count++;
      t.in[k] = in[i];
      if constexpr (std::is_same_v<Table, WriteTable>) t.out[k] = out[i];
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
  hipError_t e = each_table<ReadTable>(count, in, nullptr, n, dtype, chunk, [&](const ReadTable& t, unsigned blocks) {
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
  return each_table<WriteTable>(count, in, out, n, dtype, chunk, [&](const WriteTable& t, unsigned blocks) {
    k_grad_clip<<<blocks, 256, 0, s>>>(t, chunk, sumsq, max_norm);
  });
}

}  // namespace e2f
