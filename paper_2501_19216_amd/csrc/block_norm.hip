// The norms before and after a block, with its gate, scale and residual sum, on
// irrep features [N][(L+1)^2][C] (one component: the plain root-mean-square norm of a
// Transformer's activations):
//   rms(v)^2 = mean over the degrees l of the mean over (m, c) of v^2, plus eps
//   out    = x + s[l][c] sigma(gate) p[l][c] b / rms(b)        (b: the block's output)
//   normed = w[l][c] out / rms(out)                            (the next block's input)
// and the gradients, with rb = 1 / rms(b), ro = 1 / rms(out), a_l = 1 / ((L+1)(2l+1)C),
// do, dn the gradients of out and normed:
//   dt = do + ro w dn - ro^3 a_l out (sum of dn w out)         (= dx)
//   u  = dt s sigma p,   db = rb u - rb^3 a_l b (sum of u b),
//   dgate = sigma (1 - sigma) sum_m dt s p b rb over the degrees that the gate serves,
//   ds = sum of dt sigma p b rb,  dp = sum of dt sigma s b rb,  dw = sum of dn out ro  over (atom, m).
// Every value is read once and written once: an atom's rows stay in registers
// between the two reductions, a thread holding V channels of every component, so
// that what belongs to a channel or a degree (weights, gates, their gradients) stays
// in the thread and only the two norms go across threads.  ds and dp are one sum,
// A = sum of dt sigma b rb, times p and s.  Sums, statistics and everything
// between the loads and the stores are float; outputs are rounded once.
#include <hip/hip_runtime.h>

#include "e2f_launch.h"

namespace e2f {
namespace {

// V channels as they are stored; the address needs no more than an element's alignment
template <typename T, int V>
struct Vec {
  T v[V];
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
  Vec<T, V> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float* f) {
  Vec<T, V> r;
#pragma unroll
  for (int u = 0; u < V; ++u) r.v[u] = (T)f[u];  // round to nearest even
  __builtin_memcpy(p, &r, sizeof(r));
}

// Sum over the `tpr` threads of a row (a power of two); red: a float for every wave
__device__ __forceinline__ float row_sum(float v, int tpr, float* red) {
  for (int o = min(tpr, 64) >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if (tpr <= 64) return v;
  const int wave = threadIdx.x >> 6, per = tpr >> 6, w0 = wave / per * per;
  __syncthreads();  // (the sums before have been read)
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = w0; w < w0 + per; ++w) v += red[w];
  return v;
}

// (by exp of -|x|: a shut gate keeps its digits, down to the smallest floats)
__device__ __forceinline__ float sigmoid(float x) {
  const float e = expf(-fabsf(x));
  return (x < 0.0f ? e : 1.0f) / (1.0f + e);
}

// What a thread keeps of the weights: V channels of every degree
template <int L, int V>
struct Weights {
  float post[L + 1][V], scale[L + 1][V], pre[L + 1][V];
  __device__ __forceinline__ void read(const NormArgs& a, int c, bool on) {
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        post[l][u] = a.post_w && on ? a.post_w[l * a.C + c + u] : 1.0f;
        scale[l][u] = a.scale && on ? a.scale[l * a.C + c + u] : 1.0f;
        pre[l][u] = a.pre_w && on ? a.pre_w[l * a.C + c + u] : 1.0f;
      }
  }
};

template <int L, typename T, int V>
__device__ __forceinline__ void read_gates(const NormArgs& a, int64_t row, int c, bool on, float (&g)[L + 1][V]) {
#pragma unroll
  for (int l = 0; l <= L; ++l) {
    if (l > 0 && a.G == 1) {
#pragma unroll
      for (int u = 0; u < V; ++u) g[l][u] = g[0][u];
      continue;
    }
    if (a.G && on) {
      const Vec<T, V> v = load<T, V>((const T*)a.gate + (row * a.G + l) * a.C + c);
#pragma unroll
      for (int u = 0; u < V; ++u) g[l][u] = sigmoid(to_float(v.v[u]));
    } else {
#pragma unroll
      for (int u = 0; u < V; ++u) g[l][u] = 1.0f;
    }
  }
}

// The thread's values of one array: in registers, or (KEEP false: rows larger
// than the registers) read again where they are used
template <typename T, int V, int K, bool KEEP>
struct Held {
  Vec<T, V> v[KEEP ? K : 1];
  const T* p;
  int C;
  bool on;
  __device__ __forceinline__ void begin(const void* base, int64_t row, int C_, int c, bool on_) {
    p = (const T*)base + row * K * C_ + c;
    C = C_;
    on = on_ && base;
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = on ? load<T, V>(p + k * C) : Vec<T, V>{};
    }
  }
  __device__ __forceinline__ void get(int k, float (&f)[V]) const {
    Vec<T, V> r{};
    if constexpr (KEEP)
      r = v[k];
    else if (on)
      r = load<T, V>(p + k * C);
#pragma unroll
    for (int u = 0; u < V; ++u) f[u] = to_float(r.v[u]);
  }
};

template <int L, typename T, int V, bool KEEP>
__global__ __launch_bounds__(KEEP ? 256 : 1024) void k_norm_forward(NormArgs a, int tpr, T* out, T* normed, float* rstd) {
  constexpr int K = (L + 1) * (L + 1);
  __shared__ float red[16];
  const int slot = threadIdx.x / tpr, c = threadIdx.x % tpr * V, slots = blockDim.x / tpr;
  const int64_t row = (int64_t)blockIdx.x * slots + slot;
  const bool on = row < a.n && c < a.C;
  Weights<L, V> w;
  w.read(a, c, on);
  Held<T, V, K, KEEP> x, b;
  x.begin(a.x, row, a.C, c, on);
  float rb = 1.0f, gate[L + 1][V];
  if (a.block) {
    b.begin(a.block, row, a.C, c, on);
    read_gates<L, T, V>(a, row, c, on, gate);
    if (a.post_w) {
      float s = 0.0f;
#pragma unroll
      for (int l = 0; l <= L; ++l) {
        float t = 0.0f;
#pragma unroll
        for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
          float f[V];
          b.get(k, f);
#pragma unroll
          for (int u = 0; u < V; ++u) t += f[u] * f[u];
        }
        s += t * (1.0f / (2 * l + 1));
      }
      rb = 1.0f / sqrtf(row_sum(s, tpr, red) / (float)((L + 1) * a.C) + a.eps);
    }
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) gate[l][u] *= w.scale[l][u] * w.post[l][u] * rb;
  }
  // the residual sum, where it is needed again
  auto sum_at = [&](int l, int k, float(&o)[V]) {
    x.get(k, o);
    if (!a.block) return;
    float f[V];
    b.get(k, f);
#pragma unroll
    for (int u = 0; u < V; ++u) o[u] += gate[l][u] * f[u];
  };
  float ro = 1.0f, s = 0.0f;
#pragma unroll
  for (int l = 0; l <= L; ++l) {
    float t = 0.0f;
#pragma unroll
    for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
      float o[V];
      sum_at(l, k, o);
#pragma unroll
      for (int u = 0; u < V; ++u) t += o[u] * o[u];
      if (out && on) store<T, V>(out + (row * K + k) * a.C + c, o);
    }
    s += t * (1.0f / (2 * l + 1));
  }
  if (a.pre_w) {
    ro = 1.0f / sqrtf(row_sum(s, tpr, red) / (float)((L + 1) * a.C) + a.eps);
    if (on) {
#pragma unroll
      for (int l = 0; l <= L; ++l)
#pragma unroll
        for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
          float o[V];
          sum_at(l, k, o);
#pragma unroll
          for (int u = 0; u < V; ++u) o[u] *= ro * w.pre[l][u];
          store<T, V>(normed + (row * K + k) * a.C + c, o);
        }
    }
  }
  if (rstd && row < a.n && c == 0) rstd[2 * row] = rb, rstd[2 * row + 1] = ro;
}

template <int L, typename T, int V, bool KEEP>
__global__ __launch_bounds__(KEEP ? 256 : 1024) void k_norm_backward(NormArgs a, NormGrad g, int tpr) {
  constexpr int K = (L + 1) * (L + 1);
  extern __shared__ float sums[];  // [2][L + 1][C], with more than one row a workgroup
  __shared__ float red[16];
  const int slot = threadIdx.x / tpr, c = threadIdx.x % tpr * V, slots = blockDim.x / tpr;
  Weights<L, V> w;
  w.read(a, c, c < a.C);
  float sa[L + 1][V] = {}, sp[L + 1][V] = {};  // the weights' sums over the thread's rows
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n; first += (int64_t)gridDim.x * slots) {
    const int64_t row = first + slot;
    const bool on = row < a.n && c < a.C;
    const float rb = on ? g.rstd[2 * row] : 0.0f, ro = on ? g.rstd[2 * row + 1] : 0.0f;
    Held<T, V, K, KEEP> x, b, dn, dout;
    x.begin(a.x, row, a.C, c, on);
    if (a.pre_w) dn.begin(g.gnormed, row, a.C, c, on);
    dout.begin(g.gout, row, a.C, c, on);
    float gate[L + 1][V], f1[L + 1][V];
    if (a.block) {
      b.begin(a.block, row, a.C, c, on);
      read_gates<L, T, V>(a, row, c, on, gate);
#pragma unroll
      for (int l = 0; l <= L; ++l)
#pragma unroll
        for (int u = 0; u < V; ++u) f1[l][u] = gate[l][u] * w.scale[l][u] * w.post[l][u] * rb;
    }
    auto sum_at = [&](int l, int k, float(&o)[V]) {
      x.get(k, o);
      if (!a.block) return;
      float f[V];
      b.get(k, f);
#pragma unroll
      for (int u = 0; u < V; ++u) o[u] += f1[l][u] * f[u];
    };
    float s1 = 0.0f;
    if (a.pre_w) {
#pragma unroll
      for (int l = 0; l <= L; ++l) {
        float t[V] = {};
#pragma unroll
        for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
          float o[V], d[V];
          sum_at(l, k, o);
          dn.get(k, d);
#pragma unroll
          for (int u = 0; u < V; ++u) t[u] += o[u] * d[u];
        }
#pragma unroll
        for (int u = 0; u < V; ++u) s1 += w.pre[l][u] * t[u], sp[l][u] += ro * t[u];
      }
      s1 = row_sum(on ? s1 : 0.0f, tpr, red) * ro * ro * ro / (float)((L + 1) * a.C);
    }
    // dt, where it is needed again
    auto total_at = [&](int l, int k, float(&d)[V]) {
      dout.get(k, d);
      if (!a.pre_w) return;
      float o[V], f[V];
      sum_at(l, k, o);
      dn.get(k, f);
#pragma unroll
      for (int u = 0; u < V; ++u) d[u] += ro * w.pre[l][u] * f[u] - s1 * (1.0f / (2 * l + 1)) * o[u];
    };
    float s2 = 0.0f, gg[V] = {};
#pragma unroll
    for (int l = 0; l <= L; ++l) {
      float t[V] = {};
#pragma unroll
      for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
        float d[V], f[V];
        total_at(l, k, d);
        if (on && g.gx) store<T, V>((T*)g.gx + (row * K + k) * a.C + c, d);
        if (!a.block) continue;
        b.get(k, f);
#pragma unroll
        for (int u = 0; u < V; ++u) t[u] += d[u] * f[u];
      }
      if (!a.block) continue;
      float dg[V];
#pragma unroll
      for (int u = 0; u < V; ++u) {
        s2 += gate[l][u] * w.scale[l][u] * w.post[l][u] * t[u];
        sa[l][u] += gate[l][u] * rb * t[u];
        dg[u] = (1.0f - gate[l][u]) * f1[l][u] * t[u];
        gg[u] += dg[u];
      }
      if (on && g.ggate && a.G > 1) store<T, V>((T*)g.ggate + (row * a.G + l) * a.C + c, dg);
    }
    if (!a.block) continue;
    if (on && g.ggate && a.G == 1) store<T, V>((T*)g.ggate + row * a.C + c, gg);
    if (!g.gblock) continue;
    s2 = a.post_w ? row_sum(on ? s2 : 0.0f, tpr, red) * rb * rb * rb / (float)((L + 1) * a.C) : 0.0f;
    if (on) {
#pragma unroll
      for (int l = 0; l <= L; ++l)
#pragma unroll
        for (int k = l * l; k < (l + 1) * (l + 1); ++k) {
          float d[V], f[V];
          total_at(l, k, d);
          b.get(k, f);
#pragma unroll
          for (int u = 0; u < V; ++u) d[u] = f1[l][u] * d[u] - s2 * (1.0f / (2 * l + 1)) * f[u];
          store<T, V>((T*)g.gblock + (row * K + k) * a.C + c, d);
        }
    }
  }
  if (!g.part) return;
  float* mine = g.part + (int64_t)blockIdx.x * 2 * (L + 1) * a.C;
  for (int k = 0; k < slots; ++k) {  // the workgroup's rows, one after the other
    if (slots > 1) __syncthreads();
    if (k != slot || c >= a.C) continue;
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const int at = l * a.C + c + u, bt = (L + 1) * a.C + at;
        const float va = sa[l][u] + (k ? sums[at] : 0.0f), vp = sp[l][u] + (k ? sums[bt] : 0.0f);
        if (k + 1 < slots)
          sums[at] = va, sums[bt] = vp;
        else
          mine[at] = va, mine[bt] = vp;
      }
  }
}

// The weights' gradients from the workgroups' sums: 64 columns a workgroup
__global__ __launch_bounds__(1024) void k_norm_weights(NormArgs a, NormGrad g, int parts, int count) {
  __shared__ double red[2][16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), s = threadIdx.x >> 6;
  double va = 0.0, vp = 0.0;
  if (c < count)
    for (int b = s; b < parts; b += 16) {
      va += g.part[(int64_t)b * 2 * count + c];
      vp += g.part[(int64_t)b * 2 * count + count + c];
    }
  red[0][s][threadIdx.x & 63] = va, red[1][s][threadIdx.x & 63] = vp;
  __syncthreads();
  if (s || c >= count) return;
  for (int k = 1; k < 16; ++k) va += red[0][k][threadIdx.x], vp += red[1][k][threadIdx.x];
  if (g.gscale) g.gscale[c] = (float)(va * (a.post_w ? a.post_w[c] : 1.0f));
  if (g.gpost_w) g.gpost_w[c] = (float)(va * (a.scale ? a.scale[c] : 1.0f));
  if (g.gpre_w) g.gpre_w[c] = (float)vp;
}

// Channels of a thread: as many as keep a row's arrays in its registers
int channels_per_thread(int L, bool bf16) { return L <= 1 ? 4 : L <= 3 ? 2 : bf16 ? 2 : 1; }

struct Shape {
  int V, tpr, threads;
  bool keep;
};
Shape shape_of(int L, int C, bool bf16) {
  Shape s;
  s.V = channels_per_thread(L, bf16);
  s.tpr = 1;
  while (s.tpr * s.V < C) s.tpr <<= 1;
  s.keep = s.tpr <= 256;
  s.threads = s.keep ? 256 : s.tpr;
  return s;
}

}  // namespace

int norm_parts(int L, int C, bool bf16, int n) {
  const Shape s = shape_of(L, C, bf16);
  const int slots = s.threads / s.tpr;
  const int64_t want = ((int64_t)n + slots - 1) / slots;
  return (int)(want < 1024 ? want : 1024);
}

#define E2F_NORM_V(LL, T, VV)      \
  if (s.keep)                      \
    E2F_NORM(LL, T, VV, true);     \
  else                             \
    E2F_NORM(LL, T, VV, false);    \
  break;
#define E2F_NORM_SWITCH                                              \
  switch (L * 2 + (bf16 ? 1 : 0)) {                                  \
    case 0: E2F_NORM_V(0, float, 4) case 1: E2F_NORM_V(0, __bf16, 4) \
    case 2: E2F_NORM_V(1, float, 4) case 3: E2F_NORM_V(1, __bf16, 4) \
    case 4: E2F_NORM_V(2, float, 2) case 5: E2F_NORM_V(2, __bf16, 2) \
    case 6: E2F_NORM_V(3, float, 2) case 7: E2F_NORM_V(3, __bf16, 2) \
    case 8: E2F_NORM_V(4, float, 1) case 9: E2F_NORM_V(4, __bf16, 2) \
    case 10: E2F_NORM_V(5, float, 1) case 11: E2F_NORM_V(5, __bf16, 2) \
    case 12: E2F_NORM_V(6, float, 1) case 13: E2F_NORM_V(6, __bf16, 2) \
    default: return hipErrorInvalidValue;                            \
  }

hipError_t launch_norm_forward(int L, bool bf16, const NormArgs& a, void* out, void* normed, float* rstd,
                               hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const Shape s = shape_of(L, a.C, bf16);
  const int slots = s.threads / s.tpr;
  const unsigned grid = (unsigned)(((int64_t)a.n + slots - 1) / slots);
#define E2F_NORM(LL, T, VV, KEEP) \
  k_norm_forward<LL, T, VV, KEEP><<<grid, s.threads, 0, st>>>(a, s.tpr, (T*)out, (T*)normed, rstd)
  E2F_NORM_SWITCH
#undef E2F_NORM
  return hipGetLastError();
}

hipError_t launch_norm_backward(int L, bool bf16, const NormArgs& a, const NormGrad& g, hipStream_t st) {
  const int count = (L + 1) * a.C, parts = a.n ? norm_parts(L, a.C, bf16, a.n) : 0;
  if (a.n) {
    const Shape s = shape_of(L, a.C, bf16);
    const size_t lds = s.threads > s.tpr ? sizeof(float) * 2 * count : 0;
#define E2F_NORM(LL, T, VV, KEEP) k_norm_backward<LL, T, VV, KEEP><<<parts, s.threads, lds, st>>>(a, g, s.tpr)
    E2F_NORM_SWITCH
#undef E2F_NORM
  }
  if (g.gscale || g.gpost_w || g.gpre_w) k_norm_weights<<<(count + 63) / 64, 1024, 0, st>>>(a, g, parts, count);
  return hipGetLastError();
}

}  // namespace e2f
