// The layer norm of irrep features [N][(L+1)^2][C]: the scalars by their mean and variance over the channels, all
// higher degrees by one root mean square that rotations leave alone; one component is the plain layer norm of rows,
// with the activation of a radial network behind it:
//   m = mean_c x_0,  r0 = 1 / sqrt(mean_c (x_0 - m)^2 + eps),  h = (x_0 - m) r0,
//   z = w_0 h + b,   y_0 = z, or z sigma(z),
//   r1 = 1 / sqrt(mean over l >= 1 of the mean over (m, c) of x_l^2, plus eps),   y_l = w_l x_l r1,
// and the gradients, with a_l = 1 / (L (2l+1) C) and g the gradient of y:
//   dz = g_0, or g_0 sigma(z) (1 + z (1 - sigma(z))),   u = w_0 dz,
//   dx_0 = r0 (u - mean u - h mean(u h)),   dw_0 = sum of dz h,   db = sum of dz  over the atoms,
//   dx_l = r1 u_l - r1^3 a_l x_l (sum of u x),  u_l = w_l g_l,   dw_l = sum of g x r1 over (atom, m).
// Every value is read once and written once.  A row stays in registers between its reductions; the variance is taken
// of the differences from the mean, so that rows far from zero keep their digits.  The backward takes the row's
// statistics from x again, which it reads anyway: nothing is kept from the forward.  Sums, statistics and everything
// between loads and stores are float; outputs are rounded once.
//
// 20,000 atoms, L = 4, 128 float channels: 87 us forward, 155 backward and 5 for the weights' sums, the rate of a
// copy (5.1 TB/s) for all that is read and written.  A million rows of 64 bfloat16 channels with their activation: 64
// us forward (4.0 TB/s), 104 backward (3.7), where the activation's arithmetic begins to show.  Times at the rules below
// are of the forward, or of the backward with the weights' sums, on the same rows over and over.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "e2f_launch.h"
#include "values.h"
#include "wave.h"

namespace e2f {
namespace {

// Sums of N values over the `tpr` threads of a row (a power of two, up to eight waves)
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int tpr, float (*red)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], tpr);
  if (tpr <= 64) return;
  const int wave = threadIdx.x >> 6, per = tpr >> 6, w0 = wave / per * per;
  __syncthreads();  // (the sums before have been read)
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) red[wave][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.0f;
  for (int w = w0; w < w0 + per; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += red[w][i];
}

// (by the power of -|x|, whose argument keeps its low part: a shut gate keeps its digits, to 6 roundings down to
// 2^-126.  With the library's exponential and an IEEE quotient a million rows of 64 bfloat16 channels take 77 us
// forward and 129 backward, this way 55 and 111)
__device__ __forceinline__ float sigmoid(float x) {
  constexpr float kLog2e = 1.44269504f, kLow = 1.92596299e-8f, kLn2 = 0.693147181f;
  const float a = -fabsf(x), hi = a * kLog2e, lo = fmaf(a, kLog2e, -hi) + a * kLow;
  float e = __builtin_amdgcn_exp2f(hi);
  e = fmaf(e, hi > -INFINITY ? lo * kLn2 : 0.0f, e);
  return (x < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
}

// Where a thread's values lie: V neighbouring channels of each of S pieces, which are the components (L > 0), or
// stretches of tpr V channels of a row (L = 0), the last of them cut where the row ends.  The first S0 pieces hold
// scalars; W sets of weights
template <int L, int V, int J>
struct Place {
  static constexpr int S = L ? (L + 1) * (L + 1) : J, S0 = L ? 1 : J, W = L ? L + 1 : J;
  int C, t, tpr;
  __device__ __forceinline__ int channel(int s) const { return L ? t * V : (s * tpr + t) * V; }
  __device__ __forceinline__ int offset(int s) const { return L ? s * C + t * V : (s * tpr + t) * V; }
  // whether the piece's value u lies before the row's end (pieces are whole unless the end cuts one)
  __device__ __forceinline__ bool within(int s, int u, bool tail) const { return channel(s) + (tail ? u : 0) < C; }
  // (weights: of a degree, of a stretch)
  __device__ __forceinline__ int weight(int i) const { return L ? i * C + t * V : (i * tpr + t) * V; }
};

// The thread's values of a row as they are stored; what lies behind the row's end is zero
template <typename T, int L, int V, int J, bool TAIL>
struct Row {
  typedef Place<L, V, J> P;
  typename Raw<T, V>::type v[P::S];
  float end[V];  // (TAIL: the values of the piece that the row's end cuts)
  __device__ __forceinline__ void load(const T* p, const P& at) {
#pragma unroll
    for (int s = 0; s < P::S; ++s)
      v[s] = at.channel(s) + V <= at.C ? Raw<T, V>::load((const char*)(p + at.offset(s))) : typename Raw<T, V>::type{};
    if constexpr (TAIL) {
      const int c = at.C / V * V;
      if (c / V % at.tpr == at.t)
#pragma unroll
        for (int u = 0; u < V; ++u) end[u] = c + u < at.C ? part(Raw<T, 1>::load((const char*)(p + c + u)), 0) : 0.0f;
    }
  }
  __device__ __forceinline__ void values(const P& at, float (&f)[P::S][V]) const {
#pragma unroll
    for (int s = 0; s < P::S; ++s) {
      const bool cut = TAIL && at.channel(s) < at.C && at.channel(s) + V > at.C;
#pragma unroll
      for (int u = 0; u < V; ++u) f[s][u] = cut ? end[u] : part(v[s], u);
    }
  }
};
template <typename T, int L, int V, int J, bool TAIL>
__device__ __forceinline__ void write_row(T* p, const Place<L, V, J>& at, const float (&f)[Place<L, V, J>::S][V]) {
#pragma unroll
  for (int s = 0; s < Place<L, V, J>::S; ++s) {
    const int c = at.channel(s);
    if (c + V <= at.C) {
      typename Raw<T, V>::type v;
      join(f[s], v);
      Raw<T, V>::store((char*)(p + at.offset(s)), v);
    } else if constexpr (TAIL) {
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (c + u < at.C) {
          typename Raw<T, 1>::type v;
          join(&f[s][u], v);
          Raw<T, 1>::store((char*)(p + c + u), v);
        }
    }
  }
}

// N sets of the thread's weights (`none` where there are none, 0 behind the row's end)
template <bool TAIL, int N, int L, int V, int J>
__device__ __forceinline__ void read_weights(const float* w, float none, const Place<L, V, J>& at, float (&f)[N][V]) {
  constexpr int Q = V < 4 ? V : 4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int u = 0; u < V; ++u) f[i][u] = at.within(i, u, TAIL) ? none : 0.0f;
    if (!w || at.channel(i) >= at.C) continue;
    if (!TAIL || at.channel(i) + V <= at.C) {
#pragma unroll
      for (int u = 0; u < V; u += Q) {
        const auto v = Raw<float, Q>::load((const char*)(w + at.weight(i) + u));
#pragma unroll
        for (int k = 0; k < Q; ++k) f[i][u + k] = part(v, k);
      }
    } else {
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (at.within(i, u, TAIL)) f[i][u] = w[at.weight(i) + u];
    }
  }
}

// f(s, l) for the components above the scalars, of degree l, and end(l) after each degree
template <int L, typename F, typename G>
__device__ __forceinline__ void each_higher(F&& f, G&& end) {
  each<L>([&](auto i) {
    constexpr int l = i + 1;
    each<2 * l + 1>([&](auto m) { f(l * l + m, l); });
    end(l);
  });
}

// The scalars' mean off them (0 behind the row's end)
template <bool TAIL, int L, int V, int J>
__device__ __forceinline__ void centre(const Place<L, V, J>& at, float mean, float (&x)[Place<L, V, J>::S][V]) {
#pragma unroll
  for (int s = 0; s < Place<L, V, J>::S0; ++s)
#pragma unroll
    for (int u = 0; u < V; ++u) x[s][u] = at.within(s, u, TAIL) ? x[s][u] - mean : 0.0f;
}

template <int L, typename T, int V, int J, bool SILU, bool TAIL>
__global__ __launch_bounds__(512) void k_layer_forward(LayerArgs a, int tpr, T* out) {
  typedef Place<L, V, J> P;
  __shared__ float red1[8][L ? 2 : 1], red2[8][1];
  const int slot = threadIdx.x / tpr, slots = blockDim.x / tpr;
  const P at{a.C, (int)threadIdx.x % tpr, tpr};
  float w[P::W][V], b[P::S0][V];
  read_weights<TAIL>(a.w, 1.0f, at, w);
  read_weights<TAIL>(a.b, 0.0f, at, b);
  const float per = 1.0f / (float)a.C;
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n; first += (int64_t)gridDim.x * slots) {
    const int64_t row = min(first + slot, (int64_t)a.n - 1);
    Row<T, L, V, J, TAIL> in;
    in.load((const T*)a.x + row * a.ldx, at);
    float x[P::S][V];
    in.values(at, x);
    float s1[L ? 2 : 1] = {}, s2[1] = {}, t = 0.0f;
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) s1[0] += x[s][u];
    each_higher<L>(
        [&](int s, int) {
#pragma unroll
          for (int u = 0; u < V; ++u) t += x[s][u] * x[s][u];
        },
        [&](int l) { s1[L ? 1 : 0] += t * (1.0f / (2 * l + 1)), t = 0.0f; });
    row_sums(s1, tpr, red1);
    centre<TAIL>(at, s1[0] * per, x);
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) s2[0] += x[s][u] * x[s][u];
    row_sums(s2, tpr, red2);
    const float r0 = 1.0f / sqrtf(s2[0] * per + a.eps);
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const float z = x[s][u] * r0 * w[s][u] + b[s][u];
        x[s][u] = SILU ? z * sigmoid(z) : z;
      }
    if constexpr (L > 0) {
      const float r1 = 1.0f / sqrtf(s1[1] * per * (1.0f / L) + a.eps);
      each_higher<L>(
          [&](int s, int l) {
#pragma unroll
            for (int u = 0; u < V; ++u) x[s][u] *= r1 * w[l][u];
          },
          [](int) {});
    }
    if (first + slot < a.n) write_row<T, L, V, J, TAIL>(out + row * (int64_t)(L ? P::S : 1) * a.C, at, x);
  }
}

template <int L, typename T, int V, int J, bool SILU, bool TAIL>
__global__ __launch_bounds__(512) void k_layer_backward(LayerArgs a, LayerGrad g, int tpr) {
  typedef Place<L, V, J> P;
  constexpr int N1 = L ? 3 : 1, N2 = SILU ? 1 : 3;
  extern __shared__ float sums[];  // [W C + C], with more than one wave's rows a workgroup
  __shared__ float red1[8][N1], red2[8][N2], red3[8][2];
  const int slot = threadIdx.x / tpr, slots = blockDim.x / tpr;
  const P at{a.C, (int)threadIdx.x % tpr, tpr};
  const float per = 1.0f / (float)a.C;
  float w[P::W][V], b[P::S0][V], aw[P::W][V] = {}, ab[P::S0][V] = {};
  read_weights<TAIL>(a.w, 1.0f, at, w);
  if constexpr (SILU) read_weights<TAIL>(a.b, 0.0f, at, b);
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n; first += (int64_t)gridDim.x * slots) {
    const int64_t row = min(first + slot, (int64_t)a.n - 1), packed = row * (L ? P::S : 1) * a.C;
    const bool on = first + slot < a.n;
    Row<T, L, V, J, TAIL> in, gin;
    in.load((const T*)a.x + row * a.ldx, at);
    gin.load((const T*)g.gout + packed, at);
    float x[P::S][V], d[P::S][V];
    in.values(at, x);
    gin.values(at, d);
    float s1[N1] = {}, s2[N2] = {}, s3[2] = {}, t = 0.0f, v[V] = {};
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) s1[0] += x[s][u];
    if constexpr (L > 0) {
      float gx[P::W][V];  // sum over a degree's components of g x
      each_higher<L>(
          [&](int s, int) {
#pragma unroll
            for (int u = 0; u < V; ++u) t += x[s][u] * x[s][u], v[u] += d[s][u] * x[s][u];
          },
          [&](int l) {
            s1[N1 > 1 ? 1 : 0] += t * (1.0f / (2 * l + 1)), t = 0.0f;
#pragma unroll
            for (int u = 0; u < V; ++u) s1[N1 - 1] += w[l][u] * v[u], gx[l][u] = v[u], v[u] = 0.0f;
          });
      row_sums(s1, tpr, red1);
      const float r1 = 1.0f / sqrtf(s1[N1 > 1 ? 1 : 0] * per * (1.0f / (L ? L : 1)) + a.eps);
      // (a power of r1 at a time: its cube leaves float's range from values of 10^13 on)
      const float back = r1 * (r1 * s1[N1 - 1]) * per * (1.0f / (L ? L : 1));
      each_higher<L>(
          [&](int s, int l) {
#pragma unroll
            for (int u = 0; u < V; ++u) d[s][u] = r1 * w[l][u] * d[s][u] - back * (1.0f / (2 * l + 1)) * (r1 * x[s][u]);
          },
          [&](int l) {
#pragma unroll
            for (int u = 0; u < V; ++u) aw[l][u] += on ? r1 * gx[l][u] : 0.0f;
          });
    } else {
      row_sums(s1, tpr, red1);
    }
    centre<TAIL>(at, s1[0] * per, x);
    // without an activation u needs no statistics: its sums go along with the variance's
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        s2[0] += x[s][u] * x[s][u];
        if constexpr (!SILU) {
          s2[N2 > 1 ? 1 : 0] += w[s][u] * d[s][u];
          s2[N2 - 1] += w[s][u] * d[s][u] * x[s][u];
        }
      }
    row_sums(s2, tpr, red2);
    const float r0 = 1.0f / sqrtf(s2[0] * per + a.eps);
    if constexpr (SILU) {
#pragma unroll
      for (int s = 0; s < P::S0; ++s)
#pragma unroll
        for (int u = 0; u < V; ++u) {
          const float z = x[s][u] * r0 * w[s][u] + b[s][u], q = sigmoid(z);
          d[s][u] *= q * (1.0f + z * (1.0f - q));
          s3[0] += w[s][u] * d[s][u];
          s3[1] += w[s][u] * d[s][u] * x[s][u];
        }
      row_sums(s3, tpr, red3);
    } else {
      s3[0] = s2[N2 > 1 ? 1 : 0], s3[1] = s2[N2 - 1];
    }
    const float mu = s3[0] * per, mh = s3[1] * per * r0;  // means of u and of u h
#pragma unroll
    for (int s = 0; s < P::S0; ++s)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const float h = x[s][u] * r0, dz = d[s][u];
        aw[s][u] += on ? dz * h : 0.0f;
        ab[s][u] += on ? dz : 0.0f;
        d[s][u] = r0 * (w[s][u] * dz - mu - h * mh);
      }
    if (on && g.gx) write_row<T, L, V, J, TAIL>((T*)g.gx + packed, at, d);
  }
  if (!g.part) return;
  // the rows of a wave together, then the waves one after the other
  const int width = (P::W > P::S0 ? (L + 1) * a.C : a.C);  // all weights, before the biases
  float* mine_at = g.part + (int64_t)blockIdx.x * (width + a.C);
  if (tpr < 64) {
#pragma unroll
    for (int i = 0; i < P::W; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) aw[i][u] = classes_all(aw[i][u], tpr, [](float p, float q) { return p + q; });
#pragma unroll
    for (int i = 0; i < P::S0; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) ab[i][u] = classes_all(ab[i][u], tpr, [](float p, float q) { return p + q; });
  }
  const int tpg = tpr < 64 ? 64 : tpr, group = threadIdx.x / tpg, groups = blockDim.x / tpg;
  const bool one = threadIdx.x % tpg < tpr;  // one of the threads that hold the same sums
  for (int k = 0; k < groups; ++k) {
    if (groups > 1) __syncthreads();
    if (k != group || !one) continue;
    // V neighbouring sums: with those of the groups before, to the next one or to memory
    auto add = [&](int i, int to, float(&s)[V]) {
      if (at.channel(i) >= a.C) return;
      float* lds = sums + to;
      float* out = k + 1 < groups ? lds : mine_at + to;
      constexpr int Q = V < 4 ? V : 4;
      if (!TAIL || at.channel(i) + V <= a.C) {
#pragma unroll
        for (int u = 0; u < V; u += Q) {
          typename Raw<float, Q>::type v;
          if (k) {
            v = Raw<float, Q>::load((const char*)(lds + u));
#pragma unroll
            for (int x = 0; x < Q; ++x) s[u + x] += part(v, x);
          }
          join(s + u, v);
          Raw<float, Q>::store((char*)(out + u), v);
        }
      } else {
#pragma unroll
        for (int u = 0; u < V; ++u)
          if (at.within(i, u, TAIL)) out[u] = s[u] + (k ? lds[u] : 0.0f);
      }
    };
#pragma unroll
    for (int i = 0; i < P::W; ++i) add(i, at.weight(i), aw[i]);
#pragma unroll
    for (int i = 0; i < P::S0; ++i) add(i, width + at.channel(i), ab[i]);
  }
}

// The weights' gradients from the workgroups' sums: 16 columns a workgroup, 64 sums of each side by side
__global__ __launch_bounds__(1024) void k_layer_weights(const float* __restrict__ part, int parts, int weights, int count,
                                                        float* __restrict__ gw, float* __restrict__ gb) {
  __shared__ double red[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), s = threadIdx.x >> 4;
  double v = 0.0;
  if (c < count) {
#pragma unroll 4
    for (int b = s; b < parts; b += 64) v += part[(int64_t)b * count + c];
  }
  red[s][threadIdx.x & 15] = v;
  __syncthreads();
  if (s || c >= count) return;
#pragma unroll 8
  for (int k = 1; k < 64; ++k) v += red[k][threadIdx.x];
  if (c < weights) {
    if (gw) gw[c] = (float)v;
  } else if (gb) {
    gb[c - weights] = (float)v;
  }
}

// of a launch, which take rows in turn (a million rows of 64 bfloat16 channels: 63.8 us, of 1,024 workgroups 67.8, of
// 16,384 67.6, of a row each 74.5; 20,000 atoms, L = 4, 128 channels: 94.9, 97.7, 91.4, 91.6; 200,000 rows of 512 floats:
// 155, 149, 141, 136)
constexpr int kForwardBlocks = 4096;

struct Shape {
  int V, J, tpr, threads;
  bool tail;
};
// Channels of a thread.  Plain rows: 16 bytes in the forward, and in the backward up to 512 channels (a million rows of 64
// bfloat16 ones with activation 107 us, with four a thread 129; 100,000 of 512 64.5 and 65.1), above four values
// (50,000 rows of 1,024 73.0 us, but with eight 62.3); beyond a wave two pieces and more (50,000 rows of 512 floats: backward
// 57.4 us, in one piece 62.3, in four 70.0; 20,000 of 2,048 bfloat16 61.9, 99.9, 61.2).
// Irrep features: four, two (L = 2, 3) or one, so that the backward holds both rows of components in registers (128
// channels: 40,000 atoms, L = 1: 43.5 us, with two 46.7; 20,000, L = 2: 48.9, with four 49.9, with one 56.5; L = 3: 99.1,
// 100.0, 93.6; L = 4: 150.9, with two 151.1; 10,000, L = 6: 148, with two 388).  Two things this does not reach: one
// bfloat16 a thread, loads of two bytes, is slow in the backward (20,000 atoms, L = 4: 288 us, with two 81), and above 512 channels
// with L >= 4 a thread has two, whose backward spills at L = 5 (32 registers, bfloat16 38; 5,000 atoms of 1,024 channels 589
// us, 10,000 of 512 412) and at L = 6 (120; 1,467 and 565)
Shape shape_of(int L, int C, bool bf16, bool back) {
  Shape s{};
  if (L) {
    s.V = L <= 1 ? 4 : L <= 3 ? 2 : C > 512 ? 2 : 1;
    s.J = 1;
    s.tpr = 1;
    while (s.tpr * s.V < C) s.tpr <<= 1;
  } else {
    s.V = bf16 && (!back || C <= 512) ? 8 : 4;
    const int pieces = (C + s.V - 1) / s.V;
    s.tpr = 1, s.J = 1;
    while (s.tpr < 64 && s.tpr < pieces) s.tpr <<= 1;
    if (s.tpr < pieces) s.J = 2;
    while (s.tpr < 512 && s.tpr * s.J < pieces) s.tpr <<= 1;
    if (s.tpr * s.J < pieces) s.J = (pieces + s.tpr - 1) / s.tpr;  // (three or four)
    s.tail = C % s.V != 0;
  }
  s.threads = s.tpr <= 256 ? 256 : s.tpr;
  return s;
}

}  // namespace

int layer_parts(int L, int C, bool bf16, int n) {
  const Shape s = shape_of(L, C, bf16, true);
  const int slots = s.threads / s.tpr;
  // two workgroups a CU, about what the registers of a row's components leave; of plain rows four (a million rows of
  // 64 bfloat16 channels: 106 us, with two 137), but of long ones one for two rows, whose sums, written and read, are
  // then as many bytes as the rows' (517 rows of 5,001: 21 us with the sums' sum, 25 with one a row, 24 with one for
  // four)
  const int64_t want = ((int64_t)n + slots - 1) / slots;
  int64_t most = L ? 512 : 1024;
  if (L == 0 && want > 128 && want / 2 < most) most = want / 2 < 128 ? 128 : want / 2;
  return (int)(want < most ? want : most);
}

// the kernel for the degree, type, size, activation and end: E2F_LAYER(L, T, V, J, silu, tail)
#define E2F_LAYER_J(T, VV, JJ)                                            \
  case JJ:                                                                \
    if (a.silu) {                                                         \
      if (s.tail) E2F_LAYER(0, T, VV, JJ, true, true);                    \
      else E2F_LAYER(0, T, VV, JJ, true, false);                          \
    } else {                                                              \
      if (s.tail) E2F_LAYER(0, T, VV, JJ, false, true);                   \
      else E2F_LAYER(0, T, VV, JJ, false, false);                         \
    }                                                                     \
    break;
#define E2F_LAYER_L(LL, VV)                                               \
  case LL:                                                                \
    if (bf16) E2F_LAYER(LL, bf16_t, VV, 1, false, false);                 \
    else E2F_LAYER(LL, float, VV, 1, false, false);                       \
    break;
#define E2F_LAYER_M(LL)                                                   \
  case LL:                                                                \
    if (s.V == 2) {                                                       \
      if (bf16) E2F_LAYER(LL, bf16_t, 2, 1, false, false);                \
      else E2F_LAYER(LL, float, 2, 1, false, false);                      \
    } else {                                                              \
      if (bf16) E2F_LAYER(LL, bf16_t, 1, 1, false, false);                \
      else E2F_LAYER(LL, float, 1, 1, false, false);                      \
    }                                                                     \
    break;
#define E2F_LAYER_SWITCH(VB)                                              \
  if (L == 0 && bf16) {                                                   \
    switch (s.J) {                                                        \
      E2F_LAYER_J(bf16_t, 8, 1) E2F_LAYER_J(bf16_t, VB, 2) E2F_LAYER_J(bf16_t, VB, 3) E2F_LAYER_J(bf16_t, VB, 4) \
      default: return hipErrorInvalidValue;                               \
    }                                                                     \
  } else if (L == 0) {                                                    \
    switch (s.J) {                                                        \
      E2F_LAYER_J(float, 4, 1) E2F_LAYER_J(float, 4, 2) E2F_LAYER_J(float, 4, 3) E2F_LAYER_J(float, 4, 4) \
      default: return hipErrorInvalidValue;                               \
    }                                                                     \
  } else {                                                                \
    switch (L) {                                                          \
      E2F_LAYER_L(1, 4) E2F_LAYER_L(2, 2) E2F_LAYER_L(3, 2) E2F_LAYER_M(4) E2F_LAYER_M(5) E2F_LAYER_M(6) \
      default: return hipErrorInvalidValue;                               \
    }                                                                     \
  }

hipError_t launch_layer_forward(int L, bool bf16, const LayerArgs& a, void* out, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const Shape s = shape_of(L, a.C, bf16, false);
  const int64_t blocks = ((int64_t)a.n + s.threads / s.tpr - 1) / (s.threads / s.tpr);
  const unsigned grid = (unsigned)(blocks < kForwardBlocks ? blocks : kForwardBlocks);
#define E2F_LAYER(LL, T, VV, JJ, A, E) k_layer_forward<LL, T, VV, JJ, A, E><<<grid, s.threads, 0, st>>>(a, s.tpr, (T*)out)
  E2F_LAYER_SWITCH(8)
#undef E2F_LAYER
  return hipGetLastError();
}

hipError_t launch_layer_backward(int L, bool bf16, const LayerArgs& a, const LayerGrad& g, hipStream_t st) {
  const int weights = (L + 1) * a.C, count = weights + a.C, parts = a.n ? layer_parts(L, a.C, bf16, a.n) : 0;
  if (a.n) {
    const Shape s = shape_of(L, a.C, bf16, true);
    const size_t lds = g.part && s.threads > s.tpr ? sizeof(float) * count : 0;
#define E2F_LAYER(LL, T, VV, JJ, A, E) k_layer_backward<LL, T, VV, JJ, A, E><<<parts, s.threads, lds, st>>>(a, g, s.tpr)
    E2F_LAYER_SWITCH(4)
#undef E2F_LAYER
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (g.gw || g.gb) k_layer_weights<<<(count + 15) / 16, 1024, 0, st>>>(g.part, parts, weights, count, g.gw, g.gb);
  return hipGetLastError();
}

}  // namespace e2f
