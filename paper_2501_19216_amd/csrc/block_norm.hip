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

#include <type_traits>
#include <utility>

#include "e2f_launch.h"
#include "wave.h"

namespace e2f {
namespace {

// f(k) for k = 0 .. N - 1, each k a constant: what k indexes stays in registers
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}
// f(k, l) for every component k, of degree l, and end(l) after each degree: unrolled with constants where
// registers hold the components, else in loops that read a few at a time
template <int L, bool KEEP, typename F, typename G>
__device__ __forceinline__ void each_component(F&& f, G&& end) {
  each<L + 1>([&](auto l) {
    if constexpr (KEEP) {
      each<2 * l + 1>([&](auto m) { f(std::integral_constant<int, l * l + m>{}, l); });
    } else {
#pragma unroll 4
      for (int k = l * l; k < (l + 1) * (l + 1); ++k) f(k, l);
    }
    end(l);
  });
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

// Sum over the `tpr` threads of a row (a power of two); red: a float for every wave
__device__ __forceinline__ float row_sum(float v, int tpr, float* red) {
  v = lanes_sum(v, tpr);
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

// V channels of every degree of the weights (ones where there are none)
template <int L, int V>
__device__ __forceinline__ void read_weights(const float* w, int C, int c, float (&f)[L + 1][V]) {
#pragma unroll
  for (int l = 0; l <= L; ++l)
#pragma unroll
    for (int u = 0; u < V; ++u) f[l][u] = w ? w[l * C + c + u] : 1.0f;
}

// (first: the workgroup's first row; slot: the thread's after it)
template <int L, typename T, int V>
__device__ __forceinline__ void read_gates(const NormArgs& a, int64_t first, int slot, int c, float (&g)[L + 1][V]) {
#pragma unroll
  for (int l = 0; l <= L; ++l)
#pragma unroll
    for (int u = 0; u < V; ++u) g[l][u] = 1.0f;
  if (a.G == 0) return;
  const char* p = (const char*)a.gate + first * a.G * a.C * (int)sizeof(T);
  const unsigned own = (unsigned)(slot * a.G * a.C + c) * (unsigned)sizeof(T);
  typename Raw<T, V>::type v[L + 1];
#pragma unroll
  for (int l = 0; l <= L; ++l) v[l] = Raw<T, V>::load(p + (a.G > 1 ? l * a.C * (int)sizeof(T) : 0) + own);
#pragma unroll
  for (int l = 0; l <= L; ++l)
#pragma unroll
    for (int u = 0; u < V; ++u) g[l][u] = sigmoid(part(v[l], u));
}

// a gradient that is not given: zeros, with strides of 0
__device__ const float k_zeros[1024] = {};

// A thread's values of one array: in registers, or (KEEP false: rows larger than
// the registers) read again where they are used
template <typename T, int V, int K, bool KEEP>
struct Held {
  // (at L = 6 one bfloat16 is kept as the float that it is, made once all have arrived: converted where it is used
  // it takes two registers, and 20,000 atoms of 64 channels 400 us in the backward instead of 242)
  static constexpr bool WIDE = KEEP && V == 1 && sizeof(T) == 2 && K > 36;
  typedef std::conditional_t<WIDE, float, typename Raw<T, V>::type> R;
  R v[KEEP ? K : 1];
  const char* p;
  int step;
  unsigned own;
  // (slot and channel are clamped by the caller: every address is one of the array's)
  __device__ __forceinline__ void begin(const void* base, int64_t first, int slot, int C, int c) {
    p = (const char*)base + first * K * C * (int)sizeof(T);
    step = C * (int)sizeof(T);
    own = (unsigned)(slot * K * C + c) * (unsigned)sizeof(T);
    if constexpr (KEEP)
      each<K>([&](auto k) {
        if constexpr (WIDE)
          v[k] = __uint_as_float((unsigned)Raw<T, V>::load(p + k * step + own));
        else
          v[k] = Raw<T, V>::load(p + k * step + own);
      });
  }
  // after every load has been issued
  __device__ __forceinline__ void arrived() {
    if constexpr (WIDE)
      each<K>([&](auto k) {
        v[k] = __uint_as_float(__float_as_uint(v[k]) << 16);
        asm volatile("" : "+v"(v[k]));
      });
  }
  template <typename I>
  __device__ __forceinline__ R at(I k) const {
    if constexpr (KEEP)
      return v[k];
    else
      return Raw<T, V>::load(p + k * step + own);
  }
  // the compiler is to take what follows from the held values anew rather than keep results of before
  __device__ __forceinline__ void anew() {
    if constexpr (!KEEP)
      asm volatile("" ::: "memory");
    else if constexpr (sizeof(R) <= 4)
      each<K>([&](auto k) { asm volatile("" : "+v"(v[k])); });
  }
};

// BLOCK: there is a block's output; PRE: the sum is normed
template <int L, typename T, int V, bool KEEP, bool BLOCK, bool PRE>
__global__ __launch_bounds__(KEEP ? 512 : 1024) void k_norm_forward(NormArgs a, int tpr, T* out, T* normed, float* rstd) {
  constexpr int K = (L + 1) * (L + 1);
  __shared__ float red[16];
  const int slot = threadIdx.x / tpr, slots = blockDim.x / tpr;
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * slots;
  if (first >= a.n) return;  // (the last round's)
  const bool mine = threadIdx.x % tpr * V < a.C, on = mine && first + slot < a.n;
  const int c = mine ? threadIdx.x % tpr * V : 0, at = (int)min((int64_t)slot, a.n - 1 - first);
  const unsigned own = (unsigned)(at * K * a.C + c) * (unsigned)sizeof(T);
  Held<T, V, K, KEEP> x, b;
  float f1[L + 1][V], pre[L + 1][V];
  if constexpr (BLOCK) b.begin(a.block, first, at, a.C, c);
  x.begin(a.x, first, at, a.C, c);
  const float mean = 1.0f / (float)((L + 1) * a.C);
  float rb = 1.0f, ro = 1.0f;
  if constexpr (BLOCK) {
    float w[L + 1][V];
    read_gates<L, T, V>(a, first, at, c, f1);
    read_weights<L, V>(a.scale, a.C, c, w);
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) f1[l][u] *= w[l][u];
    if (a.post_w) {
      read_weights<L, V>(a.post_w, a.C, c, w);
      float s = 0.0f, t = 0.0f;
      each_component<L, KEEP>(
          [&](auto k, auto) {
            const auto v = b.at(k);
#pragma unroll
            for (int u = 0; u < V; ++u) t += part(v, u) * part(v, u);
          },
          [&](auto l) { s += t * (1.0f / (2 * l + 1)), t = 0.0f; });
      rb = 1.0f / sqrtf(row_sum(on ? s : 0.0f, tpr, red) * mean + a.eps);
      if constexpr (!KEEP) b.anew();
#pragma unroll
      for (int l = 0; l <= L; ++l)
#pragma unroll
        for (int u = 0; u < V; ++u) f1[l][u] *= w[l][u] * rb;
    }
  }
  if constexpr (PRE) read_weights<L, V>(a.pre_w, a.C, c, pre);
  // the residual sum, where it is needed
  auto sum_at = [&](auto k, auto l, float(&o)[V]) {
    const auto v = x.at(k);
#pragma unroll
    for (int u = 0; u < V; ++u) o[u] = part(v, u);
    if constexpr (BLOCK) {
      const auto f = b.at(k);
#pragma unroll
      for (int u = 0; u < V; ++u) o[u] += f1[l][u] * part(f, u);
    }
  };
  float s = 0.0f, t = 0.0f;
  each_component<L, KEEP>(
      [&](auto k, auto l) {
        float o[V];
        sum_at(k, l, o);
#pragma unroll
        for (int u = 0; u < V; ++u) t += o[u] * o[u];
        if (BLOCK && on) store<T, V>(out, (first * K + k) * a.C, own, o);
      },
      [&](auto l) { s += t * (1.0f / (2 * l + 1)), t = 0.0f; });
  if constexpr (PRE) {
    ro = 1.0f / sqrtf(row_sum(on ? s : 0.0f, tpr, red) * mean + a.eps);
    if constexpr (!KEEP) x.anew(), b.anew();
    if (on)
      each_component<L, KEEP>(
          [&](auto k, auto l) {
            float o[V];
            sum_at(k, l, o);
#pragma unroll
            for (int u = 0; u < V; ++u) o[u] *= ro * pre[l][u];
            store<T, V>(normed, (first * K + k) * a.C, own, o);
          },
          [](auto) {});
  }
  if (rstd && on && c == 0) rstd[2 * (first + slot)] = rb, rstd[2 * (first + slot) + 1] = ro;
}

template <int L, typename T, int V, bool KEEP, bool BLOCK, bool PRE>
__global__ __launch_bounds__(KEEP ? 512 : 1024, KEEP ? 2 : 4) void k_norm_backward(NormArgs a, NormGrad g, int tpr) {
  constexpr int K = (L + 1) * (L + 1);
  // dt is kept for the block's gradient (in place of what it is made of), or made again: of pairs of bfloat16
  // values, which take half its registers, and of those in memory
  constexpr bool HOLD = KEEP && BLOCK && (sizeof(T) == 4 || V == 1);
  extern __shared__ float sums[];  // [2][L + 1][C], with more than one row a workgroup
  __shared__ float red[16];
  const int slot = threadIdx.x / tpr, slots = blockDim.x / tpr;
  const bool mine = threadIdx.x % tpr * V < a.C;
  const int c = mine ? threadIdx.x % tpr * V : 0;
  const float mean = 1.0f / (float)((L + 1) * a.C);
  float pre[L + 1][V], sp1[L + 1][V];  // the weights: of the norm after the sum, and scale times the block's norm's
  if constexpr (PRE) read_weights<L, V>(a.pre_w, a.C, c, pre);
  if constexpr (BLOCK) {
    float w[L + 1][V];
    read_weights<L, V>(a.scale, a.C, c, sp1);
    read_weights<L, V>(a.post_w, a.C, c, w);
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) sp1[l][u] *= w[l][u];
  }
  float sa[L + 1][V] = {}, sp[L + 1][V] = {};  // the weights' sums over the thread's rows
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n; first += (int64_t)gridDim.x * slots) {
    const bool on = mine && first + slot < a.n;
    const int at = (int)min((int64_t)slot, a.n - 1 - first);
    const unsigned own = (unsigned)(at * K * a.C + c) * (unsigned)sizeof(T);
    const unsigned gown = (unsigned)(at * a.G * a.C + c) * (unsigned)sizeof(T);
    Held<T, V, K, KEEP> x, b, dn, dout;
    float gate[L + 1][V], f1[L + 1][V];
    if constexpr (PRE) {
      x.begin(a.x, first, at, a.C, c);
      dn.begin(g.gnormed ? g.gnormed : k_zeros, first, at, g.gnormed ? a.C : 0, c);
    }
    if constexpr (BLOCK) b.begin(a.block, first, at, a.C, c);
    dout.begin(g.gout ? g.gout : k_zeros, first, at, g.gout ? a.C : 0, c);
    const float rb = g.rstd[2 * (first + at)], ro = g.rstd[2 * (first + at) + 1];
    if constexpr (BLOCK) {
      read_gates<L, T, V>(a, first, at, c, gate);
#pragma unroll
      for (int l = 0; l <= L; ++l)
#pragma unroll
        for (int u = 0; u < V; ++u) f1[l][u] = gate[l][u] * sp1[l][u] * rb;
    }
    if constexpr (PRE) x.arrived(), dn.arrived();
    if constexpr (BLOCK) b.arrived();
    dout.arrived();
    auto sum_at = [&](auto k, auto l, float(&o)[V]) {
      const auto v = x.at(k);
#pragma unroll
      for (int u = 0; u < V; ++u) o[u] = part(v, u);
      if constexpr (BLOCK) {
        const auto f = b.at(k);
#pragma unroll
        for (int u = 0; u < V; ++u) o[u] += f1[l][u] * part(f, u);
      }
    };
    float s1 = 0.0f, t[V] = {};
    if constexpr (PRE) {
      each_component<L, KEEP>(
          [&](auto k, auto l) {
            float o[V];
            sum_at(k, l, o);
            const auto d = dn.at(k);
#pragma unroll
            for (int u = 0; u < V; ++u) t[u] += o[u] * part(d, u);
          },
          [&](auto l) {
#pragma unroll
            for (int u = 0; u < V; ++u) {
              s1 += pre[l][u] * t[u];
              sp[l][u] += on ? ro * t[u] : 0.0f;
              t[u] = 0.0f;
            }
          });
      s1 = row_sum(on ? s1 : 0.0f, tpr, red) * ro * ro * ro * mean;
      if constexpr (!HOLD) x.anew(), b.anew(), dn.anew();
    }
    float dt[HOLD ? K : 1][V];
    auto total_at = [&](auto k, auto l, float(&d)[V]) {
      const auto v = dout.at(k);
#pragma unroll
      for (int u = 0; u < V; ++u) d[u] = part(v, u);
      if constexpr (PRE) {
        float o[V];
        sum_at(k, l, o);
        const auto v = dn.at(k);
#pragma unroll
        for (int u = 0; u < V; ++u) d[u] += ro * pre[l][u] * part(v, u) - s1 * (1.0f / (2 * l + 1)) * o[u];
      }
    };
    float s2 = 0.0f, gg[V] = {};
    each_component<L, KEEP>(
        [&](auto k, auto l) {
          float d[V];
          total_at(k, l, d);
          if (on && g.gx) store<T, V>(g.gx, (first * K + k) * a.C, own, d);
          if constexpr (BLOCK) {
            const auto f = b.at(k);
#pragma unroll
            for (int u = 0; u < V; ++u) {
              t[u] += d[u] * part(f, u);
              if constexpr (HOLD) dt[k][u] = d[u];
            }
          }
        },
        [&](auto l) {
          if constexpr (BLOCK) {
            float dg[V];
#pragma unroll
            for (int u = 0; u < V; ++u) {
              s2 += gate[l][u] * sp1[l][u] * t[u];
              sa[l][u] += on ? gate[l][u] * rb * t[u] : 0.0f;
              dg[u] = (1.0f - gate[l][u]) * f1[l][u] * t[u];
              gg[u] += dg[u];
              t[u] = 0.0f;
            }
            if (on && g.ggate && a.G > 1) store<T, V>(g.ggate, (first * a.G + l) * a.C, gown, dg);
          }
        });
    if constexpr (BLOCK) {
      if (on && g.ggate && a.G == 1) store<T, V>(g.ggate, first * a.C, gown, gg);
      if (!g.gblock) continue;
      s2 = a.post_w ? row_sum(on ? s2 : 0.0f, tpr, red) * rb * rb * rb * mean : 0.0f;
      if (!on) continue;  // (the last sum over the row's threads is behind)
      if constexpr (!HOLD) x.anew(), b.anew(), dn.anew(), dout.anew();
      each_component<L, KEEP>(
          [&](auto k, auto l) {
            float d[V];
            const auto f = b.at(k);
            if constexpr (!HOLD) total_at(k, l, d);
#pragma unroll
            for (int u = 0; u < V; ++u) {
              if constexpr (HOLD) d[u] = dt[k][u];
              d[u] = f1[l][u] * d[u] - s2 * (1.0f / (2 * l + 1)) * part(f, u);
            }
            store<T, V>(g.gblock, (first * K + k) * a.C, own, d);
          },
          [](auto) {});
    }
  }
  if (!g.part) return;
  float* mine_at = g.part + (int64_t)blockIdx.x * 2 * (L + 1) * a.C;
  for (int k = 0; k < slots; ++k) {  // the workgroup's rows, one after the other
    if (slots > 1) __syncthreads();
    if (k != slot || !mine) continue;
#pragma unroll
    for (int l = 0; l <= L; ++l)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const int at = l * a.C + c + u, bt = (L + 1) * a.C + at;
        const float va = sa[l][u] + (k ? sums[at] : 0.0f), vp = sp[l][u] + (k ? sums[bt] : 0.0f);
        if (k + 1 < slots)
          sums[at] = va, sums[bt] = vp;
        else
          mine_at[at] = va, mine_at[bt] = vp;
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

// Channels of a thread: as many as keep a row's arrays in its registers (two in the forward, four in the
// backward), in loads of up to 16 bytes.  In registers 20,000 atoms at L = 4, 128 float channels take 190 us forward
// and 336 us backward; read again for each use from the caches, 358 and 904 us.
int channels_per_thread(int L, int C, bool bf16, bool back) {
  if (L == 0 && bf16 && C % 8 == 0 && !back) return 8;
  if (L <= 1) return 4;
  if (L <= 3) return 2;
  return bf16 && !back ? 2 : 1;
}

struct Shape {
  int V, tpr, threads;
  bool keep;
};
Shape shape_of(int L, int C, bool bf16, bool back) {
  Shape s;
  s.V = channels_per_thread(L, C, bf16, back);
  s.tpr = 1;
  while (s.tpr * s.V < C) s.tpr <<= 1;
  s.keep = s.tpr <= 512;
  s.threads = s.tpr <= 256 ? 256 : s.tpr;
  return s;
}

}  // namespace

int norm_parts(int L, int C, bool bf16, int n) {
  const Shape s = shape_of(L, C, bf16, true);
  const int slots = s.threads / s.tpr;
  // two workgroups a CU, about what its registers hold: 336 us where 1,024 workgroups take 350 (20,000 atoms, L = 4,
  // 128 float channels); a row of few bytes a thread wants more of them (60,000 rows of 1,024 bfloat16: 221 and 300 us)
  const int64_t want = ((int64_t)n + slots - 1) / slots, most = L == 0 && bf16 ? 1024 : 512;
  return (int)(want < most ? want : most);
}

// the kernel for the degree, type, size and parts: E2F_NORM(L, T, V, keep, block, pre)
#define E2F_NORM_V(LL, T, VV, KEEP)        \
  if (a.block && a.pre_w)                  \
    E2F_NORM(LL, T, VV, KEEP, true, true); \
  else if (a.block)                        \
    E2F_NORM(LL, T, VV, KEEP, true, false);\
  else                                     \
    E2F_NORM(LL, T, VV, KEEP, false, true);
#define E2F_NORM_L(LL, VF, VB)          \
  case LL:                              \
    if (bf16) {                         \
      E2F_NORM_V(LL, bf16_t, VB, true)  \
    } else {                            \
      E2F_NORM_V(LL, float, VF, true)   \
    }                                   \
    break;
// (a row of more than 512 threads, one channel each, does not fit its workgroup's registers)
#define E2F_NORM_M(LL, VF, VB)          \
  case LL:                              \
    if (bf16 && s.keep) {               \
      E2F_NORM_V(LL, bf16_t, VB, true)  \
    } else if (bf16) {                  \
      E2F_NORM_V(LL, bf16_t, 1, false)  \
    } else if (s.keep) {                \
      E2F_NORM_V(LL, float, VF, true)   \
    } else {                            \
      E2F_NORM_V(LL, float, VF, false)  \
    }                                   \
    break;
#define E2F_NORM_SWITCH(VB)                                                                 \
  switch (L) {                                                                              \
    case 0:                                                                                 \
      if (s.V == 8) {                                                                       \
        E2F_NORM_V(0, bf16_t, 8, true)                                                      \
        break;                                                                              \
      }                                                                                     \
    if (bf16) { E2F_NORM_V(0, bf16_t, 4, true) } else { E2F_NORM_V(0, float, 4, true) } break; \
    E2F_NORM_L(1, 4, 4) E2F_NORM_L(2, 2, 2) E2F_NORM_L(3, 2, 2)                             \
    E2F_NORM_M(4, 1, VB) E2F_NORM_M(5, 1, VB) E2F_NORM_M(6, 1, VB)                          \
    default: return hipErrorInvalidValue;                                                   \
  }

hipError_t launch_norm_forward(int L, bool bf16, const NormArgs& a, void* out, void* normed, float* rstd,
                               hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const Shape s = shape_of(L, a.C, bf16, false);
  const int slots = s.threads / s.tpr;
  const Rounds r = rounds_of(((int64_t)a.n + slots - 1) / slots, s.threads);
  const dim3 grid(r.x, r.rounds);
#define E2F_NORM(LL, T, VV, KEEP, B, P) \
  k_norm_forward<LL, T, VV, KEEP, B, P><<<grid, s.threads, 0, st>>>(a, s.tpr, (T*)out, (T*)normed, rstd)
  E2F_NORM_SWITCH(2)
#undef E2F_NORM
  return hipGetLastError();
}

hipError_t launch_norm_backward(int L, bool bf16, const NormArgs& a, const NormGrad& g, hipStream_t st) {
  const int count = (L + 1) * a.C, parts = a.n ? norm_parts(L, a.C, bf16, a.n) : 0;
  if (a.n) {
    const Shape s = shape_of(L, a.C, bf16, true);
    const size_t lds = s.threads > s.tpr ? sizeof(float) * 2 * count : 0;
#define E2F_NORM(LL, T, VV, KEEP, B, P) k_norm_backward<LL, T, VV, KEEP, B, P><<<parts, s.threads, lds, st>>>(a, g, s.tpr)
    E2F_NORM_SWITCH(1)
#undef E2F_NORM
  }
  if (g.gscale || g.gpost_w || g.gpre_w) k_norm_weights<<<(count + 63) / 64, 1024, 0, st>>>(a, g, parts, count);
  return hipGetLastError();
}

}  // namespace e2f
