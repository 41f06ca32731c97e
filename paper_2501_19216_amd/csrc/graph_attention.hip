// Attention over the neighbours of each atom with capped scores, and its
// gradients.  For the edge e = (i, j) of row i and head h, with d = |r_i - r_j|,
//   x = scale q_ih . k_jh + sum_r w_hr g_r(d),   g_r(d) = exp(-((d - mu_r) / sigma)^2),
//   s = cap tanh(x / cap)   (x itself without a cap),
//   p = exp(s - lse_ih),  lse_ih = log of the row's sum of exp(s),  alpha = env(d) p,
// over the row's edges whose atoms are of one graph; the others have alpha = 0
// and are not read any further, whatever their values.  With a = d loss / d alpha:
//   D_ih = sum of alpha a over the row,   ds = p (a env - D_ih) (1 - tanh^2),
//   dq_ih = scale sum of ds k_jh over the row,   dk_jh = scale sum of ds q_ih over the
//   edges that j sends (the heads that share k summed),   dw_hr = sum of ds g_r,
//   dd = sum_h (a p env'(d) + ds sum_r w_hr g_r'(d)),   dr_i += dd (r_i - r_j) / d,   dr_j -= the same.
#include <hip/hip_runtime.h>

#include "e2f_launch.h"

namespace e2f {
namespace {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void store(float* p, float x) { *p = x; }
__device__ __forceinline__ void store(unsigned short* p, float x) {
  *p = __builtin_bit_cast(unsigned short, (__bf16)x);  // round to nearest even
}

struct Row {
  int64_t e0, e1;
};
// row i's edges, inside [0, E] whatever row_ptr holds
__device__ __forceinline__ Row row_of(const AttnArgs& a, int64_t i) {
  Row r;
  r.e0 = min(max(a.row_ptr[i], (int64_t)0), a.E);
  r.e1 = min(max(a.row_ptr[i + 1], r.e0), a.E);
  return r;
}
__device__ __forceinline__ int atom_of(const AttnArgs& a, int c) { return min(max(c, 0), a.n - 1); }

struct Geometry {
  float x, y, z, d;
};
__device__ __forceinline__ Geometry edge_of(const AttnArgs& a, int i, int j) {
  Geometry g;
  g.x = a.pos[3 * (int64_t)i] - a.pos[3 * (int64_t)j];
  g.y = a.pos[3 * (int64_t)i + 1] - a.pos[3 * (int64_t)j + 1];
  g.z = a.pos[3 * (int64_t)i + 2] - a.pos[3 * (int64_t)j + 2];
  g.d = sqrtf(g.x * g.x + g.y * g.y + g.z * g.z);
  return g;
}
constexpr float kPi = 3.14159265358979f;
__device__ __forceinline__ float envelope(const AttnArgs& a, float d) {
  return d < a.rc ? 0.5f * (cosf(kPi / a.rc * d) + 1.0f) : 0.0f;
}
__device__ __forceinline__ float envelope_slope(const AttnArgs& a, float d) {
  return d < a.rc ? -0.5f * kPi / a.rc * sinf(kPi / a.rc * d) : 0.0f;
}

// the score x of head h
template <typename T>
__device__ __forceinline__ float score(const AttnArgs& a, int i, int j, int h, float d) {
  const int hk = h / (a.H / a.Hk);
  const T* q = (const T*)a.q + i * a.ldq + h * a.dk;
  const T* k = (const T*)a.k + j * a.ldk + hk * a.dk;
  float x = 0.0f;
  for (int t = 0; t < a.dk; ++t) x += to_float(q[t]) * to_float(k[t]);
  x *= a.scale;
  const float sigma = a.rc / (float)(a.R - 1), inv = 1.0f / sigma;
  for (int r = 0; r < a.R; ++r) {
    const float z = (d - r * sigma) * inv;
    x += a.w[h * a.R + r] * expf(-z * z);
  }
  return x;
}

// A wave a row: lane l takes head l % HP and every (64 / HP)-th edge.
template <int HP, typename T>
__global__ __launch_bounds__(256) void k_att_forward(AttnArgs a, float* alpha, float* lse) {
  constexpr int EPI = 64 / HP;
  const int i = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (i >= a.n) return;
  const int h = lane % HP, el = lane / HP;
  const Row r = row_of(a, i);
  float m = -INFINITY, den = 0.0f;
  if (h < a.H)
    for (int64_t e = r.e0 + el; e < r.e1; e += EPI) {
      const int j = atom_of(a, a.col[e]);
      if (a.gid && a.gid[i] != a.gid[j]) continue;
      float x = score<T>(a, i, j, h, edge_of(a, i, j).d);
      if (a.cap > 0.0f) x = a.cap * tanhf(x / a.cap);
      alpha[e * a.H + h] = x;
      if (x > m) {
        den = den * expf(m - x) + 1.0f;
        m = x;
      } else {
        den += expf(x - m);
      }
    }
#pragma unroll
  for (int o = 32; o >= HP; o >>= 1) {
    const float m2 = __shfl_xor(m, o), den2 = __shfl_xor(den, o), mx = fmaxf(m, m2);
    den = (m == mx ? den : den * expf(m - mx)) + (m2 == mx ? den2 : den2 * expf(m2 - mx));
    m = mx;
  }
  if (h >= a.H) return;
  const float l = m + logf(den);
  if (el == 0 && lse) lse[(int64_t)i * a.H + h] = l;
  for (int64_t e = r.e0 + el; e < r.e1; e += EPI) {
    const int j = atom_of(a, a.col[e]);
    if (a.gid && a.gid[i] != a.gid[j])
      alpha[e * a.H + h] = 0.0f;
    else
      alpha[e * a.H + h] = envelope(a, edge_of(a, i, j).d) * expf(alpha[e * a.H + h] - l);
  }
}

// ds of every edge and head (0 where the graphs differ), the edge's position
// gradient and distance, and the receiver's part of the gradients.
template <int HP, typename T>
__global__ __launch_bounds__(256) void k_att_receivers(AttnArgs a, AttnGrad g) {
  constexpr int EPI = 64 / HP;
  const int i = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (i >= a.n) return;
  const int h = lane % HP, el = lane / HP;
  const Row r = row_of(a, i);
  auto same = [&](int j) { return !a.gid || a.gid[i] == a.gid[j]; };
  float D = 0.0f;
  if (h < a.H)
    for (int64_t e = r.e0 + el; e < r.e1; e += EPI)
      if (same(atom_of(a, a.col[e]))) D += g.alpha[e * a.H + h] * g.galpha[e * a.H + h];
#pragma unroll
  for (int o = 32; o >= HP; o >>= 1) D += __shfl_xor(D, o);
  const float l = h < a.H ? g.lse[(int64_t)i * a.H + h] : 0.0f;
  const float sigma = a.rc / (float)(a.R - 1), inv = 1.0f / sigma;
  float gx = 0.0f, gy = 0.0f, gz = 0.0f;
  for (int64_t c = r.e0; c < r.e1; c += EPI) {
    const int64_t e = c + el;
    float dd = 0.0f, ds = 0.0f;
    Geometry v{0.0f, 0.0f, 0.0f, 0.0f};
    if (e < r.e1 && h < a.H) {
      const int j = atom_of(a, a.col[e]);
      if (same(j)) {
        v = edge_of(a, i, j);
        const float x = score<T>(a, i, j, h, v.d), t = a.cap > 0.0f ? tanhf(x / a.cap) : 0.0f;
        const float p = expf((a.cap > 0.0f ? a.cap * t : x) - l), ga = g.galpha[e * a.H + h];
        ds = p * (ga * envelope(a, v.d) - D) * (1.0f - t * t);
        dd = ga * p * envelope_slope(a, v.d);
        for (int q = 0; q < a.R; ++q) {
          const float z = (v.d - q * sigma) * inv;
          dd += ds * a.w[h * a.R + q] * expf(-z * z) * (-2.0f * z * inv);
        }
      }
      g.ds[e * a.H + h] = ds;
    }
#pragma unroll
    for (int o = HP / 2; o > 0; o >>= 1) dd += __shfl_xor(dd, o);
    const float f = v.d > 0.0f ? dd / v.d : 0.0f;
    if (h == 0 && e < r.e1) {
      g.edge[e * 4] = f * v.x, g.edge[e * 4 + 1] = f * v.y, g.edge[e * 4 + 2] = f * v.z, g.edge[e * 4 + 3] = v.d;
      gx += f * v.x, gy += f * v.y, gz += f * v.z;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) gx += __shfl_xor(gx, o), gy += __shfl_xor(gy, o), gz += __shfl_xor(gz, o);
  if (g.gpos && lane < 3) g.gpos[3 * (int64_t)i + lane] = lane == 0 ? gx : lane == 1 ? gy : gz;
  if (!g.gq) return;
  __threadfence_block();  // (the wave's own ds, read by other lanes)
  for (int c = lane; c < a.H * a.dk; c += 64) {
    const int hq = c / a.dk, hk = hq / (a.H / a.Hk), t = c % a.dk;
    float s = 0.0f;
    for (int64_t e = r.e0; e < r.e1; ++e) {
      const int j = atom_of(a, a.col[e]);
      if (same(j)) s += g.ds[e * a.H + hq] * to_float(((const T*)a.k)[j * a.ldk + hk * a.dk + t]);
    }
    store((T*)g.gq + (int64_t)i * a.H * a.dk + c, a.scale * s);
  }
}

// The senders' part: a wave an atom, over the transposed graph.
template <typename T>
__global__ __launch_bounds__(256) void k_att_senders(AttnArgs a, AttnGrad g) {
  const int j = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (j >= a.n) return;
  const int64_t q0 = min(max(g.rowT[j], (int64_t)0), a.E), q1 = min(max(g.rowT[j + 1], q0), a.E);
  auto edge = [&](int64_t q) { return (int64_t)min(max((int64_t)g.perm[q], (int64_t)0), a.E - 1); };
  if (g.gpos) {
    float s[3] = {0.0f, 0.0f, 0.0f};
    for (int64_t q = q0 + lane; q < q1; q += 64)
      for (int x = 0; x < 3; ++x) s[x] += g.edge[edge(q) * 4 + x];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
      for (int x = 0; x < 3; ++x) s[x] += __shfl_xor(s[x], o);
    if (lane < 3) g.gpos[3 * (int64_t)j + lane] -= lane == 0 ? s[0] : lane == 1 ? s[1] : s[2];
  }
  if (!g.gk) return;
  const int share = a.H / a.Hk;
  for (int c = lane; c < a.Hk * a.dk; c += 64) {
    const int hk = c / a.dk, t = c % a.dk;
    float s = 0.0f;
    for (int64_t q = q0; q < q1; ++q) {
      const int i = atom_of(a, g.colT[q]);
      if (a.gid && a.gid[i] != a.gid[j]) continue;
      for (int h = hk * share; h < (hk + 1) * share; ++h)
        s += g.ds[edge(q) * a.H + h] * to_float(((const T*)a.q)[i * a.ldq + h * a.dk + t]);
    }
    store((T*)g.gk + (int64_t)j * a.Hk * a.dk + c, a.scale * s);
  }
}

// dw: part[b][h][r] of every kAttnParts-th stretch of edges, then their sum
__global__ __launch_bounds__(256) void k_att_radial(AttnArgs a, AttnGrad g) {
  const float sigma = a.rc / (float)(a.R - 1), inv = 1.0f / sigma;
  const int64_t per = (a.E + kAttnParts - 1) / kAttnParts, lo = blockIdx.x * per, hi = min(lo + per, a.E);
  for (int c = threadIdx.x; c < a.H * a.R; c += 256) {
    const int h = c / a.R, r = c % a.R;
    float s = 0.0f;
    for (int64_t e = lo; e < hi; ++e) {
      const float z = (g.edge[e * 4 + 3] - r * sigma) * inv;
      s += g.ds[e * a.H + h] * expf(-z * z);
    }
    g.part[(int64_t)blockIdx.x * a.H * a.R + c] = s;
  }
}
__global__ __launch_bounds__(256) void k_att_radial_sum(const float* __restrict__ part, int parts, int count,
                                                        float* __restrict__ gw) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= count) return;
  double s = 0.0;
  for (int b = 0; b < parts; ++b) s += part[(int64_t)b * count + c];
  gw[c] = (float)s;
}

// ---- the transposed graph: edges by sender, ascending
__global__ __launch_bounds__(256) void k_t_zero(int32_t* __restrict__ cnt, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) cnt[i] = 0;
}
// rank[e]: some place of e among its sender's edges (no two alike)
__global__ __launch_bounds__(256) void k_t_count(const int32_t* __restrict__ col, int64_t E, int n,
                                                 int32_t* __restrict__ cnt, int32_t* __restrict__ rank) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e < E) rank[e] = atomicAdd(&cnt[min(max(col[e], 0), n - 1)], 1);
}
// rowT[i] = sum of cnt before i within i's stretch of kScanSpan, and the stretches' sums
constexpr int kScanSpan = 4096;
__global__ __launch_bounds__(1024) void k_t_scan(const int32_t* __restrict__ cnt, int n, int64_t* __restrict__ rowT,
                                                 int64_t* __restrict__ sums) {
  const int64_t at = (int64_t)blockIdx.x * kScanSpan + threadIdx.x * 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v[4];
  for (int u = 0; u < 4; ++u) v[u] = at + u < n ? cnt[at + u] : 0;
  const int own = v[0] + v[1] + v[2] + v[3];
  int inc = own;
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  __shared__ int w[16];
  if (lane == 63) w[wave] = inc;
  __syncthreads();
  int before = inc - own;
  for (int k = 0; k < wave; ++k) before += w[k];
  for (int u = 0; u < 4; ++u) {
    if (at + u < n) rowT[at + u] = before;
    before += v[u];
  }
  if (threadIdx.x == 1023) sums[blockIdx.x] = before;
}
__global__ __launch_bounds__(1024) void k_t_offset(int n, int64_t E, int64_t* __restrict__ rowT,
                                                   const int64_t* __restrict__ sums) {
  __shared__ int64_t w[16];
  int64_t s = 0;
  for (int b = threadIdx.x; b < (int)blockIdx.x; b += 1024) s += sums[b];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
  for (int k = 0; k < 16; ++k) s += w[k];
  for (int u = 0; u < 4; ++u) {
    const int64_t at = (int64_t)blockIdx.x * kScanSpan + threadIdx.x + 1024 * u;
    if (at < n) rowT[at] += s;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) rowT[n] = E;
}
// the edges to their senders' lists, in any order there
__global__ __launch_bounds__(256) void k_t_place(const int32_t* __restrict__ col, int n, int64_t E,
                                                 const int64_t* __restrict__ rowT, const int32_t* __restrict__ rank,
                                                 int32_t* __restrict__ perm) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e < E) perm[rowT[min(max(col[e], 0), n - 1)] + rank[e]] = (int32_t)e;
}
// a wave a sender: its list in ascending order, an edge's place the number of
// smaller ones, and the receivers by bisection of row_ptr
__global__ __launch_bounds__(256) void k_t_sort(const int64_t* __restrict__ row_ptr, int n, int64_t E,
                                                const int64_t* __restrict__ rowT, const int32_t* __restrict__ in,
                                                int32_t* __restrict__ perm, int32_t* __restrict__ colT) {
  const int j = blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (j >= n) return;
  const int64_t q0 = rowT[j], q1 = rowT[j + 1];
  for (int64_t c = q0; c < q1; c += 64) {
    const int e = c + lane < q1 ? in[c + lane] : 0;
    int place = 0;
    for (int64_t b = q0; b < q1; b += 64) {
      const int f = b + lane < q1 ? in[b + lane] : 0x7fffffff;
      for (int u = 0; u < 64; ++u) place += __builtin_amdgcn_readlane(f, u) < e;
    }
    if (c + lane >= q1) continue;
    perm[q0 + place] = e;
    int lo = 0, hi = n - 1;  // the last row that begins at or before e
    while (lo < hi) {
      const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
      if (row_ptr[mid] <= e)
        lo = mid;
      else
        hi = mid - 1;
    }
    colT[q0 + place] = lo;
  }
}

int head_slots(int H) {
  int hp = 1;
  while (hp < H) hp <<= 1;
  return hp;
}

}  // namespace

hipError_t launch_att_forward(const AttnArgs& a, float* alpha, float* lse, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const unsigned grid = (unsigned)((a.n + 3) / 4);
  switch (head_slots(a.H)) {
#define E2F_ATT(P)                                                           \
  case P:                                                                    \
    if (a.bf16)                                                              \
      k_att_forward<P, unsigned short><<<grid, 256, 0, s>>>(a, alpha, lse);  \
    else                                                                     \
      k_att_forward<P, float><<<grid, 256, 0, s>>>(a, alpha, lse);           \
    break;
    E2F_ATT(1) E2F_ATT(2) E2F_ATT(4) E2F_ATT(8) E2F_ATT(16) E2F_ATT(32) E2F_ATT(64)
#undef E2F_ATT
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_att_backward(const AttnArgs& a, const AttnGrad& g, hipStream_t s) {
  if (a.n == 0) {  // (the sum over no edges)
    if (g.gw) k_att_radial_sum<<<(a.H * a.R + 255) / 256, 256, 0, s>>>(g.part, 0, a.H * a.R, g.gw);
    return hipGetLastError();
  }
  const unsigned grid = (unsigned)((a.n + 3) / 4);
  switch (head_slots(a.H)) {
#define E2F_ATT(P)                                                    \
  case P:                                                             \
    if (a.bf16)                                                       \
      k_att_receivers<P, unsigned short><<<grid, 256, 0, s>>>(a, g);  \
    else                                                              \
      k_att_receivers<P, float><<<grid, 256, 0, s>>>(a, g);           \
    break;
    E2F_ATT(1) E2F_ATT(2) E2F_ATT(4) E2F_ATT(8) E2F_ATT(16) E2F_ATT(32) E2F_ATT(64)
#undef E2F_ATT
    default: return hipErrorInvalidValue;
  }
  if (g.gk || g.gpos) {
    if (a.bf16)
      k_att_senders<unsigned short><<<grid, 256, 0, s>>>(a, g);
    else
      k_att_senders<float><<<grid, 256, 0, s>>>(a, g);
  }
  if (g.gw) {
    k_att_radial<<<kAttnParts, 256, 0, s>>>(a, g);
    k_att_radial_sum<<<(a.H * a.R + 255) / 256, 256, 0, s>>>(g.part, kAttnParts, a.H * a.R, g.gw);
  }
  return hipGetLastError();
}

int transpose_scan_blocks(int n) { return (n + kScanSpan - 1) / kScanSpan; }

hipError_t launch_transpose(const int64_t* row_ptr, const int32_t* col, int n, int64_t E, int32_t* cnt, int64_t* sums,
                            int32_t* rank, int32_t* list, int64_t* rowT, int32_t* colT, int32_t* perm,
                            hipStream_t s) {
  if (n == 0) {
    k_t_offset<<<1, 1024, 0, s>>>(0, 0, rowT, nullptr);
    return hipGetLastError();
  }
  const unsigned blocks = (unsigned)transpose_scan_blocks(n), eb = (unsigned)((E + 255) / 256);
  k_t_zero<<<(n + 255) / 256, 256, 0, s>>>(cnt, n);
  if (E > 0) k_t_count<<<eb, 256, 0, s>>>(col, E, n, cnt, rank);
  k_t_scan<<<blocks, 1024, 0, s>>>(cnt, n, rowT, sums);
  k_t_offset<<<blocks, 1024, 0, s>>>(n, E, rowT, sums);
  if (E > 0) {
    k_t_place<<<eb, 256, 0, s>>>(col, n, E, rowT, rank, list);
    k_t_sort<<<(n + 3) / 4, 256, 0, s>>>(row_ptr, n, E, rowT, list, perm, colT);
  }
  return hipGetLastError();
}

}  // namespace e2f
