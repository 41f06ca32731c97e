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
//
// A wave takes a receiver's row (four waves, where rows are long) in batches of
// up to 64 edges of its graph; edges between graphs only get their zeros.
//   - Geometry: a lane an edge.
//   - The products: lanes over an edge's features of k, 16 bytes each, so that a
//     gather reads whole lines; the features of a head are summed over its lanes.
//     This gather, H dk values an edge out of the caches, is what bounds both
//     directions (1.5 million edges of 8 heads of 16 floats are 780 MB; with 32 radial
//     functions and 20,000 atoms forward 102 us, backward 261 for the receivers and 125
//     for the senders, the transposed graph 88).
//   - The radial part: float matrix products of 16 edges, 16 heads and 4 functions
//     (v_mfma_f32_16x16x4_f32), each lane evaluating the functions it passes in.
//   - The softmax's running maximum and sum stay with the lanes that hold a head in
//     the product's output; the scores of up to 128 edges stay in the LDS until the
//     row's sum is known, those of longer rows in alpha.
// Heads go in groups of up to 16 (one matrix tile), a group a workgroup.  Backward:
// the receivers' kernel makes the scores again (the cap's slope and the edges beyond the
// cutoff need them) and takes p from alpha, which holds no rounding of lse (forward and backward
// 553 us; p from the scores and lse 543), ds from both, dq and each edge's position gradient,
// and sums dw as matrix products too; the senders' kernel
// gathers ds and q over the transposed graph.  No atomics in either: the same
// bits every time.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "e2f_launch.h"
#include "wave.h"

namespace e2f {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef f4 f4_any __attribute__((aligned(4)));
typedef u4 u4_any __attribute__((aligned(2)));

// 16 bytes of features: the address needs no more than an element's alignment
struct F32 {
  typedef float type;
  typedef f4 raw;
  static constexpr int VEC = 4;
  static __device__ __forceinline__ float at(const raw& r, int u) { return r[u]; }
  // the first `count` of them (1 .. VEC), zeros behind
  static __device__ __forceinline__ raw load(const float* p, int count) {
    if (count >= VEC) return *(const f4_any*)p;
    raw r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < VEC - 1; ++u)
      if (u < count) r[u] = p[u];
    return r;
  }
  static __device__ __forceinline__ void store(float* p, const float (&f)[VEC], int count) {
    if (count >= VEC) {
      *(f4_any*)p = (f4){f[0], f[1], f[2], f[3]};
      return;
    }
#pragma unroll
    for (int u = 0; u < VEC - 1; ++u)
      if (u < count) p[u] = f[u];
  }
};
struct BF16 {
  typedef unsigned short type;
  typedef u4 raw;
  static constexpr int VEC = 8;
  static __device__ __forceinline__ float at(const raw& r, int u) {
    return __uint_as_float(u & 1 ? r[u >> 1] & 0xffff0000u : r[u >> 1] << 16);
  }
  static __device__ __forceinline__ raw load(const unsigned short* p, int count) {
    if (count >= VEC) return *(const u4_any*)p;
    raw r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int u = 0; u < VEC - 1; ++u)
      if (u < count) r[u >> 1] |= (unsigned)p[u] << (u & 1 ? 16 : 0);
    return r;
  }
  static __device__ __forceinline__ void store(unsigned short* p, const float (&f)[VEC], int count) {
    unsigned short b[VEC];
#pragma unroll
    for (int u = 0; u < VEC; ++u) b[u] = __builtin_bit_cast(unsigned short, (__bf16)f[u]);  // to nearest even
    if (count >= VEC) {
      u4 r;
#pragma unroll
      for (int u = 0; u < 4; ++u) r[u] = b[2 * u] | (unsigned)b[2 * u + 1] << 16;
      *(u4_any*)p = r;
      return;
    }
#pragma unroll
    for (int u = 0; u < VEC - 1; ++u)
      if (u < count) p[u] = b[u];
  }
};

// Orders the LDS and memory accesses of a wave's lanes among each other
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr float kPi = 3.14159265358979f, kLog2e = 1.44269504088896f;
// exp(-z^2) for the radial functions: the rounding of the argument is z^2 steps of the value, and z^2 exp(-z^2) stays
// below 0.37: less than half a step of 1, which the largest function of a distance is near to
__device__ __forceinline__ float exp_radial(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// exp(x) for x <= 0 to three half steps of its value however far x is: 2^t (1 + r) with t log 2 + r = x and t near
// x log2(e): rounding x log2(e) alone leaves |x| half steps, 64 of them at 80, and saves no time (1.5 million edges,
// forward: 102 us with that and a reciprocal in the tangent, 97 with this and the quotient below).  (Below 2^-126: 0.)
__device__ __forceinline__ float exp_near(float x) {
  constexpr float ln2 = 0.693147182464599609f, low = -1.90465430e-9f;  // log 2 = ln2 + low
  const float t = x * kLog2e, r = fmaf(-t, low, fmaf(-t, ln2, x));
  const float e = __builtin_amdgcn_exp2f(t);
  return e > 0.0f ? fmaf(e, r, e) : e;  // (r of an infinite x is NaN)
}
// n / d for d in 1 .. 4: the reciprocal's quotient and one correction by its remainder
__device__ __forceinline__ float quotient(float n, float d) {
  const float r = __builtin_amdgcn_rcpf(d), q = n * r;
  return fmaf(fmaf(-d, q, n), r, q);
}
// tanh to a few half steps of its own value: the odd series to x^11 below 0.35 (its next term is below 2^-25 of x
// there), (1 - e^-2x) / (1 + e^-2x) from it on.  turn: 1 - tanh^2, there as 4 e^-2x / (1 + e^-2x)^2, which keeps its
// digits where the tangent comes near 1
__device__ __forceinline__ float tanh_near(float x, float* turn = nullptr) {
  const float a = fabsf(x), t = a * a;
  const float p = a + a * t * (-1.0f / 3 + t * (2.0f / 15 + t * (-17.0f / 315 + t * (62.0f / 2835 + t * (-1382.0f / 155925)))));
  const float e = exp_near(-2.0f * a);
  if (turn) *turn = a < 0.35f ? 1.0f - p * p : quotient(4.0f * e, (1.0f + e) * (1.0f + e));
  return copysignf(a < 0.35f ? p : quotient(1.0f - e, 1.0f + e), x);
}

// Distance and envelope have every fused product written out: forward and backward get the same bits, so that the
// backward finds the softmax's p in alpha = env p.
__device__ __forceinline__ float length(float x, float y, float z) { return sqrtf(fmaf(z, z, fmaf(y, y, x * x))); }
// (cos(pi x) + 1) / 2 = c^2 and its slope -pi s c for x = d / cutoff below 1, with c, s the cosine and sine of pi x / 2
// by their series (the next terms are below 2^-26 there); 0 from 1 on
__device__ __forceinline__ float envelope(float rc, float d, float* slope = nullptr) {
  const float h = 0.5f * kPi * (d / rc), t = h * h;
  const float c = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.0f / 479001600, -1.0f / 3628800), 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  if (slope) {
    const float s = h * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.0f / 6227020800, -1.0f / 39916800), 1.0f / 362880), -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
    *slope = d < rc ? -kPi / rc * s * c : 0.0f;
  }
  return d < rc ? c * c : 0.0f;
}

__device__ __forceinline__ int atom_of(const AttnArgs& a, int c) { return min(max(c, 0), a.n - 1); }

// Workgroups of one XCD (every eighth) take neighbouring rows, which share senders where atoms are in order
__device__ __forceinline__ int64_t row_block() {
  const int64_t nb = gridDim.x, per = nb / 8, rest = nb % 8, x = blockIdx.x % 8, k = blockIdx.x / 8;
  return x * per + min(x, rest) + k + blockIdx.z * nb;
}

// A workgroup's heads: `share` q heads from h0 on for each of the k heads from k0 on
struct Group {
  int h0, heads, k0, kheads, share;
};
__device__ __forceinline__ Group group_of(const AttnArgs& a, const AttnShape& s, int y) {
  Group g;
  if (s.share < s.sharing) {  // part of the heads of one head of k
    const int parts = (s.sharing + s.share - 1) / s.share, at = y % parts * s.share;
    g.k0 = y / parts, g.kheads = 1, g.share = min(s.share, s.sharing - at), g.h0 = g.k0 * s.sharing + at;
  } else {
    g.k0 = y * s.kheads, g.kheads = min(s.kheads, a.Hk - g.k0), g.share = s.share, g.h0 = g.k0 * s.share;
  }
  g.heads = g.kheads * g.share;
  return g;
}

// floats of an entry's scores in the LDS: 9 (up to 8 heads, in the forward, where the LDS bounds the waves of a CU: five
// instead of four a SIMD, 97 us instead of 122 for 1.5 million edges of 8 heads) or 17 (up to 16); odd: other banks
constexpr int kLd = 17;

// Lanes over a group's heads (hp, their number's next power of two) and over 64 / hp entries: a head belongs to a lane
struct Lanes {
  int head, entry, per;
  bool on;
};
__device__ __forceinline__ Lanes lanes_of(const AttnShape& s, const Group& g) {
  const int lane = threadIdx.x & 63;
  Lanes l;
  l.head = lane & (s.hp - 1), l.entry = lane >> s.hp_log, l.per = 64 >> s.hp_log;
  l.on = l.head < g.heads;
  return l;
}

// How a wave goes through a row: stretches of 64 edges, of which it takes those of the receiver's graph
struct Walk {
  int64_t e0;              // first edge of the row; the others count from it
  unsigned len, at, step;  // edges of the row, next stretch, from one of the wave's to the next
  int queued, gid;         // edges found and not yet taken
};

// The next batch, a lane an edge: its place e in the row and its sender j, -1 behind the last.  Returns their number.
// stage: 256 ints.  skip(first edge, count, lanes whose edges are between graphs) sees each stretch once.
template <typename S>
__device__ __forceinline__ int next_batch(const AttnArgs& a, Walk& w, int* stage, unsigned& e, int& j, S&& skip) {
  const int lane = threadIdx.x & 63;
  const int32_t* col = a.col + w.e0;
  j = -1, e = 0;
  if (!a.gid) {
    if (w.at >= w.len) return 0;
    const int count = (int)min(w.len - w.at, 64u);
    if (lane < count) e = w.at + lane, j = atom_of(a, col[e]);
    w.at += w.step;
    return count;
  }
  while (w.queued < 64 && w.at < w.len) {
    const unsigned mine = w.at + lane;
    int s = -1;
    bool same = false;
    if (mine < w.len) {
      s = atom_of(a, col[mine]);
      same = a.gid[s] == w.gid;
    }
    const uint64_t found = __ballot(same);
    const int count = (int)min(w.len - w.at, 64u);
    skip(w.at, count, ~found & (count == 64 ? ~0ull : (1ull << count) - 1));
    if (same) {
      const int q = w.queued + __builtin_popcountll(found & ((1ull << lane) - 1));
      stage[q] = s;
      stage[128 + q] = (int)mine;
    }
    w.queued += __builtin_popcountll(found);
    w.at += w.step;
  }
  wave_sync();
  const int count = min(w.queued, 64);
  if (lane < count) j = stage[lane], e = stage[128 + lane];
  if (w.queued > 64) {
    const bool more = lane < w.queued - 64;
    const int s = more ? stage[64 + lane] : 0, f = more ? stage[192 + lane] : 0;
    wave_sync();
    if (more) stage[lane] = s, stage[128 + lane] = f;
  }
  w.queued -= count;
  wave_sync();
  return count;
}

// row i's edges, inside [0, E] whatever row_ptr holds; the wave `part` of `wpr` takes every wpr-th stretch
__device__ __forceinline__ Walk walk_of(const AttnArgs& a, int64_t i, int part, int wpr) {
  const int64_t E = a.E, e0 = min(max(a.row_ptr[i], (int64_t)0), E), e1 = min(max(a.row_ptr[i + 1], e0), E);
  return Walk{e0, (unsigned)(e1 - e0), 64u * part, 64u * wpr, 0, a.gid ? a.gid[i] : 0};
}

// Features of a block of BE entries, LPE lanes an entry, up to eight loads of a lane at a time (`part` of PARTS)
template <int LPE, typename F>
struct Features {
  static constexpr int EPI = 64 / LPE, BE = EPI > 16 ? EPI : 16, ALL = BE / EPI, IT = ALL > 8 ? 8 : ALL, PARTS = ALL / IT;
  typename F::raw k[IT];
  static __device__ __forceinline__ int entry(int part, int i) {
    return (part * IT + i) * EPI + (threadIdx.x & 63) / LPE;
  }
  // of the atoms jj[entry], `count` of the lane's from base on; WHOLE: all or none of them
  template <bool WHOLE>
  __device__ __forceinline__ void read(const typename F::type* base, int64_t ld, const int* jj, int part, int count) {
    if constexpr (WHOLE) {
#pragma unroll
      for (int i = 0; i < IT; ++i) k[i] = F::load(base + jj[entry(part, i)] * ld, F::VEC);
      if (count <= 0) {
#pragma unroll
        for (int i = 0; i < IT; ++i) k[i] = typename F::raw{};
      }
    } else {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        k[i] = typename F::raw{};
        if (count > 0) k[i] = F::load(base + jj[entry(part, i)] * ld, count);
      }
    }
  }
  // s[entry * LD] = the sum over a head's lph lanes of q . k, by its first lane
  template <int LD>
  __device__ __forceinline__ void dots(const float (&q)[F::VEC], int lph, bool first, float* s, int part) {
    float x[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      x[i] = 0.0f;
#pragma unroll
      for (int u = 0; u < F::VEC; ++u) x[i] += q[u] * F::at(k[i], u);
    }
    auto add = [&](auto other) {
#pragma unroll
      for (int i = 0; i < IT; ++i) x[i] = other(x[i]);
    };
    if (LPE > 1 && lph > 1) add([](float v) { return v + lane_other<1>(v); });
    if (LPE > 2 && lph > 2) add([](float v) { return v + lane_other<2>(v); });
    if (LPE > 4 && lph > 4) add([](float v) { return v + lane_other<4>(v); });
    if (LPE > 8 && lph > 8) add([](float v) { return v + lane_other<8>(v); });
    if (LPE > 16 && lph > 16) add([](float v) { float p, q; lane_halves<16>(v, p, q); return p + q; });
    if (LPE > 32 && lph > 32) add([](float v) { float p, q; lane_halves<32>(v, p, q); return p + q; });
    if (first) {
#pragma unroll
      for (int i = 0; i < IT; ++i) s[entry(part, i) * LD] = x[i];
    }
  }
  // acc += sum over the lane's entries of w[entry * kLd] k
  __device__ __forceinline__ void add_weighted(const float* w, int part, float (&acc)[F::VEC]) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const float c = w[entry(part, i) * kLd];
#pragma unroll
      for (int u = 0; u < F::VEC; ++u) acc[u] += c * F::at(k[i], u);
    }
  }
};

// A lane's place among the features of a group: k head kl, its features from t VEC on, `count` of them there
struct Place {
  int kl, t, count;
};
template <int LPE, typename F>
__device__ __forceinline__ Place place_of(const AttnArgs& a, const AttnShape& sh, const Group& g, int unit) {
  Place p;
  const int at = unit * 64 + (threadIdx.x & 63) % LPE;
  p.t = at & (sh.lph - 1), p.kl = at >> sh.lph_log;
  p.count = p.kl < g.kheads ? a.dk - p.t * F::VEC : 0;
  return p;
}
template <typename F>
__device__ __forceinline__ const typename F::type* k_at(const AttnArgs& a, const Group& g, const Place& p) {
  // (lanes without features read the group's first ones, where they read)
  return (const typename F::type*)a.k + (p.count > 0 ? (g.k0 + p.kl) * a.dk + p.t * F::VEC : g.k0 * a.dk);
}
template <typename F>
__device__ __forceinline__ void read_q(const AttnArgs& a, int64_t i, int h, const Place& p, float (&q)[F::VEC]) {
  typename F::raw r = {};
  if (p.count > 0) r = F::load((const typename F::type*)a.q + i * a.ldq + (int64_t)h * a.dk + p.t * F::VEC, p.count);
#pragma unroll
  for (int u = 0; u < F::VEC; ++u) q[u] = a.scale * F::at(r, u);
}

// The products scale q . k of a block's entries with every head of the group: s[entry * LD + head].  ONE: a lane has
// one head (q1 its features), all or none of a load's features; else `units` times 64 lanes for k, and `share` heads each.  k is left in f where f
// holds all of it.
template <int LPE, bool ONE, int LD, typename F>
__device__ __forceinline__ void products(const AttnArgs& a, const AttnShape& sh, const Group& g, int64_t i,
                                         const float (&q1)[F::VEC], Features<LPE, F>& f, const int* jj, float* s) {
  for (int u = 0; u < (ONE ? 1 : sh.units); ++u) {
    const Place p = place_of<LPE, F>(a, sh, g, u);
    const auto* k = k_at<F>(a, g, p);
#pragma unroll
    for (int part = 0; part < f.PARTS; ++part) {
      f.template read<ONE>(k, a.ldk, jj, part, p.count);
      if constexpr (ONE) {
        f.template dots<LD>(q1, sh.lph, p.t == 0 && p.kl < g.kheads, s + p.kl, part);
      } else {
        for (int m = 0; m < g.share; ++m) {
          float q[F::VEC];
          read_q<F>(a, i, g.h0 + p.kl * g.share + m, p, q);
          f.template dots<LD>(q, sh.lph, p.t == 0 && p.kl < g.kheads, s + p.kl * g.share + m, part);
        }
      }
    }
  }
}

// s[entry * LD + head] of 16 entries gets its radial part (is set to it without products): the functions' values times
// the weights wr of the lane's head (the functions 4 r + quad; zeros of a head that is not there, and what a distance
// that is not finite makes of them is not kept)
template <int LD>
__device__ __forceinline__ void add_radial(const AttnArgs& a, int heads, const float* dist,
                                           const float (&wr)[8], float inv, float* s) {
  const int lane = threadIdx.x & 63, hc = lane & 15, quad = lane >> 4;
  f4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  const float z0 = dist[hc] * inv - (float)quad;
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if (4 * r < a.R) {
      const float z = z0 - 4.0f * r;
      x = __builtin_amdgcn_mfma_f32_16x16x4f32(exp_radial(-z * z), wr[r], x, 0, 0, 0);
    }
  if (hc < heads) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float* to = s + (quad * 4 + u) * LD + hc;
      *to = a.dk ? *to + x[u] : x[u];
    }
  }
}

constexpr int kKept = 128;  // edges of a row whose scores stay in the LDS

template <int LPE, bool ONE, int LD, typename F>
__global__ __launch_bounds__(256, ONE && LD == 9 ? 5 : 4) void k_att_forward(AttnArgs a, AttnShape sh, float* alpha, float* lse) {
  extern __shared__ float sm[];
  __shared__ float join[4][2][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (a scalar)
  const Group g = group_of(a, sh, blockIdx.y);
  const Lanes ln = lanes_of(sh, g);
  float* s = sm + wave * sh.lds;
  float* env = s + kKept * LD;
  int* edge = (int*)(env + kKept);
  float* dist = (float*)(edge + kKept);
  int* jj = (int*)(dist + 64);
  int* stage = jj + 64;
  const float inv = (float)(a.R - 1) / a.rc, icap = a.cap > 0.0f ? 1.0f / a.cap : 0.0f;
  float wr[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int f = 4 * r + (lane >> 4), h = lane & 15;
    wr[r] = h < g.heads && f < a.R ? a.w[(g.h0 + h) * a.R + f] : 0.0f;
  }
  const int64_t first = row_block() * sh.rows;
  for (int rr = 0; rr < sh.rows; rr += sh.wpr == 1 ? 4 : 1) {
    const int64_t i = first + rr + (sh.wpr == 1 ? wave : 0);
    if (i >= a.n) break;  // (with four waves a row the same for the workgroup)
    const int part = sh.wpr == 1 ? 0 : wave;
    Walk w = walk_of(a, i, part, sh.wpr);
    float* out = alpha + w.e0 * a.H + g.h0;  // the row's weights of the group's heads
    float q1[F::VEC] = {};
    if (ONE && a.dk) {
      const Place p = place_of<LPE, F>(a, sh, g, 0);
      read_q<F>(a, i, g.h0 + p.kl, p, q1);
    }
    const float px = a.pos[3 * i], py = a.pos[3 * i + 1], pz = a.pos[3 * i + 2];
    float m = -INFINITY, den = 0.0f;
    int kept = 0;        // edges whose scores are in the LDS
    bool spill = false;  // the scores of the row are in alpha
    auto to_alpha = [&](int count, const float* from) {
      if (ln.on)
        for (int n = ln.entry; n < count; n += ln.per)
          out[(uint64_t)(unsigned)edge[n] * a.H + ln.head] = from[n * LD + ln.head];
    };
    for (;;) {
      unsigned e;
      int j;
      const int count = next_batch(a, w, stage, e, j, [&](unsigned first, int many, uint64_t mask) {
        if (!mask || !ln.on) return;
        for (int n = ln.entry; n < many; n += ln.per)
          if (mask >> n & 1) out[(uint64_t)(first + n) * a.H + ln.head] = 0.0f;
      });
      if (count == 0) break;
      if (kept == kKept) {  // (every batch but the last has 64)
        to_alpha(kept, s);
        kept = 0, spill = true;
        wave_sync();
      }
      float* sb = s + kept * LD;
      const bool there = j >= 0;
      float dx = 0.0f, dy = 0.0f, dz = 0.0f;
      if (there) dx = px - a.pos[3 * (int64_t)j], dy = py - a.pos[3 * (int64_t)j + 1], dz = pz - a.pos[3 * (int64_t)j + 2];
      const int j0 = __builtin_amdgcn_readfirstlane(j);  // (by every lane: lane 0 has the batch's first edge)
      jj[lane] = there ? j : j0;                          // the first sender once more behind the last
      wave_sync();
      if (a.dk) {
        Features<LPE, F> f;
        for (int b = 0; b < count; b += f.BE) products<LPE, ONE, LD, F>(a, sh, g, i, q1, f, jj + b, sb + b * LD);
      }
      const float d = length(dx, dy, dz);
      dist[lane] = d;
      env[kept + lane] = envelope(a.rc, d);
      edge[kept + lane] = (int)e;
      wave_sync();
      if (a.R)
        for (int b = 0; b < count; b += 16) add_radial<LD>(a, g.heads, dist + b, wr, inv, sb + b * LD);
      wave_sync();
      // the scores, and the running maximum and sum, four entries at a time
      if (ln.on)
        for (int n0 = ln.entry; n0 < count; n0 += 4 * ln.per) {
          float x[4], mx = m;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int n = n0 + u * ln.per;
            x[u] = -INFINITY;
            if (n < count) {
              x[u] = a.dk || a.R ? sb[n * LD + ln.head] : 0.0f;
              if (a.cap > 0.0f) x[u] = a.cap * tanh_near(x[u] * icap);
              sb[n * LD + ln.head] = x[u];
            }
            mx = fmaxf(mx, x[u]);
          }
          if (mx > m) den *= exp_near(m - mx), m = mx;
          const float from = m == -INFINITY ? 0.0f : m;  // (scores of -infinity alone: terms of 0)
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (n0 + u * ln.per < count) den += exp_near(x[u] - from);
        }
      wave_sync();
      if (spill)
        to_alpha(count, s);
      else
        kept += count;
      wave_sync();
    }
    // the row's sum, over the lanes and waves of a head
    float top = classes_all(m, sh.hp, [](float p, float q) { return fmaxf(p, q); });
    den = classes_all(m == top ? den : den * exp_near(m - top), sh.hp, [](float p, float q) { return p + q; });
    if (sh.wpr > 1) {
      __syncthreads();  // (the row before has been read)
      if (lane < sh.hp) join[wave][0][lane] = top, join[wave][1][lane] = den;
      __syncthreads();
      for (int k = 0; k < 4; ++k) top = fmaxf(top, join[k][0][ln.head]);
      den = 0.0f;
      for (int k = 0; k < 4; ++k) {
        const float mk = join[k][0][ln.head], dk = join[k][1][ln.head];
        den += mk == top ? dk : dk * exp_near(mk - top);
      }
    }
    // (the weights from the maximum and the sum: exp(s - lse) would carry lse's rounding, half a step of the scores,
    // into all of a row's)
    const float rden = 1.0f / den;
    if (lse && ln.on && ln.entry == 0 && part == 0) lse[i * a.H + g.h0 + ln.head] = top + logf(den);
    if (!spill) {
      if (ln.on)
        for (int n = ln.entry; n < kept; n += ln.per)
          out[(uint64_t)(unsigned)edge[n] * a.H + ln.head] = env[n] * (exp_near(s[n * LD + ln.head] - top) * rden);
      wave_sync();  // (before the next row's scores)
      continue;
    }
    for (unsigned c = 64u * part; c < w.len; c += w.step) {
      const int count = (int)min(w.len - c, 64u);
      float v = -1.0f;  // (an edge between graphs: its zeros are written)
      if (lane < count) {
        const int j = atom_of(a, a.col[w.e0 + c + lane]);
        if (!a.gid || a.gid[j] == w.gid) {
          const float dx = px - a.pos[3 * (int64_t)j], dy = py - a.pos[3 * (int64_t)j + 1], dz = pz - a.pos[3 * (int64_t)j + 2];
          v = envelope(a.rc, length(dx, dy, dz));
        }
      }
      env[lane] = v;
      wave_sync();
      if (ln.on)
        for (int n = ln.entry; n < count; n += ln.per) {
          if (env[n] < 0.0f) continue;
          float* to = out + (uint64_t)(c + n) * a.H + ln.head;
          *to = env[n] * (exp_near(*to - top) * rden);
        }
      wave_sync();
    }
  }
}

// ds of every edge and head, the edge's position gradient, and the receivers' gradients.  A workgroup takes sh.rows
// rows and sums dw over them.
template <int LPE, bool ONE, typename F>
__global__ __launch_bounds__(256, 3) void k_att_receivers(AttnArgs a, AttnShape sh, AttnGrad gr) {
  extern __shared__ float sm[];
  __shared__ float join[4][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (a scalar)
  const Group g = group_of(a, sh, blockIdx.y);
  const Lanes ln = lanes_of(sh, g);
  float* s = sm + wave * sh.lds;  // [64][kLd] scores, then ds; heads that are not there stay 0
  for (int x = lane; x < 64 * kLd; x += 64) s[x] = 0.0f;
  float* dist = s + 64 * kLd;
  float* env = dist + 64;
  float* renv = env + 64;  // 1 / env
  float* slope = renv + 64;
  int* edge = (int*)(slope + 64);
  int* jj = edge + 64;
  float* force = (float*)(jj + 64);  // [64] d loss / d distance
  int* stage = (int*)(force + 64);
  const float inv = (float)(a.R - 1) / a.rc, icap = a.cap > 0.0f ? 1.0f / a.cap : 0.0f;
  const int hc = lane & 15, quad = lane >> 4;
  float wr[8], wt[2][4];  // weights: of the lane's head, functions 4 r + quad; of the functions 16 r + hc, heads 4 k + quad
#pragma unroll
  for (int r = 0; r < 8; ++r) wr[r] = hc < g.heads && 4 * r + quad < a.R ? a.w[(g.h0 + hc) * a.R + 4 * r + quad] : 0.0f;
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      wt[r][k] = 4 * k + quad < g.heads && 16 * r + hc < a.R ? a.w[(g.h0 + 4 * k + quad) * a.R + 16 * r + hc] : 0.0f;
  f4 dw[2] = {};  // of the lane's head, functions 16 r + 4 quad + 0 .. 3
  const int part = sh.wpr == 1 ? 0 : wave;
  const int64_t first = row_block() * sh.rows;
  for (int rr = 0; rr < sh.rows; rr += sh.wpr == 1 ? 4 : 1) {
    const int64_t i = first + rr + (sh.wpr == 1 ? wave : 0);
    const bool row = i < a.n;
    Walk w = {};
    if (row) w = walk_of(a, i, part, sh.wpr);
    const float* gal = gr.galpha + w.e0 * a.H + g.h0;  // the row's gradients of the group's heads, and its weights
    const float* al = gr.alpha + w.e0 * a.H + g.h0;
    float D = 0.0f;
    {
      const unsigned stride = ln.per * sh.wpr;
      for (unsigned e = ln.entry + part * ln.per; ln.on && e < w.len; e += 4 * stride) {
        float x[4], y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint64_t at = (uint64_t)min(e + u * stride, w.len - 1) * a.H + ln.head;
          x[u] = al[at], y[u] = gal[at];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (e + u * stride < w.len && (!a.gid || a.gid[atom_of(a, a.col[w.e0 + e + u * stride])] == w.gid))
            D += x[u] * y[u];
      }
      D = classes_all(D, sh.hp, [](float p, float q) { return p + q; });
      if (sh.wpr > 1) {
        __syncthreads();  // (the row before has been read)
        if (lane < sh.hp) join[wave][lane] = D;
        __syncthreads();
        D = join[0][ln.head] + join[1][ln.head] + join[2][ln.head] + join[3][ln.head];
      }
    }
    if (!row) continue;  // (with four waves a row, for the workgroup)
    float* rec = gr.edge + w.e0 * gr.stride;
    const float l = ln.on ? gr.lse[i * a.H + g.h0 + ln.head] : 0.0f;
    float q1[F::VEC] = {}, dq[F::VEC] = {};
    if (ONE && a.dk) {
      const Place p = place_of<LPE, F>(a, sh, g, 0);
      read_q<F>(a, i, g.h0 + p.kl, p, q1);
    }
    const float px = a.pos[3 * i], py = a.pos[3 * i + 1], pz = a.pos[3 * i + 2];
    if (!ONE && gr.gq) {
      for (int x = lane; x < sh.dq; x += 64) stage[256 + x] = 0;
      wave_sync();
    }
    for (;;) {
      unsigned e;
      int j;
      const int count = next_batch(a, w, stage, e, j, [](unsigned, int, uint64_t) {});
      if (count == 0) break;
      float dx = 0.0f, dy = 0.0f, dz = 0.0f;
      if (j >= 0) dx = px - a.pos[3 * (int64_t)j], dy = py - a.pos[3 * (int64_t)j + 1], dz = pz - a.pos[3 * (int64_t)j + 2];
      const int j0 = __builtin_amdgcn_readfirstlane(j);  // (by every lane: lane 0 has the batch's first edge)
      jj[lane] = j >= 0 ? j : j0;                         // the first sender once more behind the last
      edge[lane] = (int)e;
      const float d = length(dx, dy, dz);
      float sl;
      env[lane] = envelope(a.rc, d, &sl);
      // (a radial function's slope holds z exp(-z^2), which is to be 0 where a distance's square is past float32)
      dist[lane] = d > 1e18f ? 1e18f : d, slope[lane] = sl, renv[lane] = 1.0f / env[lane];
      wave_sync();
      Features<LPE, F> f;
      for (int b0 = 0; b0 < count; b0 += f.BE) {
        float* sb = s + b0 * kLd;
        const int many = min(count - b0, f.BE);  // of the block's entries
        float ga[4], al4[4];
        auto read_row = [&](int c) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int n = c + ln.entry + u * ln.per;
            ga[u] = al4[u] = 0.0f;
            if (ln.on && n < many) {
              const uint64_t at = (uint64_t)(unsigned)edge[b0 + n] * a.H + ln.head;
              ga[u] = gal[at], al4[u] = al[at];
            }
          }
        };
        read_row(0);
        if (a.dk) products<LPE, ONE, kLd, F>(a, sh, g, i, q1, f, jj + b0, sb);
        wave_sync();
        if (a.R)
          for (int b = 0; b < many; b += 16) add_radial<kLd>(a, g.heads, dist + b0 + b, wr, inv, sb + b * kLd);
        wave_sync();
        // ds, and the envelope's part of the distances' gradients, four entries at a time
        for (int c = 0; c < f.BE; c += 4 * ln.per) {
          if (c > 0) read_row(c);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int n = c + ln.entry + u * ln.per;
            if (c + u * ln.per >= f.BE) break;  // (the same for the wave)
            float x = 0.0f, turn = 1.0f, ds = 0.0f, dd = 0.0f;
            if (ln.on && n < f.BE) {
              if (n < many) {
                if (a.dk || a.R) x = sb[n * kLd + ln.head];
                if (a.cap > 0.0f) {
                  x = a.cap * tanh_near(x * icap, &turn);
                }
                // p from the weight; where the envelope leaves nothing of it, at the cutoff and beyond, or it is next to
                // nothing, from the score, with lse's rounding in it
                const float p = al4[u] >= 0x1p-100f ? al4[u] * renv[b0 + n] : exp_near(x - l);
                ds = p * (ga[u] * env[b0 + n] - D) * turn;
                dd = ga[u] * p * slope[b0 + n];
                if (gr.gk) rec[(uint64_t)(unsigned)edge[b0 + n] * gr.stride + g.h0 + ln.head] = ds;
              }
              sb[n * kLd + ln.head] = ds;
            }
            if (gr.gpos) {
              dd = lanes_sum(dd, sh.hp);
              if (ln.head == 0 && n < f.BE) force[b0 + n] = dd;
            }
          }
        }
        wave_sync();
        if (a.R && (gr.gw || gr.gpos))
          for (int b = 0; b < many; b += 16) {
            float dd[4] = {};
#pragma unroll
            for (int r = 0; r < 2; ++r)
              if (16 * r < a.R) {
                // us[edge][function] = the sum of ds w over the heads
                f4 us = {0.0f, 0.0f, 0.0f, 0.0f};
                if (gr.gpos) {
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (4 * k < g.heads)
                      us = __builtin_amdgcn_mfma_f32_16x16x4f32(
                          sb[(b + hc) * kLd + 4 * k + quad], wt[r][k], us, 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const int n = b + quad * 4 + u;
                  const float z = dist[b0 + n] * inv - (float)(16 * r + hc), gz = exp_radial(-z * z);
                  dd[u] += us[u] * gz * z;
                  dw[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(gz, sb[n * kLd + hc], dw[r], 0, 0, 0);
                }
              }
            if (gr.gpos) {
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const float v = lanes_sum(dd[u], 16);
                if (hc == u) force[b0 + b + quad * 4 + u] -= 2.0f * inv * v;
              }
            }
          }
        if (a.dk && gr.gq) {
          // k is read again where f does not hold all of it, a head's sum at a time, added to those of the wave in
          // the LDS where a lane has several
          [[maybe_unused]] float* acc = (float*)(stage + 256);
          for (int u = 0; u < (ONE ? 1 : sh.units); ++u) {
            const Place p = place_of<LPE, F>(a, sh, g, u);
            const auto* k = k_at<F>(a, g, p);
#pragma unroll
            for (int y = 0; y < f.PARTS; ++y) {
              if (!ONE || f.PARTS > 1) f.template read<ONE>(k, a.ldk, jj + b0, y, p.count);
              if (p.kl >= g.kheads) continue;
              if constexpr (ONE) {
                f.add_weighted(sb + p.kl, y, dq);
              } else {
                for (int mm = 0; mm < g.share; ++mm) {
                  float v[F::VEC] = {};
                  f.add_weighted(sb + p.kl * g.share + mm, y, v);
                  float* to = acc + ((lane / LPE * g.heads + p.kl * g.share + mm) * sh.lph + p.t) * F::VEC;
#pragma unroll
                  for (int x = 0; x < F::VEC; ++x) to[x] += v[x];
                }
              }
            }
          }
        }
        wave_sync();
      }
      if (gr.gpos && lane < count) {
        const float v = d > 0.0f ? force[lane] / d : 0.0f;
        *(f4*)(rec + (uint64_t)e * gr.stride + gr.force + 4 * blockIdx.y) = (f4){v * dx, v * dy, v * dz, 0.0f};
      }
      wave_sync();
    }
    if (!a.dk || !gr.gq) continue;
    // dq: over the lanes of a feature, and the waves of the row
    typename F::type* gq = (typename F::type*)gr.gq + (i * a.H + g.h0) * a.dk;
    if constexpr (ONE) {
      const Place p = place_of<LPE, F>(a, sh, g, 0);
#pragma unroll
      for (int u = 0; u < F::VEC; ++u) dq[u] = a.scale * classes_all(dq[u], LPE, [](float x, float y) { return x + y; });
      if (sh.wpr > 1) {
        float* mine = dist;  // (what follows s: 704 floats that the row has done with)
        __syncthreads();
        if (lane < LPE) {
#pragma unroll
          for (int u = 0; u < F::VEC; ++u) mine[lane * F::VEC + u] = dq[u];
        }
        __syncthreads();
        if (wave == 0 && lane < LPE) {
#pragma unroll
          for (int u = 0; u < F::VEC; ++u)
            dq[u] = dist[lane * F::VEC + u] + dist[sh.lds + lane * F::VEC + u] + dist[2 * sh.lds + lane * F::VEC + u] +
                    dist[3 * sh.lds + lane * F::VEC + u];
        }
        __syncthreads();
      }
      if (part == 0 && lane < LPE && p.count > 0) F::store(gq + p.kl * a.dk + p.t * F::VEC, dq, p.count);
    } else {
      if (sh.wpr > 1)
        __syncthreads();
      else
        wave_sync();
      const int off = (int)((float*)(stage + 256) - s), width = sh.lph * F::VEC;
      for (int x = (sh.wpr > 1 ? threadIdx.x : lane); x < g.heads * a.dk; x += 64 * sh.wpr) {
        const int h = x / a.dk, t = x - h * a.dk;
        float v = 0.0f;
        for (int k = 0; k < sh.wpr; ++k)
          for (int q = 0; q < 64 / LPE; ++q)
            v += sm[(sh.wpr > 1 ? k : wave) * sh.lds + off + (q * g.heads + h) * width + t];
        float one[F::VEC];
        one[0] = a.scale * v;
        F::store(gq + x, one, 1);
      }
      if (sh.wpr > 1)
        __syncthreads();
      else
        wave_sync();
    }
  }
  if (!gr.gw) return;
  // dw of the workgroup's waves
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int u = 0; u < 4; ++u) sm[(wave * 32 + 16 * r + quad * 4 + u) * 16 + hc] = dw[r][u];
  __syncthreads();
  for (int x = threadIdx.x; x < g.heads * a.R; x += 256) {
    const int h = x / a.R, r = x - h * a.R;
    float v = 0.0f;
    for (int k = 0; k < 4; ++k) v += sm[(k * 32 + r) * 16 + h];
    gr.part[((int64_t)blockIdx.x * a.H + g.h0 + h) * a.R + r] = v;
  }
}

// dw: the sum of the workgroups', 16 columns a workgroup
__global__ __launch_bounds__(1024) void k_att_radial_sum(const float* __restrict__ part, int parts, int count,
                                                         float* __restrict__ gw) {
  __shared__ double red[64][16];
  const int x = threadIdx.x & 15, c = blockIdx.x * 16 + x, w = threadIdx.x >> 4;
  double v = 0.0;
  if (c < count) {
#pragma unroll 8
    for (int b = w; b < parts; b += 64) v += part[(int64_t)b * count + c];
  }
  red[w][x] = v;
  __syncthreads();
  if (w || c >= count) return;
  for (int k = 1; k < 64; ++k) v += red[k][x];
  gw[c] = (float)v;
}

// dk over the edges that an atom sends, and its whole position gradient: those of the edges it receives minus those
// of the edges it sends.  Lanes over a group's features of q, LPE an edge; the heads that share k one after another.
template <int LPE, typename F>
__global__ __launch_bounds__(256) void k_att_senders(AttnArgs a, AttnShape sh, AttnGrad gr) {
  constexpr int EPI = 64 / LPE;
  __shared__ int stage[4][2][64];
  __shared__ float join[4][64 * F::VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (a scalar)
  const int64_t j = sh.wpr == 1 ? row_block() * 4 + wave : row_block();
  const bool row = j < a.n;
  const int part = sh.wpr == 1 ? 0 : wave;
  const int64_t q0 = row ? min(max(gr.rowT[j], (int64_t)0), a.E) : 0;
  const int64_t q1 = row ? min(max(gr.rowT[j + 1], q0), a.E) : 0;
  const int gid = a.gid && row ? a.gid[j] : 0;
  const int k0 = blockIdx.y * sh.kheads, kheads = min(sh.kheads, a.Hk - k0), share = sh.sharing;
  const int at = lane % LPE, t = at & (sh.lph - 1), kl = at >> sh.lph_log;
  const int count = kl < kheads ? a.dk - t * F::VEC : 0;
  int *ii = stage[wave][0], *ee = stage[wave][1];
  float acc[F::VEC] = {}, gx = 0.0f, gy = 0.0f, gz = 0.0f;
  const bool forces = gr.gpos && blockIdx.y == 0;
  if (forces && row) {
    const int64_t e0 = min(max(a.row_ptr[j], (int64_t)0), a.E), e1 = min(max(a.row_ptr[j + 1], e0), a.E);
    for (int64_t e = e0 + lane + 64 * part; e < e1; e += 64 * sh.wpr)
      if (!a.gid || a.gid[atom_of(a, a.col[e])] == gid)
        for (int y = 0; y < gr.groups; ++y) {
          const f4 v = *(const f4*)(gr.edge + e * gr.stride + gr.force + 4 * y);
          gx += v[0], gy += v[1], gz += v[2];
        }
  }
  for (int64_t c = q0 + 64 * part; c < q1; c += 64 * sh.wpr) {
    const int many = (int)min(q1 - c, (int64_t)64);
    int i = -1, e = 0;
    if (lane < many) {
      i = atom_of(a, gr.colT[c + lane]);
      e = (int)min(max((int64_t)gr.perm[c + lane], (int64_t)0), a.E - 1);
      if (a.gid && a.gid[i] != gid) i = -1;
    }
    if (gr.gk) {
      ii[lane] = i, ee[lane] = e;
      wave_sync();
      for (int b = 0; b < many; b += 8 * EPI) {
        for (int m = 0; m < share; ++m) {
          typename F::raw r[8];
          float ds[8];
          const int h = (k0 + kl) * share + m;
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int n = b + u * EPI + lane / LPE;
            const int s = n < 64 ? ii[n] : -1;
            r[u] = typename F::raw{};
            ds[u] = 0.0f;
            if (s >= 0 && count > 0) {
              r[u] = F::load((const typename F::type*)a.q + s * a.ldq + (int64_t)h * a.dk + t * F::VEC, count);
              ds[u] = gr.edge[(int64_t)ee[n] * gr.stride + h];
            }
          }
#pragma unroll
          for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int x = 0; x < F::VEC; ++x) acc[x] += ds[u] * F::at(r[u], x);
        }
      }
      wave_sync();
    }
    if (forces && i >= 0)
      for (int y = 0; y < gr.groups; ++y) {
        const f4 v = *(const f4*)(gr.edge + (int64_t)e * gr.stride + gr.force + 4 * y);
        gx -= v[0], gy -= v[1], gz -= v[2];
      }
  }
  if (gr.gk) {
#pragma unroll
    for (int u = 0; u < F::VEC; ++u) acc[u] = a.scale * classes_all(acc[u], LPE, [](float x, float y) { return x + y; });
  }
  gx = lanes_sum(gx), gy = lanes_sum(gy), gz = lanes_sum(gz);
  if (sh.wpr > 1) {
    if (lane < LPE) {
#pragma unroll
      for (int u = 0; u < F::VEC; ++u) join[wave][lane * F::VEC + u] = acc[u];
    }
    float* p = (float*)stage[wave][0];
    __syncthreads();
    if (lane == 0) p[0] = gx, p[1] = gy, p[2] = gz;
    __syncthreads();
    if (wave == 0 && lane < LPE) {
#pragma unroll
      for (int u = 0; u < F::VEC; ++u)
        acc[u] = join[0][lane * F::VEC + u] + join[1][lane * F::VEC + u] + join[2][lane * F::VEC + u] +
                 join[3][lane * F::VEC + u];
    }
    gx = gy = gz = 0.0f;
    for (int k = 0; k < 4; ++k) {
      const float* pk = (const float*)stage[k][0];
      gx += pk[0], gy += pk[1], gz += pk[2];
    }
  }
  if (!row || part) return;
  if (gr.gk && lane < LPE && count > 0)
    F::store((typename F::type*)gr.gk + (j * a.Hk + k0 + kl) * a.dk + t * F::VEC, acc, count);
  if (forces && lane < 3) gr.gpos[3 * j + lane] = lane == 0 ? gx : lane == 1 ? gy : gz;
}

// ---- the transposed graph: edges by sender, ascending.  Where the rows ascend, an edge (j, i) of row j finds by a
// search of j in row i whether its reverse (i, j) is there, which is one of the edges that j sends: j's list is the
// reverses of its own row, in order, and those of its edges that have none are counted, placed behind and sorted in.
// So a graph with every edge both ways (a radius graph) takes no atomics and no sort.  Graphs whose rows do not
// ascend count and sort every edge.
struct Transposed {
  const int64_t* row_ptr;
  const int32_t* col;
  int n;
  int64_t E;
  int32_t *cnt, *found, *extra, *pos, *list, *from;  // cnt[n]: not 0 if a row does not ascend
  int64_t *sums, *rowT;
  int32_t *colT, *perm;
};
__global__ __launch_bounds__(256) void k_t_zero(Transposed t) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i <= t.n) t.cnt[i] = 0;
  if (i < t.n) t.extra[i] = 0;
}
// the place of x among the n ascending values at p, or -1 (one read a step and none after it: scattered reads are what
// this costs; three at once in half the steps took 68 us where single ones take 52, 1.5 million edges)
__device__ __forceinline__ int place_among(const int32_t* p, int n, int x) {
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1, v = p[lo + half];
    if (v == x) return lo + half;
    if (v < x)
      lo += half + 1, n -= half + 1;
    else
      n = half;
  }
  return -1;
}
struct RowEnds {
  int64_t e0, e1;
};
// pos[e] of the edge e = (j, i): the edge (i, j), or -1 - (some place among the edges that i sends without a
// reverse); found[j]: the reverses of row j, extra[i]: the edges that i sends without one
__global__ __launch_bounds__(256) void k_t_reverse(Transposed t) {
  const int lane = threadIdx.x & 63;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = (int)row;
  if (row >= t.n || __hip_atomic_load(t.cnt + t.n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) return;
  const int64_t e0 = t.row_ptr[j], e1 = t.row_ptr[j + 1];
  bool good = e0 >= 0 && e0 <= e1 && e1 <= t.E && (j > 0 || e0 == 0) && (j + 1 < t.n || e1 == t.E);
  int found = 0, last = -1;  // last sender of the stretch before
  if (good)
    for (int64_t c = e0; c < e1; c += 64) {
      const int64_t e = c + lane;
      const int i = e < e1 ? t.col[e] : t.n;
      const int up = __shfl_up(i, 1), before = lane ? up : last;
      last = __shfl(i, 63);
      bool has = false;
      if (e < e1) {
        const bool fine = i < t.n && before < i;
        RowEnds r = {0, 0};
        if (fine) __builtin_memcpy(&r, t.row_ptr + i, sizeof(r));
        const int64_t lo = min(max(r.e0, (int64_t)0), t.E), hi = min(max(r.e1, lo), t.E);
        const int at = place_among(t.col + lo, (int)(hi - lo), j);
        has = at >= 0;
        if (has)
          t.pos[e] = (int32_t)lo + at;
        else if (fine)
          t.pos[e] = -1 - atomicAdd(t.extra + i, 1);
        good = good && fine;
      }
      found += __builtin_popcountll(__ballot(has));
    }
  if (lane == 0) t.found[j] = found;
  if (__any(!good) && lane == 0) __hip_atomic_store(t.cnt + t.n, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// (rows that do not ascend) pos[e]: some place of e among its sender's edges (no two alike)
__global__ __launch_bounds__(256) void k_t_count(Transposed t) {
  if (!t.cnt[t.n]) return;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < t.E; e += (int64_t)gridDim.x * 256)
    t.pos[e] = atomicAdd(&t.cnt[min(max(t.col[e], 0), t.n - 1)], 1);
}
// rowT[i] = sum of the counts before i within i's stretch of kScanSpan, and the stretches' sums
constexpr int kScanSpan = 4096;
__global__ __launch_bounds__(1024) void k_t_scan(Transposed t) {
  const bool any = t.cnt[t.n];
  const int64_t at = (int64_t)blockIdx.x * kScanSpan + threadIdx.x * 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v[4];
  for (int u = 0; u < 4; ++u) v[u] = at + u >= t.n ? 0 : any ? t.cnt[at + u] : t.found[at + u] + t.extra[at + u];
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
    if (at + u < t.n) t.rowT[at + u] = before;
    before += v[u];
  }
  if (threadIdx.x == 1023) t.sums[blockIdx.x] = before;
  if (gridDim.x == 1 && threadIdx.x == 0) t.rowT[t.n] = t.E;
}
__global__ __launch_bounds__(1024) void k_t_offset(Transposed t) {
  __shared__ int64_t w[16];
  int64_t s = 0;
  for (int b = threadIdx.x; b < (int)blockIdx.x; b += 1024) s += t.sums[b];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
  for (int k = 0; k < 16; ++k) s += w[k];
  for (int u = 0; u < 4; ++u) {
    const int64_t at = (int64_t)blockIdx.x * kScanSpan + threadIdx.x + 1024 * u;
    if (at < t.n) t.rowT[at] += s;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) t.rowT[t.n] = t.E;
}
// a wave a row: the reverses of its edges are its atom's list; what has none, and the lists that wait for such an
// edge, go to `list`
__global__ __launch_bounds__(256) void k_t_place(Transposed t) {
  if (t.cnt[t.n]) {
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < t.E; e += (int64_t)gridDim.x * 256)
      t.list[t.rowT[min(max(t.col[e], 0), t.n - 1)] + t.pos[e]] = (int32_t)e;
    return;
  }
  const int lane = threadIdx.x & 63;
  for (int64_t j = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); j < t.n; j += (int64_t)gridDim.x * 4) {
    const int64_t e1 = t.row_ptr[j + 1];
    int64_t to = t.rowT[j];
    const bool whole = t.extra[j] == 0;
    for (int64_t c = t.row_ptr[j]; c < e1; c += 64) {
      const int64_t e = c + lane;
      const int i = e < e1 ? t.col[e] : 0, p = e < e1 ? t.pos[e] : -1;
      const uint64_t m = __ballot(p >= 0);
      const int64_t at = to + __builtin_popcountll(m & ((1ull << lane) - 1));
      if (p >= 0 && whole)
        t.perm[at] = p, t.colT[at] = i;
      else if (e < e1) {
        const int64_t slot = p >= 0 ? at : t.rowT[i] + t.found[i] - 1 - p;
        t.list[slot] = p >= 0 ? p : (int32_t)e;
        t.from[slot] = p >= 0 ? i : (int32_t)j;
      }
      to += __builtin_popcountll(m);
    }
  }
}
// the last row of lo .. hi that begins at or before e: e's receiver
__device__ __forceinline__ int row_of(const Transposed& t, int lo, int hi, int e) {
  while (lo < hi) {
    const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
    if (t.row_ptr[mid] <= e)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
// A long list, by a workgroup: eight bits of the edges' numbers at a time, between list and pos (read for the last
// time before this kernel).  Stable: an edge comes behind those of its digit in earlier chunks (base), earlier waves
// (cnt) and earlier lanes (rank).
struct Digits {
  int base[256], cnt[4][256], sum[4];
};
__device__ void sort_long(const Transposed& t, int64_t q0, int n, Digits& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t *in = t.list + q0, *out = t.pos + q0;
  for (int shift = 0; shift < 31 && ((t.E - 1) >> shift) > 0; shift += 8) {
    s.base[tid] = 0;
    __syncthreads();
    for (int x = tid; x < n; x += 256) atomicAdd(&s.base[(in[x] >> shift) & 255], 1);
    __syncthreads();
    const int own = s.base[tid];
    int inc = own;
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 63) s.sum[wave] = inc;
    __syncthreads();
    for (int k = 0; k < wave; ++k) inc += s.sum[k];
    s.base[tid] = inc - own;
    for (int c = 0; c < n; c += 256) {
      const bool on = c + tid < n;
      const int e = on ? in[c + tid] : 0, d = (e >> shift) & 255;
      uint64_t same = __ballot(on);
      for (int b = 0; b < 8; ++b) {
        const uint64_t set = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? set : ~set;
      }
      const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
      for (int k = 0; k < 4; ++k) s.cnt[k][tid] = 0;
      __syncthreads();
      if (on && rank == 0) s.cnt[wave][d] = __builtin_popcountll(same);
      __syncthreads();
      if (on) {
        int at = s.base[d] + rank;
        for (int k = 0; k < wave; ++k) at += s.cnt[k][d];
        out[at] = e;
      }
      __syncthreads();
      s.base[tid] += s.cnt[0][tid] + s.cnt[1][tid] + s.cnt[2][tid] + s.cnt[3][tid];
    }
    __syncthreads();
    int32_t* swap = in;
    in = out, out = swap;
  }
  for (int x = tid; x < n; x += 256) {
    const int e = in[x];
    t.perm[q0 + x] = e;
    t.colT[q0 + x] = row_of(t, 0, t.n - 1, e);
  }
  __syncthreads();
}
// The lists that are not in order yet.  Up to kWaveList edges, a wave a list: an edge's place is the number of smaller
// ones, whose time grows with the list's square; longer ones by digits (the whole transposition for one sender of 128
// edges by its square, and of 129 by digits, 35 us; of 512: 158 and 35 us; of 20,000 by digits 0.54 ms, of 10^6 39 ms)
constexpr int kWaveList = 128;
__global__ __launch_bounds__(256) void k_t_sort(Transposed t) {
  __shared__ Digits digits;
  const bool any = t.cnt[t.n];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t j0 = (int64_t)blockIdx.x * 4; j0 < t.n; j0 += (int64_t)gridDim.x * 4) {
    const int64_t j = j0 + wave;
    const bool mine = j < t.n && (any || t.extra[j] != 0);
    const int64_t q0 = mine ? t.rowT[j] : 0, q1 = mine ? t.rowT[j + 1] : 0;
    const bool longer = q1 - q0 > kWaveList;
    if (!longer)
      for (int64_t c = q0; c < q1; c += 64) {
        const int e = c + lane < q1 ? t.list[c + lane] : 0;
        int place = 0;
        for (int64_t b = q0; b < q1; b += 64) {
          const int f = b + lane < q1 ? t.list[b + lane] : 0x7fffffff;
          const int many = (int)min(q1 - b, (int64_t)64);
          for (int u = 0; u < many; ++u) place += __builtin_amdgcn_readlane(f, u) < e;
        }
        if (c + lane >= q1) continue;
        t.perm[q0 + place] = e;
        t.colT[q0 + place] = any ? row_of(t, 0, t.n - 1, e) : t.from[c + lane];
      }
    if (!__syncthreads_or(longer)) continue;
    for (int64_t k = j0; k < min(j0 + 4, (int64_t)t.n); ++k) {
      const int64_t at = t.rowT[k], many = t.rowT[k + 1] - at;
      if ((any || t.extra[k] != 0) && many > kWaveList) sort_long(t, at, (int)many, digits);
    }
  }
}

// Lanes of a head, heads of a workgroup and what follows from them
AttnShape shape_of(const AttnArgs& a, bool senders) {
  const int vec = a.bf16 ? BF16::VEC : F32::VEC, share = a.H / a.Hk;
  AttnShape s{};
  s.lph = 1;
  while (s.lph * vec < a.dk) s.lph <<= 1, ++s.lph_log;
  s.sharing = share;
  // heads that share k: the receivers' sums for dq, 64 lanes of them for each, stay within 8 KB of LDS a wave
  s.share = senders ? share : std::min(share, 2048 / (64 * vec));
  s.kheads = senders ? a.Hk : std::min(a.Hk, s.share < share ? 1 : 16 / share);
  const int most = senders ? 64 : 2048 / (vec * s.share) < 256 ? 2048 / (vec * s.share) : 256;
  int p = 1;
  while (p < s.kheads) p <<= 1;
  while (p > 1 && p * s.lph > most) p >>= 1;
  s.kheads = std::min(s.kheads, p);
  s.units = (p * s.lph + 63) / 64;
  s.lpe = std::min(p * s.lph, 64);
  s.groups = s.share < share ? a.Hk * ((share + s.share - 1) / s.share) : (a.Hk + s.kheads - 1) / s.kheads;
  s.heads = s.kheads * s.share;
  s.hp = 1;
  while (s.hp < s.heads) s.hp <<= 1, ++s.hp_log;
  s.one = s.units == 1 && (share == 1 || a.dk == 0) && a.dk % vec == 0;
  // four waves a row where they find four batches on average (8 heads of 16, forward and backward: 2,000 rows of 128
  // edges 21 and 74 us by one wave, 27 and 94 by four; of 192 35 and 100, 32 and 105; of 256 45 and 127, 33 and 113;
  // 20,000 rows of 76 98 and 367, 185 and 708; of 256 344 and 1,137, 278 and 1,202).  By the average: one long row
  // among short ones is one wave's work (20,000 edges in one of 20,000 rows of 30: 3.1 and 5.3 ms, by four 0.8 and 1.7)
  s.wpr = a.E / a.n >= 256 ? 4 : 1;
  s.rows = 1;
  return s;
}

}  // namespace

// Rows of a workgroup: one round of workgroups over the card, `per_cu` a CU.  Three are what its registers hold
// (20,000 atoms, forward and backward: 556 us; two 616, six 577, twelve 568; 256 molecules of 30: 76, 80, 81 and 82)
static int rows_of(const AttnArgs& a, int wpr, int per_cu) {
  const int least = wpr == 1 ? 4 : 1;
  return least * (int)(((int64_t)a.n + least * 256 * per_cu - 1) / (least * 256 * per_cu));
}

int attention_parts(const AttnArgs& a) {
  const int rows = rows_of(a, shape_of(a, false).wpr, 3);
  return (int)(((int64_t)a.n + rows - 1) / rows);
}

// floats of an edge's record: ds of every head, and the position gradient of every head group from *force on
int attention_record(const AttnArgs& a, int* force) {
  const int f = (a.H + 3) / 4 * 4;
  if (force) *force = f;
  return f + 4 * shape_of(a, false).groups;
}

// the kernel for the lanes of an edge, the type and one head a lane or more
#define E2F_ATT_T(P, ONE)         \
  if (a.bf16) {                   \
    E2F_ATT(P, ONE, BF16);        \
  } else {                        \
    E2F_ATT(P, ONE, F32);         \
  }
#define E2F_ATT_P(P)        \
  case P:                   \
    if (sh.one) {           \
      E2F_ATT_T(P, true)    \
    } else {                \
      E2F_ATT_T(P, false)   \
    }                       \
    break;
#define E2F_ATT_SWITCH                                                                                   \
  switch (sh.lpe) {                                                                                      \
    E2F_ATT_P(1) E2F_ATT_P(2) E2F_ATT_P(4) E2F_ATT_P(8) E2F_ATT_P(16) E2F_ATT_P(32) E2F_ATT_P(64)        \
    default: return hipErrorInvalidValue;                                                                \
  }

hipError_t launch_att_forward(const AttnArgs& a, float* alpha, float* lse, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  AttnShape sh = shape_of(a, false);
  const bool few = sh.heads <= 8;
  sh.lds = kKept * ((few ? 9 : kLd) + 2) + 64 + 64 + 256;
  sh.rows = sh.wpr == 1 ? 4 : 1;
  const Rounds r = rounds_of(((int64_t)a.n + sh.rows - 1) / sh.rows, 256);
  const dim3 grid(r.x, (unsigned)sh.groups, r.rounds);
  const size_t lds = sizeof(float) * 4 * sh.lds;
#define E2F_ATT(P, ONE, F)                                              \
  if (few)                                                              \
    k_att_forward<P, ONE, 9, F><<<grid, 256, lds, s>>>(a, sh, alpha, lse); \
  else                                                                  \
    k_att_forward<P, ONE, kLd, F><<<grid, 256, lds, s>>>(a, sh, alpha, lse)
  E2F_ATT_SWITCH
#undef E2F_ATT
  return hipGetLastError();
}

hipError_t launch_att_backward(const AttnArgs& a, const AttnGrad& gr, hipStream_t s) {
  if (a.n == 0) {  // (the sum over no edges)
    if (gr.gw) k_att_radial_sum<<<(a.H * a.R + 15) / 16, 1024, 0, s>>>(gr.part, 0, a.H * a.R, gr.gw);
    return hipGetLastError();
  }
  AttnShape sh = shape_of(a, false);
  AttnGrad g = gr;
  g.groups = sh.groups;
  g.stride = attention_record(a, &g.force);
  sh.rows = rows_of(a, sh.wpr, 3);
  const int parts = attention_parts(a), vec = a.bf16 ? BF16::VEC : F32::VEC;
  sh.dq = sh.one ? 0 : 64 / sh.lpe * sh.heads * sh.lph * vec;
  sh.lds = 64 * kLd + 7 * 64 + 256 + sh.dq;
  static_assert(64 * kLd + 7 * 64 + 256 >= 512, "room for dw's sum over the waves");
  {
    const dim3 grid((unsigned)parts, (unsigned)sh.groups);
    const size_t lds = sizeof(float) * 4 * sh.lds;
#define E2F_ATT(P, ONE, F) k_att_receivers<P, ONE, F><<<grid, 256, lds, s>>>(a, sh, g)
    E2F_ATT_SWITCH
#undef E2F_ATT
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (g.gw) k_att_radial_sum<<<(a.H * a.R + 15) / 16, 1024, 0, s>>>(g.part, parts, a.H * a.R, g.gw);
  if (g.gk || g.gpos) {
    sh = shape_of(a, true);
    const Rounds r = rounds_of(sh.wpr == 1 ? ((int64_t)a.n + 3) / 4 : a.n, 256);
    const dim3 grid(r.x, (unsigned)(g.gk ? sh.groups : 1), r.rounds);
#define E2F_SEND(P)                                          \
  case P:                                                    \
    if (a.bf16)                                              \
      k_att_senders<P, BF16><<<grid, 256, 0, s>>>(a, sh, g); \
    else                                                     \
      k_att_senders<P, F32><<<grid, 256, 0, s>>>(a, sh, g);  \
    break;
    switch (sh.lpe) {
      E2F_SEND(1) E2F_SEND(2) E2F_SEND(4) E2F_SEND(8) E2F_SEND(16) E2F_SEND(32) E2F_SEND(64)
      default: return hipErrorInvalidValue;
    }
#undef E2F_SEND
  }
  return hipGetLastError();
}

int transpose_scan_blocks(int n) { return (int)(((int64_t)n + kScanSpan - 1) / kScanSpan); }

hipError_t launch_transpose(const int64_t* row_ptr, const int32_t* col, int n, int64_t E, int32_t* cnt, int64_t* sums,
                            int32_t* pos, int64_t* rowT, int32_t* colT, int32_t* perm, hipStream_t s) {
  const Transposed t{row_ptr, col,     n,           E,    cnt,  cnt + n + 1, cnt + 2 * (int64_t)n + 1,
                     pos,     pos + E, pos + 2 * E, sums, rowT, colT,        perm};
  if (n == 0) {
    k_t_offset<<<1, 1024, 0, s>>>(t);
    return hipGetLastError();
  }
  const unsigned blocks = (unsigned)transpose_scan_blocks(n), nb = (unsigned)(((int64_t)n + 3) / 4);
  const Rounds r = rounds_of(nb, 256);
  k_t_zero<<<n / 256 + 1, 256, 0, s>>>(t);
  k_t_reverse<<<dim3(r.x, r.rounds), 256, 0, s>>>(t);
  if (E > 0) k_t_count<<<(unsigned)std::min<int64_t>((E + 255) / 256, 1024), 256, 0, s>>>(t);
  k_t_scan<<<blocks, 1024, 0, s>>>(t);
  if (blocks > 1) k_t_offset<<<blocks, 1024, 0, s>>>(t);
  if (E > 0) {
    k_t_place<<<std::min(nb, 8192u), 256, 0, s>>>(t);
    k_t_sort<<<std::min(nb, 8192u), 256, 0, s>>>(t);
  }
  return hipGetLastError();
}

}  // namespace e2f
