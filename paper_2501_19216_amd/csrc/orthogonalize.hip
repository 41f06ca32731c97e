// Orthogonalised updates of matrices (the update rule of the Muon optimiser): of the gradient G, or of what the momentum
// makes of it,
//   M' = mu M + G,   U = G + mu M' (Nesterov) or M',
// the matrix with U's singular vectors and singular values near one, by Newton-Schulz steps
//   X = U / (|U|_F + eps),   P = X X^T,   X <- a X + (b P + c P^2) X,
// and the weights W' = decay W + scale X.
//
// X stands with its shorter side as rows (m <= n), so that P is m x m: m^2 n + m^3 + 2 m^2 n operations a step, of which
// the products of a matrix with its own transpose need one triangle.  The steps raise the smallest singular values by up to a^steps,
// and with them whatever rounding the large ones left in their directions: products of 11 bits end 1e-3 from the exact
// matrix and sums over a X of 22 bits 3e-5, where float gives 1e-5 (200 x 333, an eighth of the directions strong).  So X stays float and
// a X is added in float; the products, whose errors stay in the directions that are already large, take their operands as two float16 numbers,
// x = hi + lo to 22 bits, in three products (hi hi, hi lo, lo hi) on the matrix cores, summed in float.  Powers of two keep the
// operands in float16's range: from the coefficients follow bounds of all singular values (ortho_bounds).
#include <hip/hip_runtime.h>

#include <cmath>

#include "e2f_launch.h"
#include "values.h"
#include "wave.h"

namespace e2f {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;   // rows and columns of a workgroup's product; matrices are padded to it with zeros
constexpr int kStep = 32;   // of the products' long axis
constexpr int kParts = 64;  // workgroups that sum a matrix's squares, at most
constexpr int kTable = 96;  // matrices of a launch: their addresses travel in the kernel's arguments

// A matrix as the products read it: rows of steps of 32 values, each step's hi and then its lo (128 bytes)
__host__ __device__ __forceinline__ int64_t split_at(int64_t row, int ld, int k, int lo) {
  return row * 2 * ld + (k >> 5) * 64 + lo * 32 + (k & 31);
}
__device__ __forceinline__ void split(float x, float scale, _Float16& hi, _Float16& lo) {
  const float y = x * scale;
  hi = (_Float16)y;
  lo = (_Float16)(y - (float)hi);
}

struct Table {
  const void* g[kTable];
  const float* m[kTable];
  float* to[kTable];
};
static_assert(sizeof(Table) <= 3584, "kernel arguments of 4 KB");
struct Ends {
  const void* w[kTable];
  void* out[kTable];
};

struct Sizes {
  int rows, cols, m, n, mp, np;  // m <= n: X's sides; mp, np: padded
  bool turned;                   // X is the transpose of the caller's matrices
};

// element i of the gradient or update
template <typename T>
__device__ __forceinline__ float value(const void* p, int64_t i) {
  return part(Raw<T, 1>::load((const char*)((const T*)p + i)), 0);
}

// The momentum, and the sum of the update's squares in float64, in which none of them overflows
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_norm(Table t, int64_t size, int parts, float mu, bool nesterov,
                                                    double* __restrict__ part) {
  const int z = blockIdx.y;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)parts * 256) {
    float u = value<T>(t.g[z], i);
    if (t.m[z]) {
      const float m = mu * t.m[z][i] + u;
      t.to[z][i] = m;
      u = nesterov ? u + mu * m : m;
    }
    s += (double)u * (double)u;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  __shared__ double w[4];
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)z * parts + blockIdx.x] = w[0] + w[1] + w[2] + w[3];
}

// X = U / (|U| + eps), in float [mp][np] and split, as it stands and transposed [np][mp]: a tile of 64 x 64 a workgroup
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_start(Table t, Sizes d, int parts, float mu, bool nesterov, float eps,
                                                     float scale, const double* __restrict__ part, float* __restrict__ x,
                                                     _Float16* __restrict__ xs, _Float16* __restrict__ xt) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  double norm = 0.0;
  for (int k = 0; k < parts; ++k) norm += part[(int64_t)z * parts + k];
  norm = sqrt(norm) + (double)eps;
  const int a = threadIdx.x & 63, b = threadIdx.x >> 6;
#pragma unroll 4
  for (int k = b; k < 64; k += 4) {
    // neighbouring lanes read neighbouring values of the caller's rows
    const int i = d.turned ? i0 + a : i0 + k, j = d.turned ? j0 + k : j0 + a;
    float u = 0.0f;
    if (i < d.m && j < d.n) {
      const int64_t at = d.turned ? (int64_t)j * d.cols + i : (int64_t)i * d.cols + j;
      u = value<T>(t.g[z], at);
      if (t.m[z]) u = nesterov ? u + mu * t.to[z][at] : t.to[z][at];
      u = (float)((double)u / norm);
    }
    tile[i - i0][j - j0] = u;
  }
  __syncthreads();
  x += (int64_t)z * d.mp * d.np, xs += (int64_t)z * d.mp * d.np * 2, xt += (int64_t)z * d.mp * d.np * 2;
#pragma unroll 4
  for (int k = b; k < 64; k += 4) {
    const float u = tile[k][a], v = tile[a][k];
    _Float16 hi, lo;
    x[(int64_t)(i0 + k) * d.np + j0 + a] = u;
    split(u, scale, hi, lo);
    xs[split_at(i0 + k, d.np, j0 + a, 0)] = hi, xs[split_at(i0 + k, d.np, j0 + a, 1)] = lo;
    split(v, scale, hi, lo);
    xt[split_at(j0 + k, d.mp, i0 + a, 0)] = hi, xt[split_at(j0 + k, d.mp, i0 + a, 1)] = lo;
  }
}

__device__ __forceinline__ v4f mfma(h8 a, h8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

enum { GRAM, POLY, APPLY };
struct Product {
  const _Float16 *p, *q;  // [rows][ld] split, the product's rows and columns
  int64_t sp, sq;         // values from one matrix to the next
  int ld, tiles;          // tiles of a row of the result
  float unscale;          // of the sums
  // GRAM: P split with `scale`; POLY: b P + c P^2 split with `scale`, P with `old`
  float b, c, old, scale;
  const _Float16* pin;
  _Float16* out;
  // APPLY: X <- a X + sums in float, split with `scale` as it stands and transposed
  float a;
  float* x;
  _Float16 *xs, *xt;
  int mp, np;
};

// One tile of 64 x 64 of  sum_k p[i][k] q[j][k]: four waves of 32 x 32, two buffers of a step in the LDS.  GRAM and POLY are
// symmetric: the tiles on and below the diagonal, each written at both its places
template <int KIND>
__global__ __launch_bounds__(256) void k_ortho_product(Product g) {
  __shared__ __align__(16) _Float16 lds[2][2][kTile * 72];  // rows of 128 bytes, 16 apart in the banks
  int ti, tj;
  if (KIND == APPLY) {
    ti = blockIdx.x / g.tiles, tj = blockIdx.x % g.tiles;
  } else {  // the number of the tile among those of the triangle
    ti = (int)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > (int)blockIdx.x) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= (int)blockIdx.x) ++ti;
    tj = (int)blockIdx.x - ti * (ti + 1) / 2;
  }
  const int z = blockIdx.y, i0 = ti * kTile, j0 = tj * kTile;
  const _Float16 *p = g.p + z * g.sp + (int64_t)i0 * 2 * g.ld, *q = g.q + z * g.sq + (int64_t)j0 * 2 * g.ld;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
  v4f acc[2][2] = {};
  // 64 rows of 128 bytes of each operand: four threads a row, 32 bytes each
  const int lr = threadIdx.x >> 2, lc = (threadIdx.x & 3) * 16;
  h8 rp[2], rq[2];
  auto fetch = [&](int s) {
    const int64_t at = (int64_t)lr * 2 * g.ld + s * 64 + lc;
#pragma unroll
    for (int u = 0; u < 2; ++u) rp[u] = *(const h8*)(p + at + u * 8), rq[u] = *(const h8*)(q + at + u * 8);
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      *(h8*)(&lds[buf][0][lr * 72 + lc + u * 8]) = rp[u];
      *(h8*)(&lds[buf][1][lr * 72 + lc + u * 8]) = rq[u];
    }
  };
  const int steps = g.ld / kStep;
  fetch(0);
  put(0);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
    if (s + 1 < steps) fetch(s + 1);
    const _Float16 *lp = lds[s & 1][0], *lq = lds[s & 1][1];
    h8 ph[2], pl[2], qh[2], ql[2];
    const int r = lane & 15, k = (lane >> 4) * 8;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ph[u] = *(const h8*)(lp + (wi + u * 16 + r) * 72 + k), pl[u] = *(const h8*)(lp + (wi + u * 16 + r) * 72 + 32 + k);
      qh[u] = *(const h8*)(lq + (wj + u * 16 + r) * 72 + k), ql[u] = *(const h8*)(lq + (wj + u * 16 + r) * 72 + 32 + k);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        acc[u][v] = mfma(pl[u], qh[v], acc[u][v]);
        acc[u][v] = mfma(ph[u], ql[v], acc[u][v]);
        acc[u][v] = mfma(ph[u], qh[v], acc[u][v]);
      }
    if (s + 1 < steps) put((s + 1) & 1);
  }
  // a lane holds rows 4 (lane / 16) .. + 3 of column lane % 16
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int i = i0 + wi + u * 16 + (lane >> 4) * 4, j = j0 + wj + v * 16 + (lane & 15);
      h4 hi, lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float s = acc[u][v][k] * g.unscale;
        if constexpr (KIND == POLY) {
          const _Float16* in = g.pin + z * g.sp;
          s = g.b * (((float)in[split_at(i + k, g.ld, j, 0)] + (float)in[split_at(i + k, g.ld, j, 1)]) * g.old) + g.c * s;
        }
        if constexpr (KIND == APPLY) {
          float* at = g.x + ((int64_t)z * g.mp + i + k) * g.np + j;
          s += g.a * *at;
          *at = s;
        }
        _Float16 h, l;
        split(s, g.scale, h, l);
        hi[k] = h, lo[k] = l;
        _Float16* out = KIND == APPLY ? g.xs + (int64_t)z * g.mp * g.np * 2 : g.out + (int64_t)z * g.mp * g.mp * 2;
        const int ld = KIND == APPLY ? g.np : g.mp;
        out[split_at(i + k, ld, j, 0)] = h, out[split_at(i + k, ld, j, 1)] = l;
      }
      if (KIND == APPLY || ti != tj) {
        _Float16* out = KIND == APPLY ? g.xt + (int64_t)z * g.mp * g.np * 2 : g.out + (int64_t)z * g.mp * g.mp * 2;
        *(h4*)(out + split_at(j, g.mp, i, 0)) = hi, *(h4*)(out + split_at(j, g.mp, i, 1)) = lo;
      }
    }
}

// W' = decay W + scale X
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_end(Ends t, Sizes d, float scale, float decay, const float* __restrict__ x) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, a = threadIdx.x & 63, b = threadIdx.x >> 6;
  x += (int64_t)z * d.mp * d.np;
#pragma unroll 4
  for (int k = b; k < 64; k += 4) tile[k][a] = x[(int64_t)(i0 + k) * d.np + j0 + a];
  __syncthreads();
#pragma unroll 4
  for (int k = b; k < 64; k += 4) {
    const int i = d.turned ? i0 + a : i0 + k, j = d.turned ? j0 + k : j0 + a;
    if (i >= d.m || j >= d.n) continue;
    const int64_t at = d.turned ? (int64_t)j * d.cols + i : (int64_t)i * d.cols + j;
    float f[1] = {scale * tile[i - i0][j - j0]};
    if (t.w[z]) f[0] += decay * value<T>(t.w[z], at);
    typename Raw<T, 1>::type v;
    join(f, v);
    Raw<T, 1>::store((char*)((T*)t.out[z] + at), v);
  }
}

Sizes sizes_of(int rows, int cols) {
  Sizes d{};
  d.rows = rows, d.cols = cols, d.turned = rows > cols;
  d.m = d.turned ? cols : rows, d.n = d.turned ? rows : cols;
  d.mp = (d.m + kTile - 1) / kTile * kTile, d.np = (d.n + kTile - 1) / kTile * kTile;
  return d;
}
struct Layout {
  size_t part, x, xs, xt[2], p, q, total;
};
Layout layout_of(const Sizes& d, int count) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) & ~size_t(255);
    return was;
  };
  const size_t all = 4 * (size_t)d.mp * d.np * count, square = 4 * (size_t)d.mp * d.mp * count;
  l.part = take(sizeof(double) * kParts * (size_t)count);
  l.x = take(all), l.xs = take(all), l.xt[0] = take(all), l.xt[1] = take(all), l.p = take(square), l.q = take(square);
  l.total = at;
  return l;
}

}  // namespace

bool ortho_bounds(int steps, const float* coef, int* x_exp, int* a_exp, int* b_exp) {
  // the largest exponent with which a value of this size, and one a little over it, stays below 2^15
  auto exponent = [](double most) {
    int e;
    frexp(most * 1.01, &e);  // most 1.01 < 2^e
    return 15 - e;
  };
  double top = 1.0;  // of the singular values: |U|_F bounds them
  for (int k = 0; k <= steps; ++k) {
    if (!(top <= 64.0)) return false;
    x_exp[k] = exponent(top < 0x1p-8 ? 0x1p-8 : top);
    if (k == steps) break;
    const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
    const double s2 = top * top;
    a_exp[k] = exponent(s2 < 0x1p-16 ? 0x1p-16 : s2);
    // |s (a + b t + c t^2)| and |b t + c t^2|, t = s^2: at their ends and where their derivatives vanish
    double next = 0.0, poly = 0.0;
    auto at = [&](double t) {
      if (!(t >= 0.0 && t <= s2)) return;
      next = std::fmax(next, std::fabs(std::sqrt(t) * (a + b * t + c * t * t)));
      poly = std::fmax(poly, std::fabs(b * t + c * t * t));
    };
    at(s2);
    if (c != 0.0) {
      at(-b / (2.0 * c));
      const double disc = 9.0 * b * b - 20.0 * a * c;
      if (disc >= 0.0) at((-3.0 * b + std::sqrt(disc)) / (10.0 * c)), at((-3.0 * b - std::sqrt(disc)) / (10.0 * c));
    } else if (b != 0.0) {
      at(-a / (3.0 * b));
    }
    if (!(poly <= 4096.0)) return false;
    b_exp[k] = exponent(poly < 0x1p-8 ? 0x1p-8 : poly);
    top = next * 1.001;
  }
  return true;
}

int ortho_batch(int rows, int cols, int count) {
  const Sizes d = sizes_of(rows, cols);
  const double each = 16.0 * d.mp * d.np + 8.0 * d.mp * d.mp;
  int b = each * kTable > 0x1p30 ? (int)(0x1p30 / each) : kTable;
  if (b < 1) b = 1;
  return count < b ? count : b;
}

size_t ortho_workspace(int rows, int cols, int count) {
  return layout_of(sizes_of(rows, cols), ortho_batch(rows, cols, count)).total;
}

hipError_t launch_orthogonalize(const OrthoArgs& a, void* workspace, hipStream_t st) {
  const Sizes d = sizes_of(a.rows, a.cols);
  const int batch = ortho_batch(a.rows, a.cols, a.count);
  const Layout l = layout_of(d, batch);
  char* ws = (char*)workspace;
  double* part = (double*)(ws + l.part);
  float* x = (float*)(ws + l.x);
  _Float16 *xs = (_Float16*)(ws + l.xs), *xt[2] = {(_Float16*)(ws + l.xt[0]), (_Float16*)(ws + l.xt[1])},
           *p = (_Float16*)(ws + l.p), *q = (_Float16*)(ws + l.q);
  int xe[kOrthoMaxSteps + 1], ae[kOrthoMaxSteps], be[kOrthoMaxSteps];
  if (!ortho_bounds(a.steps, a.coef, xe, ae, be)) return hipErrorInvalidValue;
  const int64_t size = (int64_t)a.rows * a.cols;
  int parts = (int)((size + 4095) / 4096);
  if (parts > kParts) parts = kParts;
  for (int first = 0; first < a.count; first += batch) {
    const int count = a.count - first < batch ? a.count - first : batch;
    Table t{};
    Ends e{};
    for (int k = 0; k < count; ++k) {
      t.g[k] = a.grads[first + k];
      t.m[k] = a.moments ? a.moments[first + k] : nullptr;
      t.to[k] = a.moments ? a.news[first + k] : nullptr;
      e.w[k] = a.weights && a.decay != 0.0f ? a.weights[first + k] : nullptr;
      e.out[k] = a.outs[first + k];
    }
    const dim3 tiles(d.np / 64, d.mp / 64, count);
    const float s0 = ldexpf(1.0f, xe[0]);
    if (a.grad_bf16) {
      k_ortho_norm<bf16_t><<<dim3(parts, count), 256, 0, st>>>(t, size, parts, a.mu, a.nesterov, part);
      k_ortho_start<bf16_t><<<tiles, 256, 0, st>>>(t, d, parts, a.mu, a.nesterov, a.eps, s0, part, x, xs, xt[0]);
    } else {
      k_ortho_norm<float><<<dim3(parts, count), 256, 0, st>>>(t, size, parts, a.mu, a.nesterov, part);
      k_ortho_start<float><<<tiles, 256, 0, st>>>(t, d, parts, a.mu, a.nesterov, a.eps, s0, part, x, xs, xt[0]);
    }
    const int mt = d.mp / kTile, nt = d.np / kTile;
    for (int k = 0; k < a.steps; ++k) {
      Product g{};
      g.mp = d.mp, g.np = d.np;
      g.p = g.q = xs, g.sp = g.sq = 2 * (int64_t)d.mp * d.np, g.ld = d.np;
      g.unscale = ldexpf(1.0f, -2 * xe[k]), g.scale = ldexpf(1.0f, ae[k]);
      Product poly = g, apply = g;
      g.out = p;
      poly.p = poly.q = poly.pin = p, poly.sp = poly.sq = 2 * (int64_t)d.mp * d.mp, poly.ld = d.mp, poly.out = q;
      poly.unscale = ldexpf(1.0f, -2 * ae[k]), poly.old = ldexpf(1.0f, -ae[k]), poly.scale = ldexpf(1.0f, be[k]);
      poly.b = a.coef[3 * k + 1], poly.c = a.coef[3 * k + 2];
      apply.p = q, apply.sp = poly.sp, apply.q = xt[k & 1], apply.sq = 2 * (int64_t)d.mp * d.np, apply.ld = d.mp;
      apply.unscale = ldexpf(1.0f, -be[k] - xe[k]), apply.scale = ldexpf(1.0f, xe[k + 1]), apply.a = a.coef[3 * k];
      apply.x = x, apply.xs = xs, apply.xt = xt[~k & 1], apply.tiles = nt;
      k_ortho_product<GRAM><<<dim3(mt * (mt + 1) / 2, count), 256, 0, st>>>(g);
      k_ortho_product<POLY><<<dim3(mt * (mt + 1) / 2, count), 256, 0, st>>>(poly);
      k_ortho_product<APPLY><<<dim3(mt * nt, count), 256, 0, st>>>(apply);
    }
    if (a.bf16)
      k_ortho_end<bf16_t><<<tiles, 256, 0, st>>>(e, d, a.scale, a.decay, x);
    else
      k_ortho_end<float><<<tiles, 256, 0, st>>>(e, d, a.scale, a.decay, x);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace e2f
