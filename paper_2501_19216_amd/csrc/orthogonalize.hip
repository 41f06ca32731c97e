// Orthogonalised updates of matrices (the update rule of the Muon optimiser): of the gradient G, or of what the
// momentum makes of it,
//   M' = mu M + G,   U = G + mu M' (Nesterov) or M',
// the matrix with U's singular vectors and singular values near one, by Newton-Schulz steps
//   X = U / (|U|_F + eps),   P = X X^T,   X <- a X + (b P + c P^2) X,
// and the weights W' = decay W + scale X.
//
// X stands with its shorter side as rows (m <= n), so that P is m x m: m^2 n + m^3 + 2 m^2 n operations a step, of
// which the products of a matrix with its own transpose need one triangle.  The steps raise the smallest singular
// values by up to a^steps, and with them whatever rounding the large ones left in their directions: products of 11
// bits end 3e-4 from the exact matrix, of 22 bits with a X among them 2e-5, where float gives 1e-5 (200 x 333, a
// sixteenth of the directions strong and the others a hundredth of them).  So X stays float and a X is added in
// float, which gives 1e-5 too; the products, whose errors stay in the directions that are already large, take their
// operands as two float16 numbers, x = hi + lo to 22 bits, in three products (hi hi, hi lo, lo hi) on the matrix
// cores, summed in float.  In all X ends 0.7e-6 to 2.2e-6 from the exact matrix (17 sizes from 16 x 16 to
// 1270 x 380, three spectra), 0.3 to 1.3 of where library products in float end; the operands' rounding alone, with exact
// sums, is 0.5e-6 to 0.7e-6 of it.  Powers of two keep the operands in float16's range: from the coefficients follow bounds of
// all singular values (ortho_bounds).
//
// Matrices that fit a workgroup's registers and LDS go through all steps there (k_ortho_small); larger ones through
// three tiled products a step.  Those hold Y = X^T alone: Y' = a Y + Y B (B = b P + c P^2 is symmetric) reads rows of
// Y and of B, and P = Y^T Y reads its operands by the LDS's transposing loads.
//
// Sixty matrices of 128 x 128 with momentum and weights take 50 us in one launch (without both 45; by three tiled
// products a step 94), of which a step is 7.4: matrix cores 3.3, reads of the LDS and four barriers between
// the phases, two waves a SIMD.  Four of 1024 x 4096 take 1.16 ms, 241 TFLOP/s (library products in float 72): P 84
// us a step, P^2 28, B X 120, the norm and the first Y 91.  B X is the sum of what its parts take alone: the matrix
// cores 45, the loads to the LDS 60 (20 bytes a cycle and CU), the float and split Y 41; more buffers of a step,
// tiles of 256, loads issued before the LDS is read, priorities of waves and other strides of memory left it where it
// is.
#include <hip/hip_runtime.h>

#include <cmath>

#include "e2f_launch.h"
#include "values.h"
#include "wave.h"

namespace e2f {
namespace {

typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kStep = 32;     // of the products' long axis
constexpr int kParts = 256;   // workgroups that sum a matrix's squares, at most
constexpr int kTable = 64;    // matrices of a launch: their addresses travel in the kernel's arguments

// A matrix as the products read it: rows of steps of 32 values, each step's hi and then its lo (128 bytes)
__host__ __device__ __forceinline__ int64_t split_at(int64_t row, int ld, int k, int lo) {
  return row * 2 * ld + (k >> 5) * 64 + lo * 32 + (k & 31);
}
// four floats, scaled, as two float16 numbers each: hi rounded to nearest, lo the rest
__device__ __forceinline__ void split(v4f x, float scale, h4& hi, h4& lo) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float y = x[k] * scale;
    hi[k] = (_Float16)y;
    lo[k] = (_Float16)(y - (float)hi[k]);
  }
}
__device__ __forceinline__ h8 both(h4 a, h4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ v4f mfma(h8 a, h8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// c += the products of operands split in two, the small parts first, and of all tiles one after the other: neighbours
// in the matrix cores' queue wait for no result
template <int A, int B>
__device__ __forceinline__ void products(const h8 (&ah)[A], const h8 (&al)[A], const h8 (&bh)[B], const h8 (&bl)[B],
                                         v4f (&c)[A][B]) {
#pragma unroll
  for (int i = 0; i < A; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) c[i][j] = mfma(al[i], bh[j], c[i][j]);
#pragma unroll
  for (int i = 0; i < A; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) c[i][j] = mfma(ah[i], bl[j], c[i][j]);
#pragma unroll
  for (int i = 0; i < A; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) c[i][j] = mfma(ah[i], bh[j], c[i][j]);
}
// Transposing load: of 16 lanes, lane s gives the address of four neighbours of row s / 4, from column 4 (s % 4) on,
// and lane t gets the four rows' values of column t
__device__ __forceinline__ h4 read_transposed(const _Float16* p) {
  return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p));
}

// 64 lanes' 16 bytes each to the LDS, lane after lane from `to` (the same for the wave) on, without passing
// registers.  By hand: the compiler, which cannot tell the LDS's buffers apart, would wait for all such loads before
// any read of the LDS. The instruction has no register for its result; who reads what it brings waits for vmcnt
// first, by hand as well.  It takes the LDS's address from m0 when it is issued; m0, which cannot be declared as
// changed, is what it was afterwards.
__device__ __forceinline__ void load_past(const _Float16* from, _Float16* to) {
  const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) _Float16*)to);
  unsigned was;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
               : "=&s"(was)
               : "s"(at), "v"(from)
               : "memory");
}

struct Table {
  const void* g[kTable];
  const float* m[kTable];
  float* to[kTable];
};
struct Ends {
  const void* w[kTable];
  void* out[kTable];
};

struct Sizes {
  int rows, cols, m, n, mp, np;  // m <= n: X's sides; mp, np: padded
  bool turned;                   // X is the transpose of the caller's matrices
};
struct Update {
  float mu, eps, scale, decay;
  bool nesterov;
};

template <typename T>
__device__ __forceinline__ float value(const void* p, int64_t i) {
  return part(Raw<T, 1>::load((const char*)((const T*)p + i)), 0);
}
// four neighbours of an array from i on, of which `have` are there (zeros behind)
template <typename T>
__device__ __forceinline__ v4f values(const void* p, int64_t i, int have) {
  v4f f = {};
  if (have >= 4) {
    const auto v = Raw<T, 4>::load((const char*)((const T*)p + i));
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = part(v, k);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < have) f[k] = value<T>(p, i + k);
  }
  return f;
}
template <typename T>
__device__ __forceinline__ void put(void* p, int64_t i, float x) {
  const float f[1] = {x};
  typename Raw<T, 1>::type v;
  join(f, v);
  Raw<T, 1>::store((char*)((T*)p + i), v);
}
template <typename T>
__device__ __forceinline__ void puts(void* p, int64_t i, int have, v4f x) {
  if (have >= 4) {
    const float f[4] = {x[0], x[1], x[2], x[3]};
    typename Raw<T, 4>::type v;
    join(f, v);
    Raw<T, 4>::store((char*)((T*)p + i), v);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < have) put<T>(p, i + k, x[k]);
  }
}

// What U is multiplied with, from the sum of its squares: NaN where a value is not finite, so that the others, which
// its reciprocal would make zeros, are NaN without a step as well
__device__ __forceinline__ double inverse_norm(double sum, float eps) {
  return sum < INFINITY ? 1.0 / (sqrt(sum) + (double)eps) : NAN;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// ------------------------------------------------------------------ matrices of a workgroup
// the steps' coefficients and, as exponents of two, the scales of X, P and B as operands
struct Steps {
  float coef[kOrthoMaxSteps][3];
  signed char x[kOrthoMaxSteps + 1], p[kOrthoMaxSteps], b[kOrthoMaxSteps];
  int count;
};
static_assert(sizeof(Table) + sizeof(Ends) + sizeof(Steps) + sizeof(Sizes) + sizeof(Update) <= 4032, "kernel arguments of 4 KB");
__device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }

// values of an LDS row, of X^T and of P: 16 rows of 32 bytes meet few equal banks
template <int MP>
struct Rows {
  static constexpr int X = MP + 24, P = MP + 16;
  static constexpr size_t bytes(int np) { return sizeof(_Float16) * 2 * ((size_t)np * X + (size_t)MP * P); }
};

// A matrix of up to MP rows and 128 S columns, a workgroup of eight waves each.  A wave holds S strips of 16 columns
// of X in registers as the matrix cores return them: lane l has rows 4 (l / 16) .. + 3 of every 16 and column l %
// 16.  These rows, of two 16s, are also what it gives as the right operand of B X, so B's columns are stored in that
// order (within 32: 16 h + 4 g + e at 8 g + 4 h + e).  X^T lies in the LDS for P.  P, and B that replaces it, are
// symmetric: a tile is stored as its transpose
template <int MP, int S, typename TG, typename T>
__global__ __launch_bounds__(512) void k_ortho_small(Table t, Ends e, Steps steps, Sizes d, Update u) {
  constexpr int MT = MP / 16, SX = Rows<MP>::X, SP = Rows<MP>::P;
  // P's tiles of a wave, in a row: of six and eight rows of tiles the one on the diagonal and half of the row's
  // others, in a circle, each written at both its places; of fewer all tiles, shared by the eight waves
  constexpr bool BAND = MT >= 6;
  constexpr int BC = BAND ? MT / 2 + 1 : MT / 2, COLS = MT / BC;
  extern __shared__ __align__(16) _Float16 lds[];
  __shared__ double squares[8];
  _Float16 *xh = lds, *xl = xh + d.np * SX, *ph = xl + d.np * SX, *pl = ph + MP * SP;
  const int z = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  // the update's four neighbours of the caller's matrix from `at` on, of which `have` are there; the momentum on the
  // way
  auto update = [&](int64_t at, int have) {
    v4f v = values<TG>(t.g[z], at, have);
    if (t.m[z]) {
      const v4f m = values<float>(t.m[z], at, have) * u.mu + v;
      puts<float>(t.to[z], at, have, m);
      v = u.nesterov ? v + u.mu * m : m;
    }
    return v;
  };
  // rows of the caller's matrix pass through the LDS where they are not X's columns: four neighbours a lane either way
  float* stage = (float*)lds;  // [MP][SN], in X^T's place
  const int SN = d.np + 4, quads = d.np / 4;
  if (!d.turned) {
    for (int k = threadIdx.x; k < MP * quads; k += 512) {
      const int i = k / quads, j = k % quads * 4;
      *(v4f*)(stage + i * SN + j) = i < d.m && j < d.n ? update((int64_t)i * d.cols + j, d.n - j) : v4f{};
    }
    __syncthreads();
  }
  v4f x[S][MT];
  double sum = 0.0;
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int tau = 0; tau < MT; ++tau) {
      const int j = (wave + 8 * s) * 16 + c, i = tau * 16 + 4 * g;
      v4f v = {};
      if (d.turned) {
        if (j < d.n && i < d.m) v = update((int64_t)j * d.cols + i, d.m - i);
      } else if (j < d.np) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = stage[(i + r) * SN + j];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += (double)v[r] * (double)v[r];
      x[s][tau] = v;
    }
  sum = wave_sum(sum);
  if (lane == 0) squares[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += squares[w];
  const double inv = inverse_norm(sum, u.eps);
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int tau = 0; tau < MT; ++tau)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[s][tau][r] = (float)((double)x[s][tau][r] * inv);

  const int br = BAND ? wave : wave / COLS;
  const bool tiles = br < MT;
  int bc[BC];
#pragma unroll
  for (int b = 0; b < BC; ++b) bc[b] = BAND ? (wave + b) % MT : wave % COLS * BC + b;
  for (int k = 0; k < steps.count; ++k) {
    const float sx = power(steps.x[k]), sp = power(steps.p[k]), sb = power(steps.b[k]);
    h4 hi[S][MT], lo[S][MT];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int tau = 0; tau < MT; ++tau) {
        split(x[s][tau], sx, hi[s][tau], lo[s][tau]);
        const int j = (wave + 8 * s) * 16 + c;
        if ((wave + 8 * s) * 16 < d.np) {
          *(h4*)(xh + j * SX + tau * 16 + 4 * g) = hi[s][tau];
          *(h4*)(xl + j * SX + tau * 16 + 4 * g) = lo[s][tau];
        }
      }
    __syncthreads();
    // P = X X^T
    v4f p[1][BC] = {}, q[1][BC] = {};
    if (tiles)
      for (int j = 0; j < d.np; j += 32) {
        const int row = (j + 8 * g + (c >> 2)) * SX + 4 * (c & 3);
        auto read = [&](const _Float16* of, int tile) {
          const _Float16* at = of + row + tile * 16;
          return both(read_transposed(at), read_transposed(at + 4 * SX));
        };
        const h8 ah[1] = {read(xh, br)}, al[1] = {read(xl, br)};
        h8 bh[BC], bl[BC];
#pragma unroll
        for (int b = 0; b < BC; ++b) bh[b] = read(xh, bc[b]), bl[b] = read(xl, bc[b]);
        products<1, BC>(ah, al, bh, bl, p);
      }
    auto store = [&](const v4f(&m)[1][BC], float scale) {
#pragma unroll
      for (int b = 0; b < BC; ++b) {
        if (BAND && b == MT / 2 && br >= MT / 2) continue;  // (the other of the two has it)
        h4 h, l;
        split(m[0][b], scale, h, l);
        const int at = (bc[b] * 16 + c) * SP + (br >> 1) * 32 + 8 * g + (br & 1) * 4;
        *(h4*)(ph + at) = h, *(h4*)(pl + at) = l;
        if (BAND && b > 0) {
          const int to = (br * 16 + 4 * g) * SP + (bc[b] >> 1) * 32 + 8 * (c >> 2) + (bc[b] & 1) * 4 + (c & 3);
#pragma unroll
          for (int r = 0; r < 4; ++r) ph[to + r * SP] = h[r], pl[to + r * SP] = l[r];
        }
      }
    };
    if (tiles) {
      const float off = power(-2 * steps.x[k]);
#pragma unroll
      for (int b = 0; b < BC; ++b) p[0][b] *= off;
      store(p, sp);
    }
    __syncthreads();
    // B = b P + c P^2
    if (tiles)
#pragma unroll
      for (int kb = 0; kb < MP; kb += 32) {
        auto read = [&](const _Float16* of, int tile) { return *(const h8*)(of + (tile * 16 + c) * SP + kb + 8 * g); };
        const h8 ah[1] = {read(ph, br)}, al[1] = {read(pl, br)};
        h8 bh[BC], bl[BC];
#pragma unroll
        for (int b = 0; b < BC; ++b) bh[b] = read(ph, bc[b]), bl[b] = read(pl, bc[b]);
        products<1, BC>(ah, al, bh, bl, q);
      }
    __syncthreads();
    if (tiles) {
      const float by = steps.coef[k][1], cy = steps.coef[k][2] * power(-2 * steps.p[k]);
#pragma unroll
      for (int b = 0; b < BC; ++b) q[0][b] = by * p[0][b] + cy * q[0][b];
      store(q, sb);
    }
    __syncthreads();
    // X <- a X + B X
    const float off = power(-steps.b[k] - steps.x[k]);
    constexpr int AT = MT % 4 ? 2 : 4;  // tiles side by side
    if (wave * 16 < d.np)
#pragma unroll
      for (int tau = 0; tau < MT; tau += AT) {
        v4f y[AT][S] = {};
#pragma unroll
        for (int kb = 0; kb < MT / 2; ++kb) {
          h8 ah[AT], al[AT], bh[S], bl[S];
#pragma unroll
          for (int a = 0; a < AT; ++a) {
            const int at = ((tau + a) * 16 + c) * SP + kb * 32 + 8 * g;
            ah[a] = *(const h8*)(ph + at), al[a] = *(const h8*)(pl + at);
          }
#pragma unroll
          for (int s = 0; s < S; ++s)
            bh[s] = both(hi[s][2 * kb], hi[s][2 * kb + 1]), bl[s] = both(lo[s][2 * kb], lo[s][2 * kb + 1]);
          products<AT, S>(ah, al, bh, bl, y);
        }
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
          for (int s = 0; s < S; ++s) x[s][tau + a] = steps.coef[k][0] * x[s][tau + a] + off * y[a][s];
      }
  }
  auto end = [&](int64_t at, int have, v4f v) {
    v *= u.scale;
    puts<T>(e.out[z], at, have, e.w[z] ? v + u.decay * values<T>(e.w[z], at, have) : v);
  };
  if (!d.turned) __syncthreads();  // (without steps what was staged is still read)
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int tau = 0; tau < MT; ++tau) {
      const int j = (wave + 8 * s) * 16 + c, i = tau * 16 + 4 * g;
      if (d.turned) {
        if (j < d.n && i < d.m) end((int64_t)j * d.cols + i, d.m - i, x[s][tau]);
      } else if (j < d.np) {
#pragma unroll
        for (int r = 0; r < 4; ++r) stage[(i + r) * SN + j] = x[s][tau][r];
      }
    }
  if (d.turned) return;
  __syncthreads();
  for (int k = threadIdx.x; k < MP * quads; k += 512) {
    const int i = k / quads, j = k % quads * 4;
    if (i < d.m && j < d.n) end((int64_t)i * d.cols + j, d.n - j, *(const v4f*)(stage + i * SN + j));
  }
}

// ------------------------------------------------------------------ larger matrices
// The momentum, and the sum of the update's squares in float64, in which none of them overflows
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_norm(Table t, int64_t size, int parts, Update u, double* __restrict__ part) {
  const int z = blockIdx.y;
  double s = 0.0;
#pragma unroll 2
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)parts * 1024) {
    const int have = (int)min(size - i, (int64_t)4);
    v4f v = values<T>(t.g[z], i, have);
    if (t.m[z]) {
      const v4f m = values<float>(t.m[z], i, have) * u.mu + v;
      puts<float>(t.to[z], i, have, m);
      v = u.nesterov ? v + u.mu * m : m;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s += (double)v[k] * (double)v[k];
  }
  s = wave_sum(s);
  __shared__ double w[4];
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)z * parts + blockIdx.x] = w[0] + w[1] + w[2] + w[3];
}

// Y = (U / (|U| + eps))^T, in float [np][mp] and split: a tile of 64 x 64 a workgroup
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_start(Table t, Sizes d, int parts, Update u, float scale,
                                                     const double* __restrict__ part, float* __restrict__ y,
                                                     _Float16* __restrict__ ys) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  double norm = 0.0;
  for (int k = threadIdx.x & 63; k < parts; k += 64) norm += part[(int64_t)z * parts + k];
  const double inv = inverse_norm(wave_sum(norm), u.eps);
  const int a = (threadIdx.x & 15) * 4, b = threadIdx.x >> 4;
  // four neighbours of the caller's matrix, of which `have` are there
  auto read = [&](int64_t at, int have) {
    v4f v = values<T>(t.g[z], at, have);
    if (t.m[z]) {
      const v4f m = values<float>(t.to[z], at, have);
      v = u.nesterov ? v + u.mu * m : m;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (float)((double)v[k] * inv);
    return v;
  };
  v4f v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = q * 16 + b;
    v[q] = v4f{};
    if (d.turned) {
      if (j0 + r < d.n && i0 + a < d.m) v[q] = read((int64_t)(j0 + r) * d.cols + i0 + a, d.m - i0 - a);
    } else if (i0 + r < d.m && j0 + a < d.n) {
      v[q] = read((int64_t)(i0 + r) * d.cols + j0 + a, d.n - j0 - a);
    }
  }
  if (!d.turned) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int k = 0; k < 4; ++k) tile[q * 16 + b][a + k] = v[q][k];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[q][k] = tile[a + k][q * 16 + b];
  }
  y += (int64_t)z * d.mp * d.np, ys += (int64_t)z * d.mp * d.np * 2;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t j = j0 + q * 16 + b;
    h4 hi, lo;
    split(v[q], scale, hi, lo);
    *(v4f*)(y + j * d.mp + i0 + a) = v[q];
    *(h4*)(ys + split_at(j, d.mp, i0 + a, 0)) = hi;
    *(h4*)(ys + split_at(j, d.mp, i0 + a, 1)) = lo;
  }
}

enum { GRAM, POLY, APPLY, LAST };
struct Product {
  const _Float16 *p, *q;  // split matrices: rows of the product's rows and columns (GRAM: of its sums), ld values each
  int64_t sp, sq;         // from one matrix to the next
  int ld, steps;          // of kStep
  int tiles, count;       // tiles of a matrix's result, matrices
  float unscale;          // of the sums
  float a, b, c, old, scale;
  _Float16* out;          // GRAM: P; POLY: B = b P + c P^2, P (p) scaled with `old`; APPLY: Y, all split with `scale`
  float* y;               // APPLY: Y <- a Y + sums;  LAST: the same, to the caller's matrices
  int mp, np;
};

// One tile of TILE x TILE of  sum_k p[i][k] q[j][k]  (GRAM: p[k][i] q[k][j]), WI x WJ waves, or WK times as many that
// take the steps in turn and add their sums at the end, with ST buffers of a (WK) step(s) in the LDS: the values of
// ST - 1 steps are on their way there, without passing registers, while one step's products run. GRAM and POLY are
// symmetric: the tiles on and below the diagonal, each written at both its places.  A lane has four neighbouring rows
// i of a column j, which are neighbours in memory at row j of Y, and of the symmetric P and B.
//
// In the LDS a row of 128 bytes (GRAM: of 4 TILE bytes) has its 16 bytes at position c ^ row % 8 (its 32 bytes at c ^
// a number of the row): lanes that read together meet different banks, and the loads, which write 64 x 16 bytes in
// their order, read the places that belong there
template <int KIND, int TILE, int WI, int WJ, int WK, int ST, typename T>
__global__ __launch_bounds__(64 * WI * WJ * WK) void k_ortho_product(Product g, Ends e, Sizes d, Update u) {
  constexpr int FI = TILE / 16 / WI, FJ = TILE / 16 / WJ, N = TILE / 8 / (WI * WJ);  // N: loads of a wave and operand
  __shared__ __align__(16) _Float16 lds[ST][WK][2][TILE * 64];
  static_assert(sizeof(lds) >= sizeof(float) * TILE * TILE, "a tile of floats");
  // neighbouring workgroups lie on different dies: each die takes a stretch of neighbouring tiles, which share rows
  // in its L2
  const int all = g.tiles * g.count, each = (all + 7) >> 3, at_ = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if (at_ >= all || (int)(blockIdx.x >> 3) >= each) return;
  const int z = at_ / g.tiles, tile = at_ % g.tiles;
  int ti, tj;
  if (KIND >= APPLY) {
    ti = tile % (g.mp / TILE), tj = tile / (g.mp / TILE);
  } else {  // the number of the tile among those of the triangle
    ti = (int)((sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    tj = tile - ti * (ti + 1) / 2;
  }
  const int i0 = ti * TILE, j0 = tj * TILE;
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = all_waves % (WI * WJ), wk = all_waves / (WI * WJ);  // (and which of a round's steps it has)
  const int wi = wave / WJ * (FI * 16), wj = wave % WJ * (FJ * 16), lg = lane >> 4, lc = lane & 15;
  // where this lane's 16 bytes of each load come from, and how far a step is
  const int64_t step = KIND == GRAM ? (int64_t)kStep * 2 * g.ld : 2 * kStep;
  const _Float16 *p[N], *q[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int chunk = (wave * N + n) * 64 + lane;
    int64_t from;
    if (KIND == GRAM) {
      constexpr int PER = TILE / 4;  // of a row
      const int k = chunk / PER, to = chunk % PER, h = (k & 3) | (k >> 3 & 1) << 2;
      from = (int64_t)k * 2 * g.ld + (((to >> 1) ^ h) * 2 + (to & 1)) * 8;
    } else {
      const int r = chunk >> 3;
      from = (int64_t)r * 2 * g.ld + ((chunk & 7) ^ (r & 7)) * 8;
    }
    from += wk * step;
    p[n] = g.p + z * g.sp + (KIND == GRAM ? 2 * i0 : (int64_t)i0 * 2 * g.ld) + from;
    q[n] = g.q + z * g.sq + (KIND == GRAM ? 2 * j0 : (int64_t)j0 * 2 * g.ld) + from;
  }
  auto fetch = [&](int buf) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      load_past(p[n], &lds[buf][wk][0][(wave * N + n) * 512]);
      load_past(q[n], &lds[buf][wk][1][(wave * N + n) * 512]);
      p[n] += WK * step, q[n] += WK * step;
    }
  };
  // 16 of the tile's rows from `row` on, part 0 (hi) or 1 (lo), as an operand
  auto operand = [&](const _Float16* l, int row, int part) {
    if constexpr (KIND == GRAM) {
      const int h = (lc >> 2) | (lg & 1) << 2, pair = (row >> 5) * 4 + part * 2 + (row >> 4 & 1);
      const _Float16* a = l + (8 * lg + (lc >> 2)) * (2 * TILE) + (pair ^ h) * 16 + 4 * (lc & 3);
      return both(read_transposed(a), read_transposed(a + 4 * 2 * TILE));
    } else {
      return *(const h8*)(l + (row + lc) * 64 + ((part * 4 + lg) ^ (lc & 7)) * 8);
    }
  };
  v4f acc[FI][FJ] = {}, old[KIND >= APPLY ? FI : 1][KIND >= APPLY ? FJ : 1];
  const int steps = g.steps / WK;
#pragma unroll
  for (int s = 0; s + 1 < ST; ++s)
    if (s < steps) fetch(s);
  if constexpr (KIND >= APPLY) {  // Y, needed at the end
#pragma unroll
    for (int a = 0; a < FI; ++a)
#pragma unroll
      for (int b = 0; b < FJ; ++b)
        old[a][b] = *(const v4f*)(g.y + ((int64_t)z * g.np + j0 + wj + b * 16 + lc) * g.mp + i0 + wi + a * 16 + lg * 4);
  }
  int buf = 0, to = ST - 1;
  for (int s = 0; s < steps; ++s) {
    // this step's values are there (those of the steps behind it may be on their way), and the buffer that is filled
    // next has been read by every wave
    if (s + ST - 1 <= steps)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((ST - 2) * 2 * N) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const _Float16 *lp = lds[buf][wk][0], *lq = lds[buf][wk][1];
    h8 ph[FI], pl[FI], qh[FJ], ql[FJ];
#pragma unroll
    for (int a = 0; a < FI; ++a) ph[a] = operand(lp, wi + a * 16, 0), pl[a] = operand(lp, wi + a * 16, 1);
#pragma unroll
    for (int b = 0; b < FJ; ++b) qh[b] = operand(lq, wj + b * 16, 0), ql[b] = operand(lq, wj + b * 16, 1);
    if (s + ST - 1 < steps) fetch(to);
    products<FI, FJ>(ph, pl, qh, ql, acc);
    buf = buf + 1 == ST ? 0 : buf + 1, to = to + 1 == ST ? 0 : to + 1;
  }
  float* turn = (float*)&lds[0][0][0][0];  // [TILE][TILE]
  if constexpr (KIND == LAST || WK > 1) __syncthreads();  // (the last step's operands have been read)
  if constexpr (WK > 1) {  // the sums of a tile's waves together, in their order
#pragma unroll
    for (int w = 1; w < WK; ++w) {
      if (wk == w) {
#pragma unroll
        for (int a = 0; a < FI; ++a)
#pragma unroll
          for (int b = 0; b < FJ; ++b) *(v4f*)(turn + (((wave * FI + a) * FJ + b) * 64 + lane) * 4) = acc[a][b];
      }
      __syncthreads();
      if (wk == 0) {
#pragma unroll
        for (int a = 0; a < FI; ++a)
#pragma unroll
          for (int b = 0; b < FJ; ++b) acc[a][b] += *(const v4f*)(turn + (((wave * FI + a) * FJ + b) * 64 + lane) * 4);
      }
      __syncthreads();
    }
  }
  if (wk == 0) {
#pragma unroll
    for (int a = 0; a < FI; ++a)
#pragma unroll
      for (int b = 0; b < FJ; ++b) {
        const int i = i0 + wi + a * 16 + lg * 4, j = j0 + wj + b * 16 + lc;
        v4f s = acc[a][b] * g.unscale;
        if constexpr (KIND == POLY) {
          const _Float16* in = g.p + z * g.sp;
          const h4 hi = *(const h4*)(in + split_at(j, g.mp, i, 0)), lo = *(const h4*)(in + split_at(j, g.mp, i, 1));
#pragma unroll
          for (int k = 0; k < 4; ++k) s[k] = g.b * (((float)hi[k] + (float)lo[k]) * g.old) + g.c * s[k];
        }
        if constexpr (KIND >= APPLY) {
          s += g.a * old[a][b];
          if constexpr (KIND == APPLY) *(v4f*)(g.y + ((int64_t)z * g.np + j) * g.mp + i) = s;
        }
        if constexpr (KIND == LAST) {
          if (d.turned) {
            if (j >= d.n || i >= d.m) continue;
            const int64_t at = (int64_t)j * d.cols + i;
            s *= u.scale;
            puts<T>(e.out[z], at, d.m - i, e.w[z] ? s + u.decay * values<T>(e.w[z], at, d.m - i) : s);
          } else {
            // the caller's rows are i: by the LDS, 16 columns at a place that goes by the row (four lanes' rows meet
            // other banks)
#pragma unroll
            for (int k = 0; k < 4; ++k) turn[(i - i0 + k) * TILE + ((j - j0) ^ (lg * 16))] = s[k];
          }
        } else {
          h4 hi, lo;
          split(s, g.scale, hi, lo);
          _Float16* out = g.out + (int64_t)z * (KIND == APPLY ? g.np : g.mp) * g.mp * 2;
          *(h4*)(out + split_at(j, g.mp, i, 0)) = hi, *(h4*)(out + split_at(j, g.mp, i, 1)) = lo;
          if (KIND != APPLY && ti != tj) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              out[split_at(i + k, g.mp, j, 0)] = hi[k], out[split_at(i + k, g.mp, j, 1)] = lo[k];
          }
        }
      }
  }
  if constexpr (KIND == LAST) {
    if (d.turned) return;
    __syncthreads();
#pragma unroll 4
    for (int k = threadIdx.x; k < TILE * TILE / 4; k += 64 * WI * WJ * WK) {
      const int r = k / (TILE / 4), c = k % (TILE / 4) * 4, i = i0 + r, j = j0 + c;
      if (i >= d.m || j >= d.n) continue;
      const v4f s = *(const v4f*)(turn + r * TILE + (c ^ (r >> 2 & 3) * 16)) * u.scale;
      const int64_t at = (int64_t)i * d.cols + j;
      puts<T>(e.out[z], at, d.n - j, e.w[z] ? s + u.decay * values<T>(e.w[z], at, d.n - j) : s);
    }
  }
}

// no steps: out = decay W + scale X from Y
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_end(Ends e, Sizes d, Update u, const float* __restrict__ y) {
  const int z = blockIdx.y;
  const int64_t size = (int64_t)d.m * d.n;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < size; at += (int64_t)gridDim.x * 256) {
    const int r = (int)(at / d.cols), c = (int)(at % d.cols), i = d.turned ? c : r, j = d.turned ? r : c;
    const float v = u.scale * y[((int64_t)z * d.np + j) * d.mp + i];
    put<T>(e.out[z], at, e.w[z] ? v + u.decay * value<T>(e.w[z], at) : v);
  }
}

// The rows that k_ortho_small is made for, 0 where a matrix does not fit a workgroup, and its strips of a wave
int small_rows(int m) { return m <= 32 ? 32 : m <= 64 ? 64 : m <= 96 ? 96 : m <= 128 ? 128 : 0; }
constexpr size_t kLds = 160 * 1024 - 1024;
size_t small_bytes(int mp, int np) {
  return mp == 32 ? Rows<32>::bytes(np) : mp == 64 ? Rows<64>::bytes(np) : mp == 96 ? Rows<96>::bytes(np) : Rows<128>::bytes(np);
}

Sizes sizes_of(int rows, int cols, int count, bool* small, int* tile) {
  Sizes d{};
  d.rows = rows, d.cols = cols, d.turned = rows >= cols;  // (of square ones the transpose, whose columns are rows in memory)
  d.m = d.turned ? cols : rows, d.n = d.turned ? rows : cols;
  d.mp = small_rows(d.m), d.np = (d.n + 31) / 32 * 32;
  // (without momentum and weights, as all times here: sixty of 128 x 128 45 us, by tiled products 94; one 44 and 76, 200 of
  // them 177 and 365; sixty of 64 x 384, whose four strips of a wave leave four registers in memory, 45 and 107)
  *small = d.mp && d.np <= 512 && small_bytes(d.mp, d.np) <= kLds;
  if (*small) return d;
  // tiles of 128, each value of which is loaded and read from the LDS half as often, where they fill the GPU and pad
  // little (four matrices of 1024 x 4096 1.10 ms, with tiles of 64 1.25; one 397 us and 414; 64 of 512 x 512 0.97 and 1.04
  // ms; but 30 of 400 x 400, which become 512, 428 and 371 us, and one of 1024 x 1024, 64 tiles, 281 and 190)
  const int64_t tiles = (int64_t)((d.m + 127) / 128) * ((d.n + 127) / 128);
  const int64_t fine = (int64_t)((d.m + 63) / 64) * ((d.n + 63) / 64);
  *tile = tiles * (count < kTable ? count : kTable) >= 256 && 40 * tiles <= 11 * fine ? 128 : 64;
  d.mp = (d.m + *tile - 1) / *tile * *tile, d.np = (d.n + *tile - 1) / *tile * *tile;
  return d;
}
struct Layout {
  size_t part, y, ys[2], p, b, total;
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
  l.y = take(all), l.ys[0] = take(all), l.ys[1] = take(all), l.p = take(square), l.b = take(square);
  l.total = at;
  return l;
}

// matrices at a time: as many as a launch's arguments hold, and 1 GB of workspace
int batch_of(const Sizes& d, int count) {
  const double each = 12.0 * d.mp * d.np + 8.0 * d.mp * d.mp;
  int b = each * kTable > 0x1p30 ? (int)(0x1p30 / each) : kTable;
  if (b < 1) b = 1;
  return count < b ? count : b;
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

size_t ortho_workspace(int rows, int cols, int count) {
  bool small;
  int tile;
  const Sizes d = sizes_of(rows, cols, count, &small, &tile);
  return small ? 0 : layout_of(d, batch_of(d, count)).total;
}

namespace {

// an attribute of the kernel, not of a stream: allowed while one is captured
template <typename K>
hipError_t allow_lds(K kernel, size_t bytes) {
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename TG, typename T>
hipError_t launch_small(const Table& t, const Ends& e, const Steps& steps, const Sizes& d, const Update& u, int count,
                        hipStream_t st) {
  const int strips = (d.np + 127) / 128;
  const size_t bytes = small_bytes(d.mp, d.np);
#define E2F_ORTHO(MP, S)                                                                             \
  do {                                                                                               \
    const hipError_t err = allow_lds(k_ortho_small<MP, S, TG, T>, bytes);                            \
    if (err != hipSuccess) return err;                                                               \
    k_ortho_small<MP, S, TG, T><<<count, 512, bytes, st>>>(t, e, steps, d, u);                       \
  } while (0)
  if (d.mp == 128)
    E2F_ORTHO(128, 1);
  else if (d.mp == 96 && strips == 1)
    E2F_ORTHO(96, 1);
  else if (d.mp == 96)
    E2F_ORTHO(96, 2);
  else if (d.mp == 64 && strips == 1)
    E2F_ORTHO(64, 1);
  else if (d.mp == 64 && strips == 2)
    E2F_ORTHO(64, 2);
  else if (d.mp == 64)
    E2F_ORTHO(64, 4);
  else if (strips == 1)
    E2F_ORTHO(32, 1);
  else if (strips == 2)
    E2F_ORTHO(32, 2);
  else
    E2F_ORTHO(32, 4);
#undef E2F_ORTHO
  return hipGetLastError();
}

template <int KIND, typename T>
void launch_product(int tile, Product g, const Ends& e, const Sizes& d, const Update& u, hipStream_t st) {
  const int mt = g.mp / tile;
  g.tiles = KIND >= APPLY ? mt * (g.np / tile) : mt * (mt + 1) / 2;
  const unsigned blocks = (unsigned)((g.tiles * g.count + 7) / 8 * 8);
  if (tile == 128)
    k_ortho_product<KIND, 128, 2, 4, 1, 2, T><<<blocks, 512, 0, st>>>(g, e, d, u);
  // (300 x 3000 204 us, with four waves 250; 1024 x 1024 190 and 219; six of 517 x 200 119 and 126.  Beyond the bounds it
  // makes no difference: 12 of 300 x 3000 404 us and 409, one of 200 x 200 93.5 and 95.0)
  else if (g.tiles * g.count <= 256 && g.steps >= 16)
    k_ortho_product<KIND, 64, 2, 2, 2, 3, T><<<blocks, 512, 0, st>>>(g, e, d, u);
  else
    k_ortho_product<KIND, 64, 2, 2, 1, 3, T><<<blocks, 256, 0, st>>>(g, e, d, u);
}

template <typename TG, typename T>
hipError_t launch_large(const Table& t, const Ends& e, const Steps& steps, const Sizes& d, const Update& u, int tile,
                        int count, const Layout& l, char* ws, hipStream_t st) {
  double* part = (double*)(ws + l.part);
  float* y = (float*)(ws + l.y);
  _Float16 *ys[2] = {(_Float16*)(ws + l.ys[0]), (_Float16*)(ws + l.ys[1])}, *p = (_Float16*)(ws + l.p), *b = (_Float16*)(ws + l.b);
  const int64_t size = (int64_t)d.rows * d.cols;
  int64_t parts = (size + 8191) / 8192;
  if (parts > kParts) parts = kParts;
  k_ortho_norm<TG><<<dim3((unsigned)parts, count), 256, 0, st>>>(t, size, (int)parts, u, part);
  k_ortho_start<TG><<<dim3(d.np / 64, d.mp / 64, count), 256, 0, st>>>(t, d, (int)parts, u, ldexpf(1.0f, steps.x[0]), part,
                                                                       y, ys[0]);
  const int mt = d.mp / 128;
  // (the triangle's tiles are fewer: tiles of 64 until 512 of 128 are there.  One matrix of 4096 x 4096, 528 of them, 4.36
  // ms against 5.26 with 64; four of 1024 x 4096, 144 of them, 1.21 ms against 1.09)
  const int tri = tile == 128 && (int64_t)mt * (mt + 1) / 2 * count >= 512 ? 128 : 64;
  for (int k = 0; k < steps.count; ++k) {
    const int xe = steps.x[k], pe = steps.p[k], be = steps.b[k];
    Product g{};
    g.mp = d.mp, g.np = d.np, g.count = count, g.y = y, g.ld = d.mp;
    g.a = steps.coef[k][0], g.b = steps.coef[k][1], g.c = steps.coef[k][2];
    const int64_t all = 2 * (int64_t)d.mp * d.np, square = 2 * (int64_t)d.mp * d.mp;
    Product poly = g, apply = g;
    g.p = g.q = ys[k & 1], g.sp = g.sq = all, g.steps = d.np / kStep, g.out = p;
    g.unscale = ldexpf(1.0f, -2 * xe), g.scale = ldexpf(1.0f, pe);
    poly.p = poly.q = p, poly.sp = poly.sq = square, poly.steps = d.mp / kStep, poly.out = b;
    poly.unscale = ldexpf(1.0f, -2 * pe), poly.old = ldexpf(1.0f, -pe), poly.scale = ldexpf(1.0f, be);
    apply.p = b, apply.sp = square, apply.q = ys[k & 1], apply.sq = all, apply.steps = d.mp / kStep, apply.out = ys[~k & 1];
    apply.unscale = ldexpf(1.0f, -be - xe), apply.scale = ldexpf(1.0f, steps.x[k + 1]);
    launch_product<GRAM, float>(tri, g, Ends{}, d, u, st);
    launch_product<POLY, float>(tri, poly, Ends{}, d, u, st);
    if (k + 1 < steps.count)
      launch_product<APPLY, float>(tile, apply, Ends{}, d, u, st);
    else
      launch_product<LAST, T>(tile, apply, e, d, u, st);
  }
  if (steps.count == 0) k_ortho_end<T><<<dim3((unsigned)((size + 1023) / 1024), count), 256, 0, st>>>(e, d, u, y);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_orthogonalize(const OrthoArgs& a, void* workspace, hipStream_t st) {
  bool small;
  int tile = 0;
  const Sizes d = sizes_of(a.rows, a.cols, a.count, &small, &tile);
  const int batch = small ? kTable : batch_of(d, a.count);
  const Layout l = small ? Layout{} : layout_of(d, batch);
  Steps steps{};
  int xe[kOrthoMaxSteps + 1], pe[kOrthoMaxSteps], be[kOrthoMaxSteps];
  if (!ortho_bounds(a.steps, a.coef, xe, pe, be)) return hipErrorInvalidValue;
  steps.count = a.steps;
  for (int k = 0; k <= a.steps; ++k) {
    steps.x[k] = (signed char)xe[k];
    if (k == a.steps) break;
    steps.p[k] = (signed char)pe[k], steps.b[k] = (signed char)be[k];
    for (int c = 0; c < 3; ++c) steps.coef[k][c] = a.coef[3 * k + c];
  }
  const Update u{a.mu, a.eps, a.scale, a.decay, a.nesterov};
  for (int first = 0; first < a.count; first += batch) {
    const int count = a.count - first < batch ? a.count - first : batch;
    Table t{};
    Ends e{};
    for (int k = 0; k < count; ++k) {
      t.g[k] = a.grads[first + k];
      t.m[k] = a.moments ? a.moments[first + k] : nullptr;
      t.to[k] = a.moments ? a.news[first + k] : nullptr;
      e.w[k] = a.weights ? a.weights[first + k] : nullptr;
      e.out[k] = a.outs[first + k];
    }
    hipError_t err;
    if (small)
      err = a.grad_bf16 ? (a.bf16 ? launch_small<bf16_t, bf16_t> : launch_small<bf16_t, float>)(t, e, steps, d, u, count, st)
                        : (a.bf16 ? launch_small<float, bf16_t> : launch_small<float, float>)(t, e, steps, d, u, count, st);
    else
      err = (a.grad_bf16 ? (a.bf16 ? launch_large<bf16_t, bf16_t> : launch_large<bf16_t, float>)
                         : (a.bf16 ? launch_large<float, bf16_t> : launch_large<float, float>))(t, e, steps, d, u, tile, count, l,
                                                                                                (char*)workspace, st);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace e2f
