// Rows of a table by the types of atoms (of edges, of tokens), as the scalars of irrep features, and the table's gradient:
//   out[i][0][c] = s T[z_i][c],   out[i][k][c] = 0 for the components k >= 1,   0 for z_i outside of the table,
//   dT[v][c] = s sum over the i with z_i = v of g[i][0][c].
// The forward reads a row and writes one: memory.  The gradient sorts the rows by their types (a stable sort by digits of 8
// bits, so that a type's rows keep their order) and sums them in stretches of the sorted order, as many rows each whatever
// the types are: a type that holds half of all rows costs no more than many small ones.  A stretch writes the sums of the
// types that begin and end in it; of one that goes on it keeps the part, and a last kernel adds a type's parts in
// their order and writes zeros for types without rows.  No atomics: the same bits every time.
#include <hip/hip_runtime.h>

#include "e2f_launch.h"
#include "values.h"
#include "wave.h"

namespace e2f {
namespace {

// the type of row i, V (behind the table) for those outside of it
template <typename I>
__device__ __forceinline__ int type_of(const void* index, int64_t i, int V) {
  const I z = ((const I*)index)[i];
  return z >= 0 && z < (I)V ? (int)z : V;
}

// ------------------------------------------------------------------ forward
// tpr threads a row, each V neighbouring values at a time (V divides C: a row's scalars end between two of them)
template <typename TT, typename T, typename I, int V>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a, const TT* __restrict__ table, T* __restrict__ out, int tpr) {
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / tpr) + threadIdx.x / tpr;
  if (row >= a.n) return;
  const int z = type_of<I>(a.index, row, a.V);
  T* to = out + row * a.ld;
  const TT* from = table + (int64_t)z * a.C;
  const int all = a.K * a.C, scalars = z < a.V ? a.C : 0;
  for (int o = threadIdx.x % tpr * V; o < all; o += tpr * V) {
    float f[V] = {};
    if (o < scalars) {
      const auto v = Raw<TT, V>::load((const char*)(from + o));
#pragma unroll
      for (int u = 0; u < V; ++u) f[u] = part(v, u) * a.scale;
    }
    typename Raw<T, V>::type v;
    join(f, v);
    Raw<T, V>::store((char*)(to + o), v);
  }
}

// ------------------------------------------------------------------ rows by type
constexpr int kSegments = 1024;  // waves that sort, at most: each a stretch of neighbouring rows
constexpr int kSmall = 8192;     // rows that one workgroup sorts

// what lanes of this wave wrote to the LDS is there for its other lanes
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// lanes of the wave with this lane's digit, among those that are on
__device__ __forceinline__ uint64_t same_digit(int d, bool on) {
  uint64_t m = __ballot(on);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint64_t s = __ballot(on && (d >> b & 1));
    m &= d >> b & 1 ? s : ~s;
  }
  return m;
}
__device__ __forceinline__ int below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}

// Numbers of each digit in each wave's rows: counts [256][segments].  The first pass also clears the types' first rows
template <typename I>
__global__ __launch_bounds__(256) void k_embed_count(const void* __restrict__ index, const int* __restrict__ keys, int n,
                                                     int V, int shift, int per, int segments, int* __restrict__ counts,
                                                     int* __restrict__ first) {
  __shared__ int have[4][256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, seg = blockIdx.x * 4 + wave;
  if (first)
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < V; v += (int64_t)gridDim.x * 256) first[v] = -1;
  for (int d = lane; d < 256; d += 64) have[wave][d] = 0;
  wave_sync();
  const int64_t lo = (int64_t)seg * per, hi = min(lo + per, (int64_t)n);
  for (int64_t i = lo; i < hi; i += 64) {
    const bool on = i + lane < hi;
    const int64_t at = min(i + lane, hi - 1);
    const int d = (keys ? keys[at] : type_of<I>(index, at, V)) >> shift & 255;
    const uint64_t m = same_digit(d, on);
    if (on && below(m) == 0) have[wave][d] += __popcll(m);
    wave_sync();
  }
  if (seg < segments)
    for (int d = lane; d < 256; d += 64) counts[d * segments + seg] = have[wave][d];
}

// Sums of a workgroup's threads before each, and of all
__device__ __forceinline__ int scan(int v, int* waves, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(s, o);
    if (lane >= o) s += t;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < nw; ++w) {
    if (w < wave) before += waves[w];
    total += waves[w];
  }
  return before + s - v;
}

// of each digit: the numbers before each segment (in place), and their total; segments <= 1024
__global__ __launch_bounds__(256) void k_embed_scan(int* __restrict__ counts, int segments, int* __restrict__ totals) {
  __shared__ int waves[4];
  int* row = counts + blockIdx.x * segments;
  const int s0 = threadIdx.x * 4;
  int v[4], t = 0, total;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = s0 + k < segments ? row[s0 + k] : 0, t += v[k];
  t = scan(t, waves, total);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (s0 + k < segments) row[s0 + k] = t;
    t += v[k];
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = total;
}

template <typename I>
__global__ __launch_bounds__(256) void k_embed_scatter(const void* __restrict__ index, const int* __restrict__ keys,
                                                       const int* __restrict__ rows, int n, int V, int shift, int per,
                                                       int segments, const int* __restrict__ counts,
                                                       const int* __restrict__ totals, int* __restrict__ keys_out,
                                                       int* __restrict__ rows_out) {
  __shared__ int next[4][256], base[256], waves[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, seg = blockIdx.x * 4 + wave;
  int total;
  base[threadIdx.x] = scan(totals[threadIdx.x], waves, total);
  __syncthreads();
  if (seg < segments)
    for (int d = lane; d < 256; d += 64) next[wave][d] = base[d] + counts[d * segments + seg];
  wave_sync();
  const int64_t lo = (int64_t)seg * per, hi = min(lo + per, (int64_t)n);
  for (int64_t i = lo; i < hi; i += 64) {
    const bool on = i + lane < hi;
    const int64_t at = min(i + lane, hi - 1);
    const int key = keys ? keys[at] : type_of<I>(index, at, V), d = key >> shift & 255;
    const uint64_t m = same_digit(d, on);
    const int rank = below(m), to = next[wave][d] + rank;
    wave_sync();
    if (on) {
      keys_out[to] = key;
      rows_out[to] = rows ? rows[at] : (int)at;
      if (rank == 0) next[wave][d] = to + __popcll(m);
    }
    wave_sync();
  }
}

// All passes of up to kSmall rows in one workgroup's LDS: 16 waves, a stretch of neighbouring rows each
template <typename I>
__global__ __launch_bounds__(1024) void k_embed_sort(const void* __restrict__ index, int n, int V, int passes,
                                                     int* __restrict__ keys_out, int* __restrict__ rows_out,
                                                     int* __restrict__ first) {
  __shared__ int key[2][kSmall], waves[16];
  __shared__ unsigned short row[2][kSmall];
  __shared__ int next[16][256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int64_t v = threadIdx.x; v < V; v += 1024) first[v] = -1;
  for (int i = threadIdx.x; i < n; i += 1024) key[0][i] = type_of<I>(index, i, V), row[0][i] = (unsigned short)i;
  const int per = ((n + 15) / 16 + 63) / 64 * 64, lo = min(wave * per, n), hi = min(lo + per, n);
  for (int p = 0; p < passes; ++p) {
    const int* k0 = key[p & 1];
    const unsigned short* r0 = row[p & 1];
    for (int d = lane; d < 256; d += 64) next[wave][d] = 0;
    __syncthreads();
    for (int i = lo; i < hi; i += 64) {
      const bool on = i + lane < hi;
      const int d = k0[min(i + lane, hi - 1)] >> (8 * p) & 255;
      const uint64_t m = same_digit(d, on);
      if (on && below(m) == 0) next[wave][d] += __popcll(m);
      wave_sync();
    }
    __syncthreads();
    // places by digit, then by wave: four threads a digit, four waves each
    int c[4], t = 0, total;
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = next[(threadIdx.x & 3) * 4 + k][threadIdx.x >> 2], t += c[k];
    t = scan(t, waves, total);
#pragma unroll
    for (int k = 0; k < 4; ++k) next[(threadIdx.x & 3) * 4 + k][threadIdx.x >> 2] = t, t += c[k];
    __syncthreads();
    for (int i = lo; i < hi; i += 64) {
      const bool on = i + lane < hi;
      const int at = min(i + lane, hi - 1), k = k0[at], d = k >> (8 * p) & 255;
      const uint64_t m = same_digit(d, on);
      const int rank = below(m), to = next[wave][d] + rank;
      wave_sync();
      if (on) {
        key[~p & 1][to] = k, row[~p & 1][to] = r0[at];
        if (rank == 0) next[wave][d] = to + __popcll(m);
      }
      wave_sync();
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n; i += 1024) keys_out[i] = key[passes & 1][i], rows_out[i] = row[passes & 1][i];
}

// ------------------------------------------------------------------ sums
struct Sorted {
  const int *keys, *rows;
  int* range;   // [V] first place of a type in the sorted order, or -1, then [V] one past its last
  float* part;  // [stretches][2][C]: of the type that began before the stretch, of the one that goes on behind it
  int per, stretches;
};

// tpr threads a stretch, each V neighbouring channels; blocks of tpr V channels along y
template <typename TT, typename T, int V>
__global__ __launch_bounds__(256) void k_embed_sums(EmbedArgs a, const T* __restrict__ g, Sorted s, TT* __restrict__ gt,
                                                    int tpr) {
  constexpr int U = 8;  // rows in flight
  const int64_t q = (int64_t)blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
  if (q >= s.stretches) return;
  const int c = (blockIdx.y * tpr + threadIdx.x % tpr) * V;
  const bool on = c < a.C;
  const int at = on ? c : 0;
  const bool lead = blockIdx.y == 0 && threadIdx.x % tpr == 0;
  const int64_t lo = q * s.per;
  const int hi = (int)min(lo + s.per, (int64_t)a.n);
  float sum[V] = {};
  int key = lo ? s.keys[lo - 1] : -1;  // of the running sum
  bool before = true;                  // it began before the stretch
  auto flush = [&](int p, int next) {  // the sum of `key` ends at place p (or the stretch does)
    const bool behind = p == hi && next == key;
    if (key >= 0 && key < a.V && (p > lo || !before)) {
      if (before || behind) {
        float* to = s.part + (q * 2 + (before ? 0 : 1)) * a.C + at;
        if (on) Raw<float, V>::store((char*)to, [&] { typename Raw<float, V>::type v; join(sum, v); return v; }());
      } else if (on) {
        float f[V];
#pragma unroll
        for (int u = 0; u < V; ++u) f[u] = sum[u] * a.scale;
        typename Raw<TT, V>::type v;
        join(f, v);
        Raw<TT, V>::store((char*)(gt + (int64_t)key * a.C + at), v);
      }
    }
    if (lead && !behind && key >= 0 && key < a.V) s.range[a.V + key] = p;
#pragma unroll
    for (int u = 0; u < V; ++u) sum[u] = 0.0f;
  };
  for (int p = (int)lo; p < hi; p += U) {
    int k[U];
    typename Raw<T, V>::type v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(p + u, hi - 1);
      k[u] = s.keys[i];
      v[u] = Raw<T, V>::load((const char*)(g + (int64_t)s.rows[i] * a.ld + at));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u >= hi) break;
      if (k[u] != key) {
        flush(p + u, k[u]);
        key = k[u], before = false;
        if (lead && key < a.V) s.range[key] = p + u;
      }
#pragma unroll
      for (int x = 0; x < V; ++x) sum[x] += part(v[u], x);
    }
  }
  flush(hi, hi < a.n ? s.keys[hi] : -1);
}

// What no stretch held whole: a workgroup a type and 64 channels, the parts of its stretches in 16 interleaved sums
template <typename TT>
__global__ __launch_bounds__(1024) void k_embed_join(EmbedArgs a, Sorted s, TT* __restrict__ gt) {
  __shared__ float red[16][64];
  const int64_t v = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (v >= a.V) return;
  const int first = s.range[v], end = first < 0 ? 0 : s.range[a.V + v];
  const int q0 = first / s.per, q1 = first < 0 ? 0 : (end - 1) / s.per;
  if (first >= 0 && q0 == q1) return;
  const int slot = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int c0 = blockIdx.z * 64; c0 < a.C; c0 += gridDim.z * 64) {
    const int c = c0 + lane;
    float sum = 0.0f;
    if (first >= 0 && c < a.C)
      for (int q = q0 + slot; q <= q1; q += 16) sum += s.part[((int64_t)q * 2 + (q == q0 ? 1 : 0)) * a.C + c];
    __syncthreads();
    red[slot][lane] = sum;
    __syncthreads();
    if (slot || c >= a.C) continue;
    for (int k = 1; k < 16; ++k) sum += red[k][lane];
    const float f[1] = {first < 0 ? 0.0f : sum * a.scale};
    typename Raw<TT, 1>::type w;
    join(f, w);
    Raw<TT, 1>::store((char*)(gt + v * a.C + c), w);
  }
}

int pieces_of(int C, bool bf16) {  // values of a thread: 16 bytes of the narrower type, as far as they divide C
  int V = bf16 ? 8 : 4;
  while (C % V) V >>= 1;
  return V;
}

struct Layout {
  int passes, per_wave, segments, per, stretches;
  size_t keys[2], rows[2], counts, totals, range, part, total;
};
Layout layout_of(int n, int V, int C) {
  Layout l{};
  l.passes = 1;
  while (l.passes < 4 && (uint64_t)V >> (8 * l.passes)) ++l.passes;  // (types 0 .. V)
  l.per_wave = (int)(((int64_t)n + kSegments - 1) / kSegments + 63) / 64 * 64;
  if (l.per_wave < 64) l.per_wave = 64;
  l.segments = (int)(((int64_t)n + l.per_wave - 1) / l.per_wave);
  // rows of a stretch: enough stretches to fill the GPU
  l.per = 16;
  while (l.per < 256 && (int64_t)n * ((C + 255) / 256) / l.per > 8192) l.per <<= 1;
  l.stretches = (int)(((int64_t)n + l.per - 1) / l.per);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) & ~size_t(255);
    return was;
  };
  for (int k = 0; k < 2; ++k) l.keys[k] = take(sizeof(int) * (size_t)n), l.rows[k] = take(sizeof(int) * (size_t)n);
  l.counts = take(sizeof(int) * 256 * (size_t)l.segments);
  l.totals = take(sizeof(int) * 256);
  l.range = take(sizeof(int) * 2 * (size_t)V);
  l.part = take(sizeof(float) * 2 * (size_t)l.stretches * C);
  l.total = at;
  return l;
}

}  // namespace

size_t embed_workspace(int n, int V, int C) { return layout_of(n, V, C).total; }

#define E2F_EMBED_V(TT, T)                    \
  switch (V) {                                \
    case 8: E2F_EMBED(TT, T, 8); break;       \
    case 4: E2F_EMBED(TT, T, 4); break;       \
    case 2: E2F_EMBED(TT, T, 2); break;       \
    default: E2F_EMBED(TT, T, 1);             \
  }
#define E2F_EMBED_V4(TT, T)                   \
  switch (V) {                                \
    case 4: E2F_EMBED(TT, T, 4); break;       \
    case 2: E2F_EMBED(TT, T, 2); break;       \
    default: E2F_EMBED(TT, T, 1);             \
  }

hipError_t launch_embed_forward(const EmbedArgs& a, const void* table, void* out, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const int V = pieces_of(a.C, a.table_bf16 && a.bf16);
  const int64_t pieces = (int64_t)a.K * a.C / V;
  int tpr = 1;
  while (tpr < 64 && tpr < pieces) tpr <<= 1;
  const Rounds r = rounds_of(((int64_t)a.n + 256 / tpr - 1) / (256 / tpr), 256);
  const dim3 grid(r.x, r.rounds);
#define E2F_EMBED(TT, T, VV)                                                                               \
  a.wide ? k_embed<TT, T, int64_t, VV><<<grid, 256, 0, st>>>(a, (const TT*)table, (T*)out, tpr)            \
         : k_embed<TT, T, int32_t, VV><<<grid, 256, 0, st>>>(a, (const TT*)table, (T*)out, tpr)
  if (a.table_bf16 && a.bf16) {
    E2F_EMBED_V(bf16_t, bf16_t)
  } else if (a.table_bf16) {
    E2F_EMBED_V4(bf16_t, float)
  } else if (a.bf16) {
    E2F_EMBED_V4(float, bf16_t)
  } else {
    E2F_EMBED_V4(float, float)
  }
#undef E2F_EMBED
  return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedArgs& a, const void* gout, void* gtable, void* workspace, hipStream_t st) {
  const Layout l = layout_of(a.n, a.V, a.C);
  char* ws = (char*)workspace;
  int *keys[2] = {(int*)(ws + l.keys[0]), (int*)(ws + l.keys[1])}, *rows[2] = {(int*)(ws + l.rows[0]), (int*)(ws + l.rows[1])};
  int *counts = (int*)(ws + l.counts), *totals = (int*)(ws + l.totals), *range = (int*)(ws + l.range);
  int now = 0;
  if (a.n <= kSmall) {
    if (a.wide)
      k_embed_sort<int64_t><<<1, 1024, 0, st>>>(a.index, a.n, a.V, l.passes, keys[0], rows[0], range);
    else
      k_embed_sort<int32_t><<<1, 1024, 0, st>>>(a.index, a.n, a.V, l.passes, keys[0], rows[0], range);
  } else {
    const int blocks = (l.segments + 3) / 4;
    for (int p = 0; p < l.passes; ++p, now ^= 1) {
      const int *k = p ? keys[now] : nullptr, *r = p ? rows[now] : nullptr;
      int* first = p ? nullptr : range;
      if (a.wide) {
        k_embed_count<int64_t><<<blocks, 256, 0, st>>>(a.index, k, a.n, a.V, 8 * p, l.per_wave, l.segments, counts, first);
        k_embed_scan<<<256, 256, 0, st>>>(counts, l.segments, totals);
        k_embed_scatter<int64_t><<<blocks, 256, 0, st>>>(a.index, k, r, a.n, a.V, 8 * p, l.per_wave, l.segments, counts,
                                                         totals, keys[now ^ 1], rows[now ^ 1]);
      } else {
        k_embed_count<int32_t><<<blocks, 256, 0, st>>>(a.index, k, a.n, a.V, 8 * p, l.per_wave, l.segments, counts, first);
        k_embed_scan<<<256, 256, 0, st>>>(counts, l.segments, totals);
        k_embed_scatter<int32_t><<<blocks, 256, 0, st>>>(a.index, k, r, a.n, a.V, 8 * p, l.per_wave, l.segments, counts,
                                                         totals, keys[now ^ 1], rows[now ^ 1]);
      }
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const Sorted s{keys[now], rows[now], range, (float*)(ws + l.part), l.per, l.stretches};
  if (a.n) {
    const int V = pieces_of(a.C, false);
    int tpr = 1;
    while (tpr < 64 && tpr < a.C / V) tpr <<= 1;
    const dim3 grid((unsigned)(((int64_t)l.stretches + 256 / tpr - 1) / (256 / tpr)), (unsigned)((a.C / V + tpr - 1) / tpr));
#define E2F_EMBED(TT, T, VV) k_embed_sums<TT, T, VV><<<grid, 256, 0, st>>>(a, (const T*)gout, s, (TT*)gtable, tpr)
    if (a.table_bf16 && a.bf16) {
      E2F_EMBED_V4(bf16_t, bf16_t)
    } else if (a.table_bf16) {
      E2F_EMBED_V4(bf16_t, float)
    } else if (a.bf16) {
      E2F_EMBED_V4(float, bf16_t)
    } else {
      E2F_EMBED_V4(float, float)
    }
#undef E2F_EMBED
  }
  const Rounds r = rounds_of(a.V, 1024);
  const int columns = (a.C + 63) / 64;
  const dim3 grid(r.x, r.rounds, a.V < 4096 ? columns : 1);
  if (a.table_bf16)
    k_embed_join<bf16_t><<<grid, 1024, 0, st>>>(a, s, (bf16_t*)gtable);
  else
    k_embed_join<float><<<grid, 1024, 0, st>>>(a, s, (float*)gtable);
  return hipGetLastError();
}

}  // namespace e2f
