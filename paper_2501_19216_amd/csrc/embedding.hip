// Rows of a table by the types of atoms (of edges, of tokens), as the scalars of irrep features, and the table's
// gradient:
//   out[i][0][c] = s T[z_i][c],   out[i][k][c] = 0 for the components k >= 1,   0 for z_i outside of the table,
//   dT[v][c] = s sum over the i with z_i = v of g[i][0][c].
// The forward reads a row and writes one: memory.  The gradient sorts the rows by their types (a stable sort by
// digits of 8 bits, so that a type's rows keep their order) and sums them in stretches of the sorted order, as many
// rows each whatever the types are: a type that holds half of all rows costs no more than many small ones.  A stretch
// writes the sums of the types that begin and end in it; of one that goes on it keeps the part, and a last kernel
// adds a type's parts in their order and writes zeros for types without rows.  No float atomics: the same bits every
// time.
//
// 20,000 atoms of 100 types, L = 4, 128 channels: 51 us forward (256 MB at the rate of a copy; 34 where the last pass's
// rows are written over), 23 backward in five kernels of 4 to 8 us.  1.5 million rows of 64 bfloat16 channels of 100
// types: 60 us forward (41 over the last pass's rows), 81 backward, of which the sums 64 by themselves (192 MB of rows
// gathered at 3 TB/s, whatever the length of a stretch) and the sort 25.  16,384 tokens of 32,768 types, 1,024 bfloat16
// channels: 14 us forward (9 over the last pass's), 47 backward, of which 20 are the zeros of absent types.
//
// Times at the rules below are of whole gradients (at the forward's of forwards) on the same rows over and over, types
// as often as atoms have them.
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

// V neighbouring values, in pieces of up to 16 bytes
template <typename T, int V>
__device__ __forceinline__ void read_values(const T* p, float (&f)[V]) {
  constexpr int Q = V * sizeof(T) > 16 ? 16 / sizeof(T) : V;
#pragma unroll
  for (int u = 0; u < V; u += Q) {
    const auto v = Raw<T, Q>::load((const char*)(p + u));
#pragma unroll
    for (int k = 0; k < Q; ++k) f[u + k] = part(v, k);
  }
}
template <typename T, int V>
__device__ __forceinline__ void write_values(T* p, const float (&f)[V]) {
  constexpr int Q = V * sizeof(T) > 16 ? 16 / sizeof(T) : V;
#pragma unroll
  for (int u = 0; u < V; u += Q) {
    typename Raw<T, Q>::type v;
    join(f + u, v);
    Raw<T, Q>::store((char*)(p + u), v);
  }
}

// ------------------------------------------------------------------ forward
// tpr threads a row, each V neighbouring values at a time (V divides C: a row's scalars end between two of them); R
// rows of a thread, side by side with the others' rows, all their loads in flight together
template <typename TT, typename T, typename I, int V, int R>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a, const TT* __restrict__ table, T* __restrict__ out, int tpr) {
  const int slots = 256 / tpr, all = a.K * a.C;
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (slots * R) + threadIdx.x / tpr;
  int z[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = first + r * slots;
    z[r] = row < a.n ? type_of<I>(a.index, row, a.V) : a.V;
  }
  for (int o = threadIdx.x % tpr * V; o < all; o += tpr * V) {
    float f[R][V] = {};
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (o < a.C && z[r] < a.V) read_values(table + (int64_t)z[r] * a.C + o, f[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * slots;
      if (row >= a.n) continue;
#pragma unroll
      for (int u = 0; u < V; ++u) f[r][u] *= a.scale;
      write_values(out + row * a.ld + o, f[r]);
    }
  }
}

// ------------------------------------------------------------------ rows by type
// rows that one workgroup sorts (2,000 rows of 128 channels: 17.7 us, by many 18.9; 4,000 21.3 and 19.8; 7,680 28 and 20)
constexpr int kSmall = 2048;

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

// A workgroup's rows: R rounds of 64 for each of its four waves, neighbouring ones.  The type of lane's row of round r
template <typename I, int R>
__device__ __forceinline__ void read_types(const void* index, const int* keys, int n, int V, int64_t lo, int (&key)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t at = min(lo + r * 64 + (threadIdx.x & 63), (int64_t)n - 1);
    key[r] = keys ? keys[at] : type_of<I>(index, at, V);
  }
}

// Numbers of each digit in each workgroup's rows: counts [256][workgroups].  The first pass also clears the types'
// first rows
template <typename I, int R>
__global__ __launch_bounds__(256) void k_embed_count(const void* __restrict__ index, const int* __restrict__ keys, int n,
                                                     int V, int shift, int* __restrict__ counts, int* __restrict__ first) {
  __shared__ int have[256];
  if (first)
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < V; v += (int64_t)gridDim.x * 256) first[v] = -1;
  have[threadIdx.x] = 0;
  const int64_t lo = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (R * 64);
  int key[R];
  read_types<I, R>(index, keys, n, V, lo, key);
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (lo + r * 64 + (threadIdx.x & 63) < n) atomicAdd(&have[key[r] >> shift & 255], 1);  // (whole numbers: any order)
  __syncthreads();
  counts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = have[threadIdx.x];
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

// of each digit: the numbers before each workgroup (in place), and their total
__global__ __launch_bounds__(256) void k_embed_scan(int* __restrict__ counts, int groups, int* __restrict__ totals) {
  __shared__ int waves[4];
  int* row = counts + (int64_t)blockIdx.x * groups;
  int before = 0;
  for (int g0 = 0; g0 < groups; g0 += 1024) {
    const int g = g0 + threadIdx.x * 4;
    int v[4], t = 0, total;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = g + k < groups ? row[g + k] : 0, t += v[k];
    t = before + scan(t, waves, total);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (g + k < groups) row[g + k] = t;
      t += v[k];
    }
    before += total;
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

template <typename I, int R>
__global__ __launch_bounds__(256) void k_embed_scatter(const void* __restrict__ index, const int* __restrict__ keys,
                                                       const int* __restrict__ rows, int n, int V, int shift,
                                                       const int* __restrict__ counts, const int* __restrict__ totals,
                                                       int* __restrict__ keys_out, int* __restrict__ rows_out) {
  __shared__ int next[4][256], waves[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t lo = ((int64_t)blockIdx.x * 4 + wave) * (R * 64);
  int key[R], row[R], total;
  read_types<I, R>(index, keys, n, V, lo, key);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t at = lo + r * 64 + lane;
    row[r] = rows ? rows[min(at, (int64_t)n - 1)] : (int)at;
  }
  const int before = counts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x];
#pragma unroll
  for (int w = 0; w < 4; ++w) next[w][threadIdx.x] = 0;
  int base = scan(totals[threadIdx.x], waves, total) + before;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (lo + r * 64 + lane < n) atomicAdd(&next[wave][key[r] >> shift & 255], 1);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {  // (a thread a digit)
    const int v = next[w][threadIdx.x];
    next[w][threadIdx.x] = base;
    base += v;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (lo + r * 64 >= n) break;
    const bool on = lo + r * 64 + lane < n;
    const int d = key[r] >> shift & 255;
    const uint64_t m = same_digit(d, on);
    const int rank = below(m), to = next[wave][d] + rank;
    wave_sync();
    if (on) {
      keys_out[to] = key[r];
      rows_out[to] = row[r];
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
  int *first, *end;  // [V] first place of a type in the sorted order, or -1, and [V] one past its last
  float* part;  // [workgroups][2][C]: of the type that began before the workgroup's rows, of the one that goes on behind
  int per, wide;  // rows of a stretch, of a workgroup
};

// tpr threads a stretch, each V neighbouring channels; blocks of tpr V channels along y; a workgroup's stretches side
// by side, joined in the LDS: of the parts that go on from one to the next only the workgroup's own two are left
template <typename TT, typename T, int V>
__global__ __launch_bounds__(256) void k_embed_sums(EmbedArgs a, const T* __restrict__ g, Sorted s, TT* __restrict__ gt,
                                                    int tpr) {
  constexpr int U = 8;  // rows in flight
  __shared__ float part_of[2][256 * V];
  __shared__ int key_of[2][256];  // the type of a stretch's first part (-1: none), and where it ends there; of its last
  __shared__ bool ends[256];
  const int slots = 256 / tpr, slot = threadIdx.x / tpr, t = threadIdx.x % tpr;
  const int64_t start = (int64_t)blockIdx.x * s.wide, lo = min(start + (int64_t)slot * s.per, (int64_t)a.n);
  const int c = (blockIdx.y * tpr + t) * V;
  const bool on = c < a.C, lead = blockIdx.y == 0 && t == 0;
  const int at = on ? c : 0, hi = (int)min(lo + s.per, (int64_t)a.n);
  float sum[V] = {};
  int key = lo ? s.keys[lo - 1] : -1;  // of the running sum
  bool before = true;                  // it began before the stretch
  if (t == 0) key_of[0][slot] = key_of[1][slot] = -1;
  auto write = [&](int v) {
    float f[V];
#pragma unroll
    for (int u = 0; u < V; ++u) f[u] = sum[u] * a.scale;
    if (on) write_values(gt + (int64_t)v * a.C + at, f);
  };
  auto flush = [&](int p, int next) {  // the sum of `key` ends at place p (or the stretch does)
    const bool behind = p == hi && next == key;
    if (key >= 0 && key < a.V && (p > lo || !before)) {
      if (before || behind) {
        if (t == 0) {
          key_of[before ? 0 : 1][slot] = key;
          if (before) ends[slot] = !behind;
        }
#pragma unroll
        for (int u = 0; u < V; ++u) part_of[before ? 0 : 1][threadIdx.x * V + u] = sum[u];
      } else {
        write(key);
      }
    }
    if (lead && !behind && key >= 0 && key < a.V) s.end[key] = p;
#pragma unroll
    for (int u = 0; u < V; ++u) sum[u] = 0.0f;
  };
  for (int p = (int)lo; p < hi; p += U) {
    int k[U], row[U];
    typename Raw<T, V>::type v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(p + u, hi - 1);
      k[u] = s.keys[i], row[u] = s.rows[i];
    }
    // (rows outside of the table, the last ones, are read and their sum is dropped)
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = Raw<T, V>::load((const char*)(g + (int64_t)row[u] * a.ld + at));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u >= hi) break;
      if (k[u] != key) {
        flush(p + u, k[u]);
        key = k[u], before = false;
        if (lead && key < a.V) s.first[key] = p + u;
      }
#pragma unroll
      for (int x = 0; x < V; ++x) sum[x] += part(v[u], x);
    }
  }
  if (lo < hi) flush(hi, hi < a.n ? s.keys[hi] : -1);
  __syncthreads();
  if (slot) return;
  // the parts in their order, by the first stretch's threads
  int now = -1;
  before = true;
  auto store = [&]() {
    if (on) write_values(s.part + ((int64_t)blockIdx.x * 2 + (before ? 0 : 1)) * a.C + at, sum);
  };
#pragma unroll
  for (int u = 0; u < V; ++u) sum[u] = 0.0f;
  for (int w = 0; w < slots; ++w) {
    if (key_of[0][w] >= 0) {
      now = key_of[0][w];
#pragma unroll
      for (int u = 0; u < V; ++u) sum[u] += part_of[0][(w * tpr + t) * V + u];
      if (ends[w]) {
        if (before)
          store();
        else
          write(now);
        now = -1;
      }
    }
    if (key_of[1][w] >= 0) {
      now = key_of[1][w], before = false;
#pragma unroll
      for (int u = 0; u < V; ++u) sum[u] = part_of[1][(w * tpr + t) * V + u];
    }
  }
  if (now >= 0) store();
}

// What no workgroup held whole: zeros for a type without rows, and the parts of one that several workgroups hold, V
// channels a lane.  A wave takes up to kEach types, taken far apart (types that many rows have stand side by side in
// most numberings); where a type has more than kMany parts all threads of its workgroup add them, as many side by
// side as the channels leave room for.
// (kMany: 20,000 rows of 128 channels 20.8 us, with 8 20.8, with 128 24.4; 1.5 million of 64 bfloat16 ones 69.2, 69.9 and
// 73.0.  kEach: 20,000 rows of 2,000,000 types, 4 channels: one type a wave 867 us, two 665, eight 504, 32 486; 16,384 rows
// of 32,768 types, 1,024 channels: 55.2, 52.9, 53.1, 53.1)
constexpr int kMany = 32, kEach = 8;
template <typename TT, int V>
__global__ __launch_bounds__(1024) void k_embed_join(EmbedArgs a, Sorted s, TT* __restrict__ gt, unsigned apart, int each,
                                                     int tpr) {
  __shared__ float red[1024 * V];
  __shared__ int many[16 * kEach];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t group = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  auto add = [&](int c, int q, int q0, float (&sum)[V]) {
    float f[V];
    read_values(s.part + ((int64_t)q * 2 + (q == q0 ? 1 : 0)) * a.C + c, f);
#pragma unroll
    for (int u = 0; u < V; ++u) sum[u] += f[u];
  };
  auto put = [&](int c, int64_t v, float (&sum)[V]) {
#pragma unroll
    for (int u = 0; u < V; ++u) sum[u] *= a.scale;
    write_values(gt + v * a.C + c, sum);
  };
  // the ranges of the wave's `each` types, a lane one
  const int64_t mine = group + ((int64_t)lane * 16 + wave) * apart;
  const bool is = lane < each && group < apart && mine < a.V;
  const int first = is ? s.first[mine] : 0, end = is && first >= 0 ? s.end[mine] : 0;
  const int q0 = first < 0 ? 0 : first / s.wide, q1 = end > first ? (end - 1) / s.wide : q0;
  if (lane < each) many[lane * 16 + wave] = is && q1 - q0 >= kMany;
  const uint64_t todo = __ballot(is && (first < 0 || (q1 > q0 && q1 - q0 < kMany)));
  for (int k = 0; k < each; ++k) {
    if (!(todo >> k & 1)) continue;
    const int64_t v = group + ((int64_t)k * 16 + wave) * apart;
    const int f = __builtin_amdgcn_readlane(first, k), b = __builtin_amdgcn_readlane(q0, k), e = __builtin_amdgcn_readlane(q1, k);
    for (int c = (blockIdx.y * 64 + lane) * V; c < a.C; c += gridDim.y * 64 * V) {
      float sum[V] = {};
      if (f >= 0) {
#pragma unroll 4
        for (int q = b; q <= e; ++q) add(c, q, b, sum);
      }
      put(c, v, sum);
    }
  }
  __syncthreads();
  const int slots = 1024 / tpr, slot = threadIdx.x / tpr, t = threadIdx.x % tpr;
  for (int w = 0; w < 16 * each; ++w) {
    if (!many[w]) continue;
    const int64_t type = group + (int64_t)w * apart;
    const int b = s.first[type] / s.wide, e = (s.end[type] - 1) / s.wide;
    for (int c0 = blockIdx.y * tpr * V; c0 < a.C; c0 += gridDim.y * tpr * V) {
      const int c = c0 + t * V;
      float sum[V] = {};
      if (c < a.C) {
#pragma unroll 4
        for (int q = b + slot; q <= e; q += slots) add(c, q, b, sum);
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < V; ++u) red[threadIdx.x * V + u] = sum[u];
      // halves of the threads, a fixed order
      for (int k = slots >> 1; k > 0; k >>= 1) {
        __syncthreads();
        if (slot < k) {
#pragma unroll
          for (int u = 0; u < V; ++u) sum[u] += red[(threadIdx.x + k * tpr) * V + u], red[threadIdx.x * V + u] = sum[u];
        }
      }
      if (slot == 0 && c < a.C) put(c, type, sum);
      __syncthreads();
    }
  }
}

int pieces_of(int C, bool bf16) {  // values of a thread: 16 bytes of the narrower type, as far as they divide C
  int V = bf16 ? 8 : 4;
  while (C % V) V >>= 1;
  return V;
}

int lanes_of(int C, int V) {
  int tpr = 1;
  while (tpr < 64 && tpr < C / V) tpr <<= 1;
  return tpr;
}

struct Layout {
  int passes, rounds, groups, tpr, per, wide, blocks;
  size_t keys[2], rows[2], counts, totals, range, part, total;
};
Layout layout_of(int n, int V, int C, bool bf16) {
  Layout l{};
  l.passes = 1;
  while (l.passes < 4 && (uint64_t)V >> (8 * l.passes)) ++l.passes;  // (types 0 .. V)
  // rounds of 64 rows a wave of the sort: up to 512 workgroups with one, then up to 2,048 with four, then 16 (130,000 rows
  // of 64 bfloat16 channels: one 27.8 us, four 28.3, 16 37.5; 262,144 rows 36.0, 33.8, 45.1; 1.5 million 86.7, 69.6, 76.7;
  // six million of 16 channels 290, 212, 200)
  l.rounds = n <= 1 << 17 ? 1 : n <= 1 << 21 ? 4 : 16;
  l.groups = (int)(((int64_t)n + 256 * l.rounds - 1) / (256 * l.rounds));
  // rows of a stretch: 8 (all in flight) until the workgroups are 2,048, then up to 64 (20,000 rows of 128 channels: 8
  // rows 20.8 us, 16 20.9, 32 22.1, 64 24.4; 400,000 of 64 bfloat16 ones 40.0, 39.2, 38.0, 39.8; 1.5 million 76.5, 70.2,
  // 69.2, 70.0)
  const int Q = pieces_of(C, bf16);
  l.tpr = lanes_of(C, Q);
  const int columns = (C / Q + l.tpr - 1) / l.tpr;
  l.per = 8;
  while (l.per < 64 && (int64_t)n * columns / ((int64_t)l.per * (256 / l.tpr)) > 2048) l.per <<= 1;
  l.wide = l.per * (256 / l.tpr);
  l.blocks = (int)(((int64_t)n + l.wide - 1) / l.wide);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) & ~size_t(255);
    return was;
  };
  for (int k = 0; k < 2; ++k) l.keys[k] = take(sizeof(int) * (size_t)n), l.rows[k] = take(sizeof(int) * (size_t)n);
  if (n > kSmall) l.counts = take(sizeof(int) * 256 * (size_t)l.groups), l.totals = take(sizeof(int) * 256);
  l.range = take(sizeof(int) * 2 * (size_t)V);
  l.part = take(sizeof(float) * 2 * (size_t)l.blocks * C);
  l.total = at;
  return l;
}

}  // namespace

size_t embed_workspace(int n, int V, int C, bool bf16) { return layout_of(n, V, C, bf16).total; }

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
  const int V = pieces_of(a.C, a.bf16);
  const int64_t pieces = (int64_t)a.K * a.C / V;
  int tpr = 1;
  while (tpr < 64 && tpr < pieces) tpr <<= 1;
  // four rows a thread where a row is one round of its threads and there are enough to fill the GPU (64 bfloat16
  // channels: 60,000 rows 4.6 us with one, 5.2 with four; 262,144 10.0 and 10.4; 1.5 million 39.6 and 35.0)
  const bool four = pieces <= 64 && (int64_t)a.n * tpr > 1 << 20;
  const int64_t rows = 256 / tpr * (four ? 4 : 1);
  const Rounds r = rounds_of(((int64_t)a.n + rows - 1) / rows, 256);
  const dim3 grid(r.x, r.rounds);
#define E2F_EMBED_R(TT, T, I, VV)                                                                  \
  four ? k_embed<TT, T, I, VV, 4><<<grid, 256, 0, st>>>(a, (const TT*)table, (T*)out, tpr)         \
       : k_embed<TT, T, I, VV, 1><<<grid, 256, 0, st>>>(a, (const TT*)table, (T*)out, tpr)
#define E2F_EMBED(TT, T, VV)                 \
  if (a.wide)                                \
    E2F_EMBED_R(TT, T, int64_t, VV);         \
  else                                       \
    E2F_EMBED_R(TT, T, int32_t, VV)
  if (a.table_bf16 && a.bf16) {
    E2F_EMBED_V(bf16_t, bf16_t)
  } else if (a.table_bf16) {
    E2F_EMBED_V4(bf16_t, float)
  } else if (a.bf16) {
    E2F_EMBED_V(float, bf16_t)
  } else {
    E2F_EMBED_V4(float, float)
  }
#undef E2F_EMBED
#undef E2F_EMBED_R
  return hipGetLastError();
}

template <typename I, int R>
void sort_pass(const EmbedArgs& a, const Layout& l, const int* k, const int* r, int shift, int* counts, int* totals,
               int* first, int* keys, int* rows, hipStream_t st) {
  k_embed_count<I, R><<<l.groups, 256, 0, st>>>(a.index, k, a.n, a.V, shift, counts, first);
  k_embed_scan<<<256, 256, 0, st>>>(counts, l.groups, totals);
  k_embed_scatter<I, R><<<l.groups, 256, 0, st>>>(a.index, k, r, a.n, a.V, shift, counts, totals, keys, rows);
}

hipError_t launch_embed_backward(const EmbedArgs& a, const void* gout, void* gtable, void* workspace, hipStream_t st) {
  const Layout l = layout_of(a.n, a.V, a.C, a.bf16);
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
    for (int p = 0; p < l.passes; ++p, now ^= 1) {
      const int *k = p ? keys[now] : nullptr, *r = p ? rows[now] : nullptr;
      int* first = p ? nullptr : range;
      auto pass = a.wide ? (l.rounds == 1 ? sort_pass<int64_t, 1> : l.rounds == 4 ? sort_pass<int64_t, 4> : sort_pass<int64_t, 16>)
                         : (l.rounds == 1 ? sort_pass<int32_t, 1> : l.rounds == 4 ? sort_pass<int32_t, 4> : sort_pass<int32_t, 16>);
      pass(a, l, k, r, 8 * p, counts, totals, first, keys[now ^ 1], rows[now ^ 1], st);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const Sorted s{keys[now], rows[now], range, range + a.V, (float*)(ws + l.part), l.per, l.wide};
  if (a.n) {
    const int V = pieces_of(a.C, a.bf16);
    const dim3 grid(l.blocks, (unsigned)((a.C / V + l.tpr - 1) / l.tpr));
#define E2F_EMBED(TT, T, VV) k_embed_sums<TT, T, VV><<<grid, 256, 0, st>>>(a, (const T*)gout, s, (TT*)gtable, l.tpr)
    if (a.table_bf16 && a.bf16) {
      E2F_EMBED_V(bf16_t, bf16_t)
    } else if (a.table_bf16) {
      E2F_EMBED_V4(bf16_t, float)
    } else if (a.bf16) {
      E2F_EMBED_V(float, bf16_t)
    } else {
      E2F_EMBED_V4(float, float)
    }
#undef E2F_EMBED
  }
  // (the table's type alone: the parts are float)
  const int V = pieces_of(a.C, a.table_bf16), tpr = lanes_of(a.C, V), columns = (a.C / V + 63) / 64;
  // types of a wave: as many workgroups as the GPU holds at once, where there are that many types; where there are
  // fewer, a type's channels side by side as well (1,024 channels: 2,000 rows of 200 types 16.0 us, one after the other
  // 18.2; 20,000 of 4,000 types 44.2 and 41.9; but 16,384 of 32,768 types 69.2 and 53.1)
  int each = 1;
  while (each < kEach && a.V / (16 * each) > 512) each <<= 1;
  const unsigned apart = ((unsigned)a.V + 16 * each - 1) / (16 * each);
  const Rounds r = rounds_of(apart, 1024);
  const dim3 grid(r.x, apart < 512 ? columns : 1, r.rounds);
#define E2F_EMBED(TT, T, VV) k_embed_join<TT, VV><<<grid, 1024, 0, st>>>(a, s, (TT*)gtable, apart, each, tpr)
  if (a.table_bf16) {
    E2F_EMBED_V(bf16_t, float)
  } else {
    E2F_EMBED_V4(float, float)
  }
#undef E2F_EMBED
  return hipGetLastError();
}

}  // namespace e2f
