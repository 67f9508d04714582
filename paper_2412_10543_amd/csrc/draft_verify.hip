// Verification of drafted tokens against the model's logits, from given random
// numbers (gfx950).
//
// Node i of a sequence has the logits of what follows it; p_i = softmax(logits / T).
//   without the drafter's probabilities (trees, chains): a token is drawn at every node,
//     t_i = the first index whose running sum of p_i exceeds u_i (T = 0: the first of
//     the largest logits); from node 0 the walk goes to the child whose token is t_i;
//   with them (chains): node i >= 1 is accepted where u_i q_i(x_i) < p_{i-1}(x_i); behind
//     the first that is not, the next token is drawn from max(p - q, 0), or from the last
//     node's p where all are accepted, with u_0.
//
// A draw by running sums turns on the sum of everything before the drawn token: with
// 128,000 likely tokens, sums in fp32 would move one draw in ten.  Exponentials and sums
// are therefore fp64 (the vector units' rate for it is that of fp32), and the exponential
// is its power series, 2^x = 2^n sum (x - n)^k ln2^k / k!, |x - n| <= 1/2, to k = 11
// (2^-47 relative).
//
// HBM-bound by the logits, which are read once: a workgroup takes kVChunk of a row and
// leaves its maximum and sum; the last workgroup of a row to finish places the draw in a
// chunk and reads that chunk again; the last row of a sequence walks.  With the
// drafter's probabilities a second launch sums max(p - q, 0) for the one row a sequence.
#include "common.h"
#include "serve.h"

#include <climits>
#include <algorithm>

namespace rag {

namespace {

constexpr int kVThreads = 256, kVWaves = kVThreads / kWave;
constexpr int kVPer = 16;                       // logits of a thread
constexpr int kVChunk = kVThreads * kVPer;
constexpr int kVCounters = kVerifyMaxRows + 2 * kVerifyMaxSeqs;

// A chunk's maximum, sum of exp((x - maximum) / T) and first index of the maximum.
struct VStat {
  double sum;
  float top;
  int arg;
};
// A row's.
struct VRow {
  double total;                 // sum of exp((x - top) / T)
  float top;
  int token;                    // drawn, or the first of the largest; with drafts: the latter
  int accept;                   // with drafts: whether the next node is accepted
  int pad;
};

struct VWs {
  int* rows;                    // [kVerifyMaxRows] arrivals
  int* seqs;                    // [2][kVerifyMaxSeqs]
  VStat* stats;                 // [num_rows][chunks]
  VRow* row;                    // [num_rows]
  double* rest;                 // [num_seqs][chunks]
};

__host__ __device__ __forceinline__ int verify_chunks(int vocab) {
  return (int)(((int64_t)vocab + kVChunk - 1) / kVChunk);
}

__host__ __device__ __forceinline__ size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

__host__ __device__ __forceinline__ VWs verify_ws(char* base, int num_rows, int vocab) {
  VWs w;
  const size_t chunks = (size_t)verify_chunks(vocab);
  w.rows = reinterpret_cast<int*>(base);
  w.seqs = w.rows + kVerifyMaxRows;
  base += up256(kVCounters * sizeof(int));
  w.stats = reinterpret_cast<VStat*>(base);
  base += up256(num_rows * chunks * sizeof(VStat));
  w.row = reinterpret_cast<VRow*>(base);
  base += up256(num_rows * sizeof(VRow));
  w.rest = reinterpret_cast<double*>(base);
  return w;
}

// ---- values that another XCD reads -------------------------------------------------
template <class T>
__device__ __forceinline__ void put(T* p, const T& v) {
  static_assert(sizeof(T) % 8 == 0, "8-byte pieces");
  uint64_t x[sizeof(T) / 8];
  __builtin_memcpy(x, &v, sizeof(T));
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 8; ++i)
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p) + i, x[i], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T get(const T* p) {
  uint64_t x[sizeof(T) / 8];
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 8; ++i)
    x[i] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p) + i, __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
  T v;
  __builtin_memcpy(&v, x, sizeof(T));
  return v;
}

// 2^x for x <= 0 (and rounding above it); below -1100, and for NaN, 0.
__device__ __forceinline__ double exp2_f64(double x) {
  x = __builtin_fmax(x, -1100.0);
  const double n = __builtin_rint(x), f = x - n;
  constexpr double kL = 0.69314718055994530942;
  double r = 1.0;
  constexpr double c1 = kL, c2 = c1 * kL / 2, c3 = c2 * kL / 3, c4 = c3 * kL / 4, c5 = c4 * kL / 5,
                   c6 = c5 * kL / 6, c7 = c6 * kL / 7, c8 = c7 * kL / 8, c9 = c8 * kL / 9,
                   c10 = c9 * kL / 10, c11 = c10 * kL / 11;
  r = __builtin_fma(c11, f, c10);
  r = __builtin_fma(r, f, c9);
  r = __builtin_fma(r, f, c8);
  r = __builtin_fma(r, f, c7);
  r = __builtin_fma(r, f, c6);
  r = __builtin_fma(r, f, c5);
  r = __builtin_fma(r, f, c4);
  r = __builtin_fma(r, f, c3);
  r = __builtin_fma(r, f, c2);
  r = __builtin_fma(r, f, c1);
  r = __builtin_fma(r, f, 1.0);
  return __builtin_ldexp(r, (int)n);
}

// exp((x - top) / T), k = log2(e) / T; NaN and what lies at or below -inf count 0.
__device__ __forceinline__ double weight(float x, float top, double k) {
  return exp2_f64(((double)x - (double)top) * k);
}

// Eight logits of a row from element e on; -inf behind its end.  Rows may start at any
// element: the loads are of 16 bytes at any even address.
struct __attribute__((packed, aligned(2))) Any16 { u32x4 v; };
struct __attribute__((packed, aligned(4))) Any16f { f32x4 v; };

template <bool kWide>
__device__ __forceinline__ void load8(const void* row, int e, int vocab, float (&x)[8]) {
  if (e + 8 <= vocab) {
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 y = reinterpret_cast<const Any16f*>((const float*)row + e + 4 * i)->v;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j];
      }
    } else {
      const u32x4 y = reinterpret_cast<const Any16*>((const bf16_t*)row + e)->v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(y[i] << 16);
        x[2 * i + 1] = __uint_as_float(y[i] & 0xffff0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = -INFINITY;
    if (e + i < vocab)
      x[i] = kWide ? ((const float*)row)[e + i]
                   : __uint_as_float((uint32_t)((const bf16_t*)row)[e + i] << 16);
  }
}

template <bool kWide>
__device__ __forceinline__ const void* logits_row(const VerifyArgs& a, int row) {
  return (const char*)a.logits + (size_t)row * a.logits_stride * (kWide ? 4 : 2);
}

// ---- sums and minima over the workgroup -----------------------------------------------
struct VLds {
  double d[kVWaves];
  float f[kVWaves];
  int i[kVWaves];
  int at, flag;
};

__device__ __forceinline__ double block_sum(VLds& lds, double x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.d[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < kVWaves; ++w) s += lds.d[w];
  return s;
}
// Sum of the threads before this one, and of all.
__device__ __forceinline__ double block_before(VLds& lds, double x, double& total) {
  double y = x;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const double z = __shfl_up(y, m, kWave);
    if ((int)(threadIdx.x & 63) >= m) y += z;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds.d[threadIdx.x >> 6] = y;
  __syncthreads();
  double before = y - x;
  total = 0;
#pragma unroll
  for (int w = 0; w < kVWaves; ++w) {
    if (w < (int)(threadIdx.x >> 6)) before += lds.d[w];
    total += lds.d[w];
  }
  return before;
}
__device__ __forceinline__ float block_max(VLds& lds, float x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = fmaxf(x, wave_xor(x, m));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.f[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = lds.f[0];
#pragma unroll
  for (int w = 1; w < kVWaves; ++w) s = fmaxf(s, lds.f[w]);
  return s;
}
__device__ __forceinline__ int block_min(VLds& lds, int x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = min(x, __shfl_xor(x, m, kWave));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.i[threadIdx.x >> 6] = x;
  __syncthreads();
  int s = lds.i[0];
#pragma unroll
  for (int w = 1; w < kVWaves; ++w) s = min(s, lds.i[w]);
  return s;
}

// Counts one arrival of the workgroup, whose stores (put) have gone out before; true for
// the last of n, for which the counter is cleared.
__device__ __forceinline__ bool last_to_arrive(VLds& lds, int* counter, int n) {
  wait_all_memory();
  __syncthreads();
  if (threadIdx.x == 0) {
    lds.flag = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (lds.flag == n - 1)
      __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return lds.flag == n - 1;
}

// The sequence that owns row `row` (cu does not decrease and starts at 0): the number of
// entries cu[1 .. num_seqs - 1] at or below it.
__device__ __forceinline__ int sequence_of(VLds& lds, const VerifyArgs& a, int row) {
  int n = 0;
  for (int s = 1 + threadIdx.x; s < a.num_seqs; s += kVThreads) n += a.cu[s] <= row;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) n += __shfl_xor(n, m, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds.i[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kVWaves; ++w) n += lds.i[w];
  return n;
}

// The first place where running sums exceed `target`: the threads' sums stand behind one
// another, `mine(i)` are the thread's eight; returns its element, or INT_MAX.
template <class F>
__device__ __forceinline__ int first_above(VLds& lds, double before, double target, int e, F mine) {
  int at = INT_MAX;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    before += mine(i);
    if (before > target) at = min(at, e + i);
  }
  return block_min(lds, at);
}

// The draw in a chunk whose weights sum up behind `before`: `fill(e, w)` gives the eight
// weights from element e on.  Where rounding leaves the target above all of them, the last
// with a weight (INT_MIN + 1: none).
template <class F>
__device__ __forceinline__ int draw_in_chunk(VLds& lds, int chunk, double before, double target,
                                             F fill) {
  int found = INT_MAX, last = INT_MAX;
#pragma unroll
  for (int v = 0; v < kVPer / 8; ++v) {
    const int e = chunk * kVChunk + (v * kVThreads + (int)threadIdx.x) * 8;
    double w[8], mine = 0;
    fill(e, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mine += w[i];
      if (w[i] > 0) last = min(last, -(e + i));
    }
    double total;
    const double b = before + block_before(lds, mine, total);
    if (found == INT_MAX) found = first_above(lds, b, target, e, [&](int i) { return w[i]; });
    before += total;
  }
  last = block_min(lds, last);
  return found != INT_MAX ? found : -last;
}

// The chunk that holds u of the total: sums(c) gives chunk c's, kVThreads at a time in
// order.  Returns it and the sum before it (the last chunk with a sum where rounding
// leaves none).
template <class F>
__device__ __forceinline__ int chunk_of(VLds& lds, int chunks, double target, F sums, double& before) {
  double all = 0, b_last = 0;
  int last = -1;
  for (int c0 = 0; c0 < chunks; c0 += kVThreads) {
    const int c = c0 + (int)threadIdx.x;
    const double x = c < chunks ? sums(c) : 0;
    double total;
    const double b = all + block_before(lds, x, total);
    const int found = block_min(lds, x > 0 && b + x > target ? c : INT_MAX);
    const int some = block_min(lds, x > 0 ? -c : INT_MAX);
    const int here = found != INT_MAX ? found : some != INT_MAX ? -some : -1;
    if (here >= 0) {
      __syncthreads();
      if (c == here) lds.d[0] = b;
      __syncthreads();
      b_last = lds.d[0];
      last = here;
    }
    if (found != INT_MAX) break;
    all += total;
  }
  before = b_last;
  return last;
}

// The token drawn from a row's weights with u (its chunks' sums are in `stats`).
template <bool kWide>
__device__ __forceinline__ int draw_row(VLds& lds, const VerifyArgs& a, const VStat* stats, int row,
                                        const VRow& r, double k, float u) {
  double before;
  const double target = (double)u * r.total;
  const int chunk = chunk_of(
      lds, verify_chunks(a.vocab), target,
      [&](int c) {
        const VStat s = get(stats + c);
        return s.sum * weight(s.top, r.top, k);
      },
      before);
  if (chunk < 0) return r.token;
  const void* x = logits_row<kWide>(a, row);
  const int t = draw_in_chunk(lds, chunk, before, target, [&](int e, double(&w)[8]) {
    float y[8];
    load8<kWide>(x, e, a.vocab, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = weight(y[i], r.top, k);
  });
  return t >= 0 && t < a.vocab ? t : r.token;
}

// ---- the walk (workgroup-parallel) ----------------------------------------------------
__device__ __forceinline__ void finish(const VerifyArgs& a, int s, int count, int token) {
  if (threadIdx.x == 0) {
    a.num_kept[s] = count;
    a.next_token[s] = token;
  }
  for (int i = count + (int)threadIdx.x; i < a.max_kept; i += kVThreads)
    a.kept[(size_t)s * a.max_kept + i] = -1;
}

// From node 0 to the child whose token is the one drawn.
__device__ __forceinline__ void walk(VLds& lds, const VerifyArgs& a, const VWs& ws, int s, int first,
                                     int n) {
  int here = 0, count = 0, token;
  for (;;) {
    if (threadIdx.x == 0) a.kept[(size_t)s * a.max_kept + count] = here;
    ++count;
    token = get(&ws.row[first + here]).token;
    if (count == a.max_kept) break;
    int child = INT_MAX;
    if (a.parents == nullptr) {
      if (here + 1 < n && a.tokens[first + here + 1] == token) child = here + 1;
    } else {
      for (int j = here + 1 + (int)threadIdx.x; j < n; j += kVThreads)
        if (child == INT_MAX && a.parents[first + j] == here && a.tokens[first + j] == token) child = j;
      child = block_min(lds, child);
    }
    if (child == INT_MAX) break;
    here = child;
  }
  finish(a, s, count, token);
}

template <bool kWide>
__global__ __launch_bounds__(kVThreads) void verify_rows_kernel(VerifyArgs a) {
  __shared__ VLds lds;
  const int chunks = verify_chunks(a.vocab);
  const VWs ws = verify_ws(a.ws, a.num_rows, a.vocab);
  for (int s = blockIdx.x * kVThreads + threadIdx.x; s < a.num_seqs; s += gridDim.x * kVThreads)
    if (a.cu[s + 1] == a.cu[s]) {          // no node: nothing kept, no token
      a.num_kept[s] = 0;
      a.next_token[s] = -1;
      for (int i = 0; i < a.max_kept; ++i) a.kept[(size_t)s * a.max_kept + i] = -1;
    }
  const int row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  if (a.num_seqs == 0 || row >= min(a.cu[a.num_seqs], a.num_rows)) return;

  float x[kVPer];
#pragma unroll
  for (int v = 0; v < kVPer / 8; ++v)
    load8<kWide>(logits_row<kWide>(a, row), chunk * kVChunk + (v * kVThreads + (int)threadIdx.x) * 8,
                 a.vocab, *reinterpret_cast<float(*)[8]>(x + 8 * v));
  const int s = sequence_of(lds, a, row);
  const int first = a.cu[s], n = a.cu[s + 1] - first;
  const float heat = a.temperature[s];
  const bool sampled = heat > 0.f;
  const double k = sampled ? 1.44269504088896340736 / (double)heat : 0.0;

  VStat st;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kVPer; ++i) top = fmaxf(top, x[i]);
  st.top = block_max(lds, top);
  st.sum = 0;
  if (sampled) {
#pragma unroll
    for (int i = 0; i < kVPer; ++i) st.sum += weight(x[i], st.top, k);
    st.sum = block_sum(lds, st.sum);
  }
  int arg = INT_MAX;
#pragma unroll
  for (int v = kVPer / 8 - 1; v >= 0; --v)
#pragma unroll
    for (int i = 7; i >= 0; --i)
      if (x[8 * v + i] == st.top) arg = chunk * kVChunk + (v * kVThreads + (int)threadIdx.x) * 8 + i;
  st.arg = block_min(lds, arg);
  VStat* stats = ws.stats + (size_t)row * chunks;
  if (threadIdx.x == 0) put(stats + chunk, st);
  if (!last_to_arrive(lds, ws.rows + row, chunks)) return;

  // ---- the row ---------------------------------------------------------------------------
  VRow r{};
  top = -INFINITY;
  for (int c = threadIdx.x; c < chunks; c += kVThreads) top = fmaxf(top, get(stats + c).top);
  r.top = block_max(lds, top);
  double total = 0;
  arg = INT_MAX;
  for (int c = threadIdx.x; c < chunks; c += kVThreads) {
    const VStat y = get(stats + c);
    if (sampled) total += y.sum * weight(y.top, r.top, k);
    if (y.top == r.top) arg = min(arg, y.arg);
  }
  r.total = block_sum(lds, total);
  arg = block_min(lds, arg);
  r.token = arg < a.vocab ? arg : 0;       // (a row of NaN: 0)
  const bool drawn = sampled && r.total > 0;
  if (a.draft == nullptr) {
    if (drawn) r.token = draw_row<kWide>(lds, a, stats, row, r, k, a.uniforms[row]);
  } else if (row + 1 < first + n) {
    const int next = a.tokens[row + 1];
    if (!drawn) {
      r.accept = next == r.token;
    } else if (next >= 0 && next < a.vocab) {
      float y;
      if constexpr (kWide)
        y = ((const float*)logits_row<kWide>(a, row))[next];
      else
        y = __uint_as_float((uint32_t)((const bf16_t*)logits_row<kWide>(a, row))[next] << 16);
      const double q = a.draft[(size_t)(row + 1) * a.draft_stride + next];
      r.accept = (double)a.uniforms[row + 1] * q < weight(y, r.top, k) / r.total;
    }
  }
  if (threadIdx.x == 0) put(ws.row + row, r);
  if (a.draft != nullptr) return;          // (the second launch goes on)
  if (!last_to_arrive(lds, ws.seqs + s, n)) return;
  walk(lds, a, ws, s, first, n);
}

// With the drafter's probabilities: the accepted nodes, and the token behind them.
template <bool kWide>
__global__ __launch_bounds__(kVThreads) void verify_rest_kernel(VerifyArgs a) {
  __shared__ VLds lds;
  const int chunks = verify_chunks(a.vocab);
  const VWs ws = verify_ws(a.ws, a.num_rows, a.vocab);
  const int s = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int first = a.cu[s], n = min(a.cu[s + 1], a.num_rows) - first;
  if (n <= 0) return;
  // the first node that is not accepted
  int count = INT_MAX;
  for (int j = threadIdx.x; j < n; j += kVThreads)
    if (count == INT_MAX && (j + 1 == n || get(&ws.row[first + j]).accept == 0)) count = j + 1;
  count = min(block_min(lds, count), a.max_kept);
  const int row = first + count - 1;
  const VRow r = get(&ws.row[row]);
  const float heat = a.temperature[s];
  const bool drawn = heat > 0.f && r.total > 0;
  // (behind max_kept nodes the next one is neither accepted nor refused)
  const bool refused = count < n && r.accept == 0;
  const double k = drawn ? 1.44269504088896340736 / (double)heat : 0.0;
  const float u = a.uniforms[first];
  if (chunk == 0) {
    for (int i = threadIdx.x; i < count; i += kVThreads) a.kept[(size_t)s * a.max_kept + i] = i;
  }
  if (!drawn || !refused) {
    if (chunk != 0) return;
    const int token = drawn ? draw_row<kWide>(lds, a, ws.stats + (size_t)row * chunks, row, r, k, u)
                            : r.token;
    finish(a, s, count, token);
    return;
  }
  const void* x = logits_row<kWide>(a, row);
  const float* q = a.draft + (size_t)(row + 1) * a.draft_stride;
  auto fill = [&](int e, double(&w)[8]) {
    float y[8], z[8];
    load8<kWide>(x, e, a.vocab, y);
    load8<true>(q, e, a.vocab, z);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      w[i] = e + i < a.vocab ? __builtin_fmax(weight(y[i], r.top, k) / r.total - (double)z[i], 0.0) : 0.0;
  };
  double sum = 0;
#pragma unroll
  for (int v = 0; v < kVPer / 8; ++v) {
    double w[8];
    fill(chunk * kVChunk + (v * kVThreads + (int)threadIdx.x) * 8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += w[i];
  }
  sum = block_sum(lds, sum);
  double* rest = ws.rest + (size_t)s * chunks;
  if (threadIdx.x == 0) put(rest + chunk, sum);
  if (!last_to_arrive(lds, ws.seqs + kVerifyMaxSeqs + s, chunks)) return;
  sum = 0;
  for (int c = threadIdx.x; c < chunks; c += kVThreads) sum += get(rest + c);
  const double total = block_sum(lds, sum);
  int token = -1;
  if (total > 0) {
    double before;
    const double target = (double)u * total;
    const int c = chunk_of(lds, chunks, target, [&](int i) { return get(rest + i); }, before);
    if (c >= 0) token = draw_in_chunk(lds, c, before, target, fill);
  }
  if (token < 0 || token >= a.vocab)       // (p = q to the last bit: p itself)
    token = draw_row<kWide>(lds, a, ws.stats + (size_t)row * chunks, row, r, k, u);
  finish(a, s, count, token);
}

}  // namespace

size_t verify_workspace(int num_rows, int num_seqs, int vocab) {
  const VWs w = verify_ws(nullptr, num_rows, vocab);
  return reinterpret_cast<size_t>(w.rest) +
         up256((size_t)num_seqs * verify_chunks(vocab) * sizeof(double));
}

int64_t verify_grid(const VerifyArgs& a) {
  return std::max<int64_t>(1, (int64_t)std::max(a.num_rows, a.draft != nullptr ? a.num_seqs : 0) *
                                  verify_chunks(a.vocab));
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  const int64_t chunks = verify_chunks(a.vocab);
  const dim3 rows((unsigned)std::max<int64_t>(1, a.num_rows * chunks)), block(kVThreads);
  const dim3 rest((unsigned)(a.num_seqs * chunks));
  if (a.wide)
    verify_rows_kernel<true><<<rows, block, 0, stream>>>(a);
  else
    verify_rows_kernel<false><<<rows, block, 0, stream>>>(a);
  if (a.draft != nullptr && a.num_rows > 0) {
    if (a.wide)
      verify_rest_kernel<true><<<rest, block, 0, stream>>>(a);
    else
      verify_rest_kernel<false><<<rest, block, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace rag
