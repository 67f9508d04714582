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
// are therefore fp64.
//
// First launch: a wave takes a segment of a row into its registers and leaves its maximum and
// sum; the logits are read once.  Second launch, without the drafter's probabilities: a wave for
// each row places the draw in a segment and reads that again; the last row of a sequence to finish
// walks.  With them: workgroups for the one row a sequence whose next token is drawn find it
// from the segments' sums, sum max(p - q, 0) in segments, and the last one draws.
//
// 16 trees of 24 to 64 nodes, 128,000 tokens in bf16: 67 us (under a trace 60 in the first launch, whose
// vector units are busy for 70%, some 20 instructions a logit; rows at T = 0 alone take 36, at 5 TB/s;
// and 14 in the second, a chain of dependent reads).  48 chains of 3 to 9 nodes with the drafter's
// probabilities, 128,077 tokens in fp32: 50 us (33, 4.8 TB/s, and 19).  One chain of five, 32,768
// tokens: 9.4, of which the kernels wait for one another's first reads.
#include "common.h"
#include "serve.h"

#include <climits>

namespace rag {

namespace {

constexpr int kVWaves = 4, kVThreads = kVWaves * kWave;
constexpr int kVStep = kWave * 8;               // logits of a wave's load
constexpr int kVCounters = 2 * kVerifyMaxSeqs;
constexpr int kVWalk = 1024;                    // nodes whose walk is in LDS

// A segment's maximum and sum of exp((x - maximum) / T): kV loads of a wave.
struct VStat {
  double sum;
  float top;
  int arg;                      // T = 0: the first index of the maximum
};

struct VWs {
  int* seqs;                    // [2][kVerifyMaxSeqs] arrivals
  VStat* stats;                 // [num_rows][segments]
  int* drawn;                   // [num_rows]
  double* rest;                 // [num_seqs][segments]
};

// Segments of a row, of kV loads each.
__host__ __device__ __forceinline__ int verify_segments(int vocab, int kv) {
  return (int)(((int64_t)vocab + kv * kVStep - 1) / (kv * kVStep));
}

__host__ __device__ __forceinline__ size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// (Sized for the shortest segments: calls of fewer rows have shorter ones.)
__host__ __device__ __forceinline__ VWs verify_ws(char* base, int num_rows, int vocab) {
  VWs w;
  const size_t segs = (size_t)verify_segments(vocab, 1);
  w.seqs = reinterpret_cast<int*>(base);
  base += up256(kVCounters * sizeof(int));
  w.stats = reinterpret_cast<VStat*>(base);
  base += up256(num_rows * segs * sizeof(VStat));
  w.drawn = reinterpret_cast<int*>(base);
  base += up256(num_rows * sizeof(int));
  w.rest = reinterpret_cast<double*>(base);
  return w;
}

// exp((x - top) / T) for x <= top; what lies under 2^-1000 counts as 0, as NaN does, and where
// top is infinite everything does.
//   2^t = 2^n p(t - n), n the nearest whole number (from the low bits of t + 1.5 2^52), p(f) =
//   1 + f r(f), r of degree 7 through (2^f - 1) / f at the Chebyshev nodes of [-1/2, 1/2]:
//   2^-38 relative, and 1 at 0 (so that equal logits have equal sums).  What of that all weights
//   share drops out of a draw, so that it moves one draw in 10^8 among 128,000 likely tokens.
struct Heat {
  double k, top;                // log2(e) / T
  float cut;
  __device__ __forceinline__ Heat(float top_, double k_) : k(k_), top(top_) {
    const double low = top - 1000.0 / k;
    cut = !(fabsf(top_) < INFINITY) ? INFINITY : low > -3.4028234663852886e38 ? (float)low : -3.4028234663852886e38f;
    // (never below: at small T a logit's last place is hundreds of powers of 2, which the exponent
    // has no room for)
    if ((double)cut < low) cut = nextafterf(cut, INFINITY);
  }
  // Of N logits, step by step side by side (one's steps wait for each other).  kExact: 0 is 0
  // (otherwise it may be as much as 2^-1022, which no sum notices).
  template <bool kExact, int N>
  __device__ __forceinline__ void weights(const float (&x)[N], double (&w)[N]) const {
    constexpr double kRound = 6755399441055744.0;
    constexpr double kP[9] = {1.0, 0.6931471805568324, 0.24022650695888503,
                              0.055504109063258665, 0.00961812913523614, 0.0013333478473685416,
                              0.00015403475186530786, 1.5303700711365693e-05, 1.325080551750225e-06};
    double f[N], p[N];
    uint32_t n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double d = (double)x[i] - top;
      const double m = __builtin_fma(d, k, kRound);
      f[i] = __builtin_fma(d, k, kRound - m);
      n[i] = (uint32_t)__builtin_bit_cast(uint64_t, m);
      p[i] = kP[8];
    }
#pragma unroll
    for (int j = 7; j >= 0; --j)
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = __builtin_fma(p[i], f[i], kP[j]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u32x2 b = __builtin_bit_cast(u32x2, p[i]);
      const bool some = x[i] >= cut;
      const u32x2 r = {kExact && !some ? 0u : b[0], some ? b[1] + (n[i] << 20) : 0u};
      w[i] = __builtin_bit_cast(double, r);
    }
  }
  __device__ __forceinline__ double weight(float x) const {
    const float one[1] = {x};
    double w[1];
    weights<true>(one, w);
    return w[0];
  }
};

// Eight logits of a row from element e on; -inf behind its end.  Rows may start at any
// element: the loads are of 16 bytes at any even address.
struct __attribute__((packed, aligned(2))) Any16 { u32x4 v; };
struct __attribute__((packed, aligned(4))) Any16f { f32x4 v; };

// Eight logits as they lie in memory.
template <bool kWide>
struct Raw8;
template <>
struct Raw8<false> {
  u32x4 a;
  __device__ __forceinline__ void load(const void* row, int e) {
    a = reinterpret_cast<const Any16*>((const bf16_t*)row + e)->v;
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<true> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void* row, int e) {
    a = reinterpret_cast<const Any16f*>((const float*)row + e)->v;
    b = reinterpret_cast<const Any16f*>((const float*)row + e + 4)->v;
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
};

template <bool kWide>
__device__ __forceinline__ void load8(const void* row, int e, int vocab, float (&x)[8]) {
  if (e + 8 <= vocab) {
    Raw8<kWide> r;
    r.load(row, e);
    r.unpack(x);
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

// A lane's share of a segment, kV loads from element e on, kVStep apart; `whole`: the wave's
// lie in the row (all are requested before the first is waited for).
template <bool kWide, int kV>
__device__ __forceinline__ void load_segment(const void* row, int e, int vocab, bool whole,
                                             float (&x)[kV][8]) {
  if (whole) {
    Raw8<kWide> r[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) r[v].load(row, e + v * kVStep);
#pragma unroll
    for (int v = 0; v < kV; ++v) r[v].unpack(x[v]);
  } else {
#pragma unroll
    for (int v = 0; v < kV; ++v) load8<kWide>(row, e + v * kVStep, vocab, x[v]);
  }
}

template <bool kWide>
__device__ __forceinline__ const void* logits_row(const VerifyArgs& a, int row) {
  return (const char*)a.logits + (size_t)row * a.logits_stride * (kWide ? 4 : 2);
}

// ---- over the wave ----------------------------------------------------------------------
// (by DPP and readlane: through LDS a sum of 64 bits takes a third of a microsecond)
template <int kCtrl, int kRows>
__device__ __forceinline__ double dpp64(double x) {
  u32x2 b = __builtin_bit_cast(u32x2, x);
#pragma unroll
  for (int i = 0; i < 2; ++i) b[i] = __builtin_amdgcn_update_dpp(0, b[i], kCtrl, kRows, 0xf, false);
  return __builtin_bit_cast(double, b);
}
// x of a lane that is the same for the wave.
__device__ __forceinline__ double lane_of(double x, int lane) {
  u32x2 b = __builtin_bit_cast(u32x2, x);
#pragma unroll
  for (int i = 0; i < 2; ++i) b[i] = __builtin_amdgcn_readlane(b[i], lane);
  return __builtin_bit_cast(double, b);
}
// Sum of the lanes up to this one: within rows of 16, then over rows 0 and 2, then over row 1's end.
__device__ __forceinline__ double wave_upto(double x) {
  x += dpp64<0x111, 0xf>(x);
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);
  return x + dpp64<0x143, 0xc>(x);
}
__device__ __forceinline__ double wave_sum(double x) { return lane_of(wave_upto(x), kWave - 1); }
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = fmaxf(x, wave_xor(x, m));
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = min(x, __shfl_xor(x, m, kWave));
  return x;
}
// Sum of the lanes before this one, and of all.
__device__ __forceinline__ double wave_before(double x, double& total) {
  const double y = wave_upto(x);
  total = lane_of(y, kWave - 1);
  return y - x;
}

// Counts one arrival of the workgroup at a counter, its coherent stores before it; true for the
// last of n, for which the counter is cleared.
__device__ __forceinline__ bool last_to_arrive(int& flag, int* counter, int n) {
  wait_all_memory();
  __syncthreads();
  if (threadIdx.x == 0) {
    flag = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (flag == n - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return flag == n - 1;
}

// The sequence that owns row `row` (cu does not decrease and starts at 0): the number of
// entries cu[1 .. num_seqs - 1] at or below it.
__device__ __forceinline__ int sequence_of(const VerifyArgs& a, int row) {
  int n = 0;
  for (int s0 = 1; s0 < a.num_seqs; s0 += kWave) {
    const int s = s0 + (int)(threadIdx.x & 63);
    n += __popcll(__builtin_amdgcn_ballot_w64(s < a.num_seqs && a.cu[min(s, a.num_seqs)] <= row));
  }
  return n;
}

__device__ __forceinline__ double log2e_over(float heat) {
  return heat > 0.f ? 1.44269504088896340736 / (double)heat : 0.0;
}

// A row from its segments' maxima and sums: `total` of exp((x - top) / T), and the first index of
// its maximum where nothing can be drawn from it (T = 0, no sum; -1: not looked for).
struct VRow {
  double total;
  float top;
  int best;
};

template <bool kWide>
__device__ __forceinline__ VRow row_of(const VerifyArgs& a, const VStat* stats, int segs, int row,
                                       float heat, double k) {
  const int lane = threadIdx.x & 63;
  VRow r{0, -INFINITY, -1};
  for (int c = lane; c < segs; c += kWave) r.top = fmaxf(r.top, stats[c].top);
  r.top = wave_max(r.top);
  const Heat w(r.top, k);
  int arg = INT_MAX;
  for (int c = lane; c < segs; c += kWave) {
    const VStat y = stats[c];
    if (heat > 0.f)
      r.total += y.sum * w.weight(y.top);
    else if (y.top == r.top)
      arg = min(arg, y.arg);
  }
  r.total = wave_sum(r.total);
  if (r.total > 0) return r;
  r.total = 0;
  if (r.top == -INFINITY) {                // (all masked: NaN among them is alike, but equals nothing)
    r.best = 0;
    return r;
  }
  if (heat > 0.f) {                        // (+inf among them)
    const void* x = logits_row<kWide>(a, row);
    for (int e = lane * 8; e < a.vocab; e += kVStep) {
      float y[8];
      load8<kWide>(x, e, a.vocab, y);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (y[i] == r.top && e + i < a.vocab) arg = min(arg, e + i);
    }
  }
  arg = wave_min(arg);
  r.best = arg < a.vocab ? arg : 0;
  return r;
}

// The segment in which running sums first exceed `target`, sums(c) being segment c's, and the
// sum before it; the last one with a sum where rounding leaves none, -1 where none has one.
template <class F>
__device__ __forceinline__ int segment_of(int segs, double target, F sums, double& before) {
  double all = 0;
  int last = -1;
  before = 0;
  for (int c0 = 0; c0 < segs; c0 += kWave) {
    const int c = c0 + (int)(threadIdx.x & 63);
    const double x = c < segs ? sums(c) : 0;
    double total;
    const double b = all + wave_before(x, total);
    const uint64_t above = __builtin_amdgcn_ballot_w64(x > 0 && b + x > target);
    const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0);
    if (some != 0) {
      const int l = above != 0 ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
      last = c0 + l;
      before = lane_of(b, l);
    }
    if (above != 0) break;
    all += total;
  }
  return last;
}

// The element of a segment in which running sums from `before` on first exceed `target`:
// w[v][i] is the weight of element e0 + v kVStep + 8 lane + i.  Where rounding leaves none the
// last with a weight; -1 where none has one.
template <int kV, class F>
__device__ __forceinline__ int element_of(int e0, double before, double target, F weights) {
  int last = -1;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    double w[8], mine = 0, total;
    weights(v, w);
    int some = -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mine += w[i];
      if (w[i] > 0) some = i;
    }
    double b = before + wave_before(mine, total);
    int at = -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      b += w[i];
      if (at < 0 && w[i] > 0 && b > target) at = i;
    }
    const uint64_t above = __builtin_amdgcn_ballot_w64(at >= 0);
    const uint64_t any = __builtin_amdgcn_ballot_w64(some >= 0);
    if (any != 0) {
      const int l = above != 0 ? __builtin_ctzll(above) : 63 - __builtin_clzll(any);
      last = e0 + v * kVStep + 8 * l + __builtin_amdgcn_readlane(above != 0 ? at : some, l);
    }
    if (above != 0) break;
    before += total;
  }
  return last;
}

// The token drawn from a row with u.
template <bool kWide, int kV>
__device__ __forceinline__ int draw_row(const VerifyArgs& a, const VStat* stats, int row, const VRow& r,
                                        double k, float u) {
  double before;
  const double target = (double)u * r.total;
  const Heat h(r.top, k);
  const int seg = segment_of(
      verify_segments(a.vocab, kV), target,
      [&](int c) { return stats[c].sum * h.weight(stats[c].top); }, before);
  const int e0 = max(seg, 0) * kV * kVStep, lane = threadIdx.x & 63;
  float x[kV][8];
  load_segment<kWide, kV>(logits_row<kWide>(a, row), e0 + lane * 8, a.vocab,
                          e0 + kV * kVStep <= a.vocab, x);
  const int t = element_of<kV>(e0, before, target,
                               [&](int v, double(&w)[8]) { h.weights<true>(x[v], w); });
  return min(max(t, 0), a.vocab - 1);
}

// What a row says without chance, or drawn with u.
template <bool kWide, int kV>
__device__ __forceinline__ int token_of(const VerifyArgs& a, const VStat* stats, int row, const VRow& r,
                                        double k, float u) {
  return r.best >= 0 ? r.best : draw_row<kWide, kV>(a, stats, row, r, k, u);
}

// ---- first launch ---------------------------------------------------------------------------
// (The workgroups' order is rows first, so that waves of a row stream neighbouring memory.)
template <bool kWide, int kV>
__global__ __launch_bounds__(kVThreads) void verify_rows_kernel(VerifyArgs a) {
  const int segs = verify_segments(a.vocab, kV), groups = (segs + kVWaves - 1) / kVWaves;
  const int row = blockIdx.x / groups, seg = blockIdx.x % groups * kVWaves + wave_id();
  if (seg >= segs) return;
  const int lane = threadIdx.x & 63, e0 = seg * kV * kVStep + lane * 8;
  float x[kV][8];
  load_segment<kWide, kV>(logits_row<kWide>(a, row), e0, a.vocab, (seg + 1) * kV * kVStep <= a.vocab, x);
  if (row >= a.cu[a.num_seqs]) return;     // behind the last sequence
  const float heat = a.temperature[sequence_of(a, row)];
  VStat st;
  st.top = -INFINITY;
  st.sum = 0;
  st.arg = INT_MAX;
#pragma unroll
  for (int v = 0; v < kV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) st.top = fmaxf(st.top, x[v][i]);
  st.top = wave_max(st.top);
  if (heat > 0.f) {
    const Heat w(st.top, log2e_over(heat));
    double sum[4] = {};
#pragma unroll
    for (int v = 0; v < kV * 2; ++v) {
      float z[4];
      double y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = x[v / 2][v % 2 * 4 + i];
      w.weights<false>(z, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += y[i];
    }
    st.sum = wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  } else {
#pragma unroll
    for (int v = kV - 1; v >= 0; --v)
#pragma unroll
      for (int i = 7; i >= 0; --i)
        if (x[v][i] == st.top) st.arg = e0 + v * kVStep + i;
    st.arg = wave_min(st.arg);
  }
  const VWs ws = verify_ws(a.ws, a.num_rows, a.vocab);
  if (lane == 0) ws.stats[(size_t)row * segs + seg] = st;
}

// ---- second launch ---------------------------------------------------------------------------
__device__ __forceinline__ void finish(const VerifyArgs& a, int s, int count, int token, int threads) {
  if (threadIdx.x == 0) {
    a.num_kept[s] = count;
    a.next_token[s] = token;
  }
  for (int i = count + (int)threadIdx.x; i < a.max_kept; i += threads)
    a.kept[(size_t)s * a.max_kept + i] = -1;
}

// Sequences without nodes: nothing kept, no token.
__device__ __forceinline__ void finish_empty(const VerifyArgs& a) {
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < a.num_seqs; s += gridDim.x * blockDim.x)
    if (a.cu[s + 1] == a.cu[s]) {
      a.num_kept[s] = 0;
      a.next_token[s] = -1;
      for (int i = 0; i < a.max_kept; ++i) a.kept[(size_t)s * a.max_kept + i] = -1;
    }
}

// From node 0 to the child whose token is the one drawn (one wave).
template <class Drawn, class Token, class Parent>
__device__ __forceinline__ void walk(const VerifyArgs& a, int s, int n, Drawn drawn, Token tokens,
                                     Parent parents) {
  int here = 0, count = 0, token;
  for (;;) {
    if (threadIdx.x == 0) a.kept[(size_t)s * a.max_kept + count] = here;
    ++count;
    token = drawn(here);
    if (count == a.max_kept) break;
    int child = INT_MAX;
    for (int j0 = here + 1; j0 < n && child == INT_MAX; j0 += kWave) {
      const int j = j0 + (int)threadIdx.x, x = min(j, n - 1);
      const uint64_t is = __builtin_amdgcn_ballot_w64(j < n && parents(x) == here && tokens(x) == token);
      if (is != 0) child = j0 + __builtin_ctzll(is);
      if (a.parents == nullptr) break;
    }
    if (child == INT_MAX) break;
    here = child;
  }
  finish(a, s, count, token, kWave);
}

// Without the drafter's probabilities: a wave draws a row's token; the last of a sequence walks.
template <bool kWide, int kV>
__global__ __launch_bounds__(kWave) void verify_walk_kernel(VerifyArgs a) {
  __shared__ int drawn[kVWalk], tokens[kVWalk], parents[kVWalk], flag;
  finish_empty(a);
  const int row = blockIdx.x;
  if (a.num_seqs == 0 || row >= min(a.cu[a.num_seqs], a.num_rows)) return;
  const VWs ws = verify_ws(a.ws, a.num_rows, a.vocab);
  const int segs = verify_segments(a.vocab, kV), s = sequence_of(a, row);
  // (rows behind num_rows are a broken precondition: no arrival of theirs is waited for)
  const int first = a.cu[s], n = min(a.cu[s + 1], a.num_rows) - first;
  const float heat = a.temperature[s], u = a.uniforms[row];
  const double k = log2e_over(heat);
  const VStat* stats = ws.stats + (size_t)row * segs;
  const VRow r = row_of<kWide>(a, stats, segs, row, heat, k);
  const int token = token_of<kWide, kV>(a, stats, row, r, k, u);
  if (threadIdx.x == 0)
    __hip_atomic_store(ws.drawn + row, token, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (!last_to_arrive(flag, ws.seqs + s, n)) return;
  auto get = [&](int i) {
    return __hip_atomic_load(ws.drawn + first + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  auto parent = [&](int i) { return a.parents != nullptr ? a.parents[first + i] : i - 1; };
  if (n > kVWalk) {
    walk(a, s, n, get, [&](int i) { return a.tokens[first + i]; }, parent);
    return;
  }
  for (int i = threadIdx.x; i < n; i += kWave) {
    drawn[i] = get(i);
    tokens[i] = a.tokens[first + i];
    parents[i] = parent(i);
  }
  __syncthreads();
  walk(a, s, n, [&](int i) { return drawn[i]; }, [&](int i) { return tokens[i]; },
       [&](int i) { return parents[i]; });
}

// With the drafter's probabilities: the kept nodes, and the token behind them.  Every workgroup
// of a sequence finds its last kept node, four rows at a time.
template <bool kWide, int kV, int kRows>
__global__ __launch_bounds__(kVThreads) void verify_rest_kernel(VerifyArgs a) {
  __shared__ double sh_total[kVWaves];
  __shared__ float sh_top[kVWaves];
  __shared__ int sh_best[kVWaves], sh_ok[kVWaves], flag;
  finish_empty(a);
  const int segs = verify_segments(a.vocab, kV), groups = (segs + kVWaves - 1) / kVWaves;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int s = blockIdx.x / groups, group = blockIdx.x % groups, seg = group * kVWaves + wave;
  const int first = a.cu[s], n = min(a.cu[s + 1], a.num_rows) - first;
  if (n <= 0) return;
  const VWs ws = verify_ws(a.ws, a.num_rows, a.vocab);
  const int row_segs = verify_segments(a.vocab, kRows);
  const float heat = a.temperature[s], u = a.uniforms[first];
  const double k = log2e_over(heat);

  int count = 0;
  VRow r;
  bool refused = false;
  while (count < a.max_kept && !refused && count < n) {
    const int i = min(count + wave, n - 1), row = first + i;
    VRow mine = row_of<kWide>(a, ws.stats + (size_t)row * row_segs, row_segs, row, heat, k);
    bool ok = false;
    if (i + 1 < n) {
      const int next = a.tokens[row + 1];
      if (mine.best >= 0) {
        ok = next == mine.best;
      } else if (next >= 0 && next < a.vocab) {
        const void* x = logits_row<kWide>(a, row);
        const float y = kWide ? ((const float*)x)[next]
                              : __uint_as_float((uint32_t)((const bf16_t*)x)[next] << 16);
        const double q = a.draft[(size_t)(row + 1) * a.draft_stride + next];
        ok = (double)a.uniforms[row + 1] * q < Heat(mine.top, k).weight(y) / mine.total;
      }
    }
    if (lane == 0) {
      sh_total[wave] = mine.total;
      sh_top[wave] = mine.top;
      sh_best[wave] = mine.best;
      sh_ok[wave] = ok;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kVWaves; ++w) {
      if (refused || count == a.max_kept || count == n) break;
      r = VRow{sh_total[w], sh_top[w], sh_best[w]};
      ++count;
      refused = sh_ok[w] == 0;             // (the last node has no next one to refuse)
    }
    __syncthreads();
  }
  refused = refused && count < n && count < a.max_kept;   // (the last that may be kept has no children)
  const int row = first + count - 1;
  const VStat* stats = ws.stats + (size_t)row * row_segs;
  if (group == 0)
    for (int i = threadIdx.x; i < count; i += kVThreads) a.kept[(size_t)s * a.max_kept + i] = i;
  if (!refused || r.best >= 0) {
    if (group != 0) return;
    int token = r.best;
    if (token < 0 && wave == 0) token = draw_row<kWide, kRows>(a, stats, row, r, k, u);
    finish(a, s, count, token, kVThreads);
    return;
  }
  const void* x = logits_row<kWide>(a, row);
  const float* q = a.draft + (size_t)(row + 1) * a.draft_stride;
  const Heat h(r.top, k);
  const double inv = 1.0 / r.total;
  float y[kV][8], z[kV][8];
  auto rest_of = [&](int v, int e0, double(&w)[8]) {     // max(p - q, 0)
    h.weights<true>(y[v], w);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      w[i] = e0 + v * kVStep + lane * 8 + i < a.vocab
                 ? __builtin_fmax(__builtin_fma(w[i], inv, -(double)z[v][i]), 0.0)
                 : 0.0;
  };
  auto load = [&](int e0) {
    load_segment<kWide, kV>(x, e0 + lane * 8, a.vocab, e0 + kV * kVStep <= a.vocab, y);
    load_segment<true, kV>(q, e0 + lane * 8, a.vocab, e0 + kV * kVStep <= a.vocab, z);
  };
  double sum = 0;
  load(seg * kV * kVStep);
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    double w[8];
    rest_of(v, seg * kV * kVStep, w);
    sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
  }
  sum = wave_sum(sum);
  uint64_t* rest = reinterpret_cast<uint64_t*>(ws.rest + (size_t)s * segs);
  if (lane == 0 && seg < segs)
    __hip_atomic_store(rest + seg, __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  if (!last_to_arrive(flag, ws.seqs + kVerifyMaxSeqs + s, groups)) return;
  auto sums = [&](int c) {
    return __builtin_bit_cast(
        double, __hip_atomic_load(rest + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  };
  int token = -1;
  if (wave == 0) {
    double total = 0, before;
    for (int c = lane; c < segs; c += kWave) total += sums(c);
    const double target = (double)u * wave_sum(total);
    const int c = segment_of(segs, target, sums, before);
    if (c >= 0) {
      load(c * kV * kVStep);
      token = element_of<kV>(c * kV * kVStep, before, target,
                             [&](int v, double(&w)[8]) { rest_of(v, c * kV * kVStep, w); });
    }
    if (token < 0 || token >= a.vocab)     // (p = q to the last bit: p itself)
      token = draw_row<kWide, kRows>(a, stats, row, r, k, u);
  }
  finish(a, s, count, token, kVThreads);
}

// Loads of a segment: as many as leave the GPU this many waves.  Microseconds of a call with one, two and
// four loads of its rows (bf16, no draft probabilities):
//   128,000 tokens  20 rows 12.6, 11.9, 12.9   40 rows 15.2, 13.3, 13.9   131 rows 24.4, 21.2, 21.3
//                   700 rows 92, 78, 70
//   32,768 tokens   66 rows 10.6, 10.6, 11.5   131 rows 13.2, 12.3, 12.7   700 rows 33, 30, 29
// Over 132 batches of 8 to 384 rows of 20,000 to 256,000 tokens the launch that this chooses is 1.1% above the
// best of the three on average (with 1024 1.9%, 4096 1.9%, 8192 4.2%).  Eight loads a wave: 2 us more where
// four are chosen.
constexpr int64_t kVFill = 2048;
constexpr int kVMaxLoads = 4;
// The same of the rows whose next token is drawn from max(p - q, 0), one a sequence: longer segments also cost
// fewer arrivals.  Chains of six, fp32:
//   128,077 tokens  8 sequences 22.4, 20.5, 22.5   16 33.6, 27.7, 27.6   48 62, 51, 46
//   32,768 tokens   8 sequences 12.8, 13.4, 15.3   48 23.1, 22.4, 24.2   96 35.1, 31.0, 32.7
// Over 132 batches of 2 to 64 sequences 1.9% above the best (with 512 2.1%, 1024 1.5% but up to 12% above
// 1792 in some, 2048 2.6%, 4096 5.9%).
constexpr int64_t kVRestFill = 1792;
constexpr int kVMaxRestLoads = 4;

int verify_loads(int64_t rows, int vocab, int64_t fill, int kv) {
  while (kv > 1 && rows * verify_segments(vocab, kv) < fill) kv /= 2;
  return kv;
}

int row_loads(const VerifyArgs& a) { return verify_loads(a.num_rows, a.vocab, kVFill, kVMaxLoads); }
int rest_loads(const VerifyArgs& a) {
  return verify_loads(a.num_seqs, a.vocab, kVRestFill, kVMaxRestLoads);
}

int64_t verify_groups(int vocab, int kv) {
  return (verify_segments(vocab, kv) + kVWaves - 1) / kVWaves;
}

template <bool kWide, int kV>
void launch_verify_v(const VerifyArgs& a, hipStream_t stream) {
  const dim3 block(kVThreads);
  if (a.num_rows > 0)
    verify_rows_kernel<kWide, kV>
        <<<dim3((unsigned)(a.num_rows * verify_groups(a.vocab, kV))), block, 0, stream>>>(a);
  if (a.draft == nullptr || a.num_rows == 0) {
    verify_walk_kernel<kWide, kV>
        <<<dim3((unsigned)std::max(a.num_rows, 1)), dim3(kWave), 0, stream>>>(a);
    return;
  }
  const int kv = rest_loads(a);
  const dim3 grid((unsigned)(a.num_seqs * verify_groups(a.vocab, kv)));
  if (kv == 1)
    verify_rest_kernel<kWide, 1, kV><<<grid, block, 0, stream>>>(a);
  else if (kv == 2)
    verify_rest_kernel<kWide, 2, kV><<<grid, block, 0, stream>>>(a);
  else
    verify_rest_kernel<kWide, 4, kV><<<grid, block, 0, stream>>>(a);
}

template <bool kWide>
void launch_verify_w(const VerifyArgs& a, hipStream_t stream) {
  switch (row_loads(a)) {
    case 1: launch_verify_v<kWide, 1>(a, stream); break;
    case 2: launch_verify_v<kWide, 2>(a, stream); break;
    default: launch_verify_v<kWide, 4>(a, stream);
  }
}

}  // namespace

size_t verify_workspace(int num_rows, int num_seqs, int vocab) {
  const VWs w = verify_ws(nullptr, num_rows, vocab);
  return reinterpret_cast<size_t>(w.rest) +
         up256((size_t)num_seqs * verify_segments(vocab, 1) * sizeof(double));
}

int64_t verify_grid(const VerifyArgs& a) {
  return std::max(a.num_rows * verify_groups(a.vocab, row_loads(a)),
                  a.num_seqs * verify_groups(a.vocab, rest_loads(a)));
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  a.wide ? launch_verify_w<true>(a, stream) : launch_verify_w<false>(a, stream);
  return hipGetLastError();
}

}  // namespace rag
