// Attention of a few query rows a sequence over a paged cache held in 4 bits
// (gfx950): one decode step, or a chain of drafted tokens judged in one step.
//
// With codes c, scales s and zero points z of a group of 64 channels (kv4.h):
//   score   q k   = sum over groups of s_k (sum_c q (128 + c) - (128 + z_k) sum_c q)
//   output  p v   = sum_k p' (128 + c) - sum_k p' (128 + z_k),   p' = bf16(p s_k)
// so that both products take the codes as they are (the bf16 numbers 128 + c, two
// by one shift and one and-or), on v_mfma_f32_16x16x32_bf16: S^T = K Q^T with the
// (row, q head) pairs of a kv head as the 16 columns, then O^T = V^T P^T, whose B
// operand the lanes hold already.  The corrections are products too: 128 + z is a bf16
// number, sum q three of them (24 bits), and the second is the same P^T under one more
// row.  Sums and maxima are fp32; p' is rounded to bf16 for the matrix unit, as P is in the
// bf16 cache's kernels, and the correction uses the rounded p', so that 128 cancels.
//
// HBM-bound where each sequence has few pairs (64 sequences of 2.6k to 10.3k keys, 32 q / 8 kv heads of
// 128: 84 us, 5.0 TB/s); with 16 to 64 pairs a sequence bound by the chains of product, softmax and
// product of the two waves that a SIMD has room for (32 chains of 3 to 9 rows, 700 to 10,304 keys: 61 us,
// vector units 41% busy, matrix units 11%; of its 256 registers the join of up to 64 pairs spills 18, addresses
// that it loads again for every piece; the loops over blocks spill none).
//
// Pages are copied straight into LDS with 16 bytes a lane and lanes in the pages' order, parameters with
// a load of their lines: a load that finds a line still on its way holds up all behind it (the 64
// sequences: 98 us with the codes loaded as the matrix operands have them, 113 with the parameters'
// lines read where they are needed).
//   up to 8 pairs   kv4_wave_few: a wave has four pages at a time, and spreads them over the matrix
//                   unit's columns that no pair needs
//   up to 64        kv4_wave: blocks of two pages, kQStages - 1 of them ahead, of which each of the four
//                   waves copies every fourth.  Up to 32 pairs a wave attends the blocks that it has
//                   copied, with one or two tiles of 16 pairs (the codes are unpacked once: 61 us for the
//                   32 chains, 64 with a tile a wave and two waves beside each other); for up to 64 two
//                   and two waves have half of the pairs each and every second block.
//   more            tiles of 64 pairs
// The waves join their states through LDS.  As many workgroups as the chip takes at a time get even shares
// of all sequences' blocks; a sequence that is cut writes partial outputs and log-sum-exps, which
// the last of its workgroups to finish joins.
#include "common.h"
#include "kv4.h"
#include "serve.h"

#include <type_traits>

namespace rag {

namespace {

constexpr int kQWaves = 4;
constexpr int kQKeys = 32;                 // keys of a block
constexpr int kQPairs = 16 * kQWaves;      // pairs of a tile, at most
// Work of a share, at least, as that of blocks of up to 16 pairs (at 17 to 32 pairs it is that of 5 blocks,
// above of 4; a tile's start counts too).  One sequence of 4,782 keys, 32 q / 8 kv heads: 13.6 us; with 4
// 2.9 more (more partials to join), with 16 0.1 more.
constexpr int kQMinBlocks = 8;
// Blocks that the start of a tile counts for: a workgroup's second piece costs 10 to 20 us more than its
// blocks (plan, first loads, states, partials; the 32 chains: 61 us; with 18 62.5, 32 63.8).
constexpr int kQStart = 24;
constexpr int kQMaxPieces = 64;            // of a tile (one lane each in the join)
// Workgroups: two a CU, as many as there is LDS for (1024: 64 sequences of 2.6k to 10.3k keys 12 us
// more).
constexpr int kQWorkgroups = 512;

// One row tile's piece of work: blocks [b0, b1) of its n.
struct Kv4Piece {
  int s, tile, b0, b1;
  int p, n, first;              // the p-th of n pieces; the unit of the first
  int qb, rows, kv_len;
  int next;                     // where in the unit's share the next piece starts
};

// All sequences' blocks and the workgroups' shares of them.
struct Kv4Plan {
  int total, share;
};

constexpr int kQStages = 3;

// A block in LDS: K codes of its two pages, V codes, parameters [page][K, V][group][token].
template <int D>
struct alignas(16) Kv4Block {
  char k[16 * D], v[16 * D];
  uint32_t p[D];
  static constexpr int kOps = D == 128 ? 6 : 3;      // loads that fill one
};

// Up to 8 pairs: what a wave has of four pages.
template <int D>
struct alignas(16) Kv4Four {
  char k[32 * D], v[32 * D];
  uint32_t kp[D], vp[D];                   // [page][group][token]
  static constexpr int kOps = D == 128 ? 12 : 6;     // loads that fill one
};

template <int D, int R, int C>
struct Kv4Lds {
  union {
    Kv4Block<D> ring[R == 1 ? kQStages : 0][kQWaves];
    Kv4Four<D> four[R == 1 ? 0 : kQWaves][2];
    float o[kQWaves][16 * C / R][D + 4];
  };
  float m[kQWaves][16 * C], l[kQWaves][16 * C];
  int start[kKv4PlanSeqs + 1];
  int wave_sum[kQWaves], longest[kQWaves], flag;
  Kv4Piece piece;
};

__device__ __forceinline__ int wave_scan(int x) {       // inclusive
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int y = __shfl_up(x, m, kWave);
    if ((int)(threadIdx.x & 63) >= m) x += y;
  }
  return x;
}

// (Tiles and partials are laid out for max_rows; more are a broken precondition, of which the first
// max_rows are attended.)
__device__ __forceinline__ void kv4_sequence(const Kv4Args& a, int s, int& qb, int& rows, int& kv) {
  qb = a.cu_q != nullptr ? a.cu_q[s] : s;
  rows = a.cu_q != nullptr ? min(a.cu_q[s + 1] - qb, a.max_rows) : 1;
  kv = min(a.kv_lens[s], a.max_blocks * 16);
}

// Waves beside each other on a block, for this many pairs.
__device__ __forceinline__ int kv4_side(int pairs) { return pairs <= 32 ? 1 : 2; }
// A block's work.  (The 32 chains: 61 us; with 3 : 4 : 7 61.3, 2 : 3 : 5 and 3 : 4 : 6 62.)
__device__ __forceinline__ int kv4_weight(int pairs) { return pairs <= 16 ? 2 : pairs <= 32 ? 3 : 4; }
constexpr int kQMaxWeight = 4;

__device__ __forceinline__ int kv4_blocks(int kv_len) {
  return (max(kv_len, 0) + kQKeys - 1) / kQKeys;
}

// The sequences' places in one row of all blocks, kQStart more in front of each tile, each counted
// by its work.
template <class Lds>
__device__ __forceinline__ void kv4_plan(const Kv4Args& a, Lds& lds, Kv4Plan& plan) {
  const int group = a.hq / a.hkv;
  int sum = 0, longest = 0, start[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = threadIdx.x * 4 + i;
    int tiles = 0, len = 0;
    if (s < a.num_seqs) {
      int qb, rows, kv;
      kv4_sequence(a, s, qb, rows, kv);
      tiles = (max(rows, 0) * group + kQPairs - 1) / kQPairs;
      len = (kv4_blocks(kv) + kQStart) * kv4_weight(max(rows, 0) * group);
    }
    start[i] = sum;
    sum += tiles * len;
    if (tiles > 0) longest = max(longest, len);
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_scan(sum);
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) longest = max(longest, __shfl_xor(longest, m, kWave));
  if (lane == 63) {
    lds.wave_sum[wave] = upto;
    lds.longest[wave] = longest;
  }
  __syncthreads();
  int before = upto - sum;
  plan.total = 0;
  longest = 0;
#pragma unroll
  for (int w = 0; w < kQWaves; ++w) {
    if (w < wave) before += lds.wave_sum[w];
    plan.total += lds.wave_sum[w];
    longest = max(longest, lds.longest[w]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) lds.start[threadIdx.x * 4 + i] = start[i] + before;
  if (threadIdx.x == 0) lds.start[kKv4PlanSeqs] = plan.total;
  // (a tile is cut into at most kQMaxPieces)
  plan.share = max(max((plan.total + a.units - 1) / a.units, kQMinBlocks * kv4_weight(1)),
                   (longest + kQMaxPieces - 3) / (kQMaxPieces - 2));
}

// The piece at `at` of the unit's share, the same for all threads; s < 0: no more.
template <class Lds>
__device__ __forceinline__ Kv4Piece kv4_find(const Kv4Args& a, Lds& lds, const Kv4Plan& plan,
                                             int unit, int at) {
  const int from = unit * plan.share, to = min(from + plan.share, plan.total), g = from + at;
  __syncthreads();                         // (the last piece's readers are done)
  if (g >= to) {
    Kv4Piece none{};
    none.s = -1;
    return none;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = threadIdx.x * 4 + i, off = g - lds.start[s];
    if (off >= 0 && g < lds.start[s + 1]) {
      Kv4Piece x;
      x.s = s;
      kv4_sequence(a, x.s, x.qb, x.rows, x.kv_len);
      const int weight = kv4_weight(x.rows * (a.hq / a.hkv));
      const int len = (kv4_blocks(x.kv_len) + kQStart) * weight;
      x.tile = off / len;
      const int t0 = lds.start[s] + x.tile * len, t1 = t0 + len;
      x.b0 = max((g - t0) / weight - kQStart, 0);
      x.b1 = max((min(to, t1) - t0) / weight - kQStart, 0);
      // (a unit whose share ends before the tile's first block has no piece of it)
      x.first = min(t0 + kQStart * weight, t1 - 1) / plan.share;
      x.n = (t1 - 1) / plan.share - x.first + 1;
      x.p = unit - x.first;
      x.next = min(to, t1) - from;
      lds.piece = x;
    }
  }
  __syncthreads();
  // (the same for all lanes, which the compiler is to know: scalar registers and loads)
  Kv4Piece x;
  const int* src = reinterpret_cast<const int*>(&lds.piece);
  int* dst = reinterpret_cast<int*>(&x);
#pragma unroll
  for (size_t i = 0; i < sizeof(x) / sizeof(int); ++i) dst[i] = __builtin_amdgcn_readfirstlane(src[i]);
  return x;
}

// Where the parameters of a page and group stand in a block.
template <int D>
__device__ __forceinline__ constexpr int kv4_place(int j, int values, int g) {
  return ((2 * j + values) * (D / 64) + g) * 16;
}

template <int N>
__device__ __forceinline__ void kv4_read(uint32_t (&x)[N], const char* p) {
  if constexpr (N == 4) {
    const u32x4 y = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i];
  } else {
    const u32x2 y = *reinterpret_cast<const u32x2*>(p);
    x[0] = y[0];
    x[1] = y[1];
  }
}

__device__ __forceinline__ bf16x8 kv4_operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4 x = {a, b, c, d};
  return as_bf16x8(x);
}

// p[i], i the same for the wave, of memory that the kernel does not write.
__device__ __forceinline__ int kv4_uniform(const int32_t* p, int i) {
  typedef __attribute__((address_space(4))) const int32_t const_i32;
  return ((const_i32*)p)[i];
}

// A wave's state of 16 (row, q head) pairs: O^T without its corrections, the corrections, the
// sum of weights (this lane's keys' share) and the maximum that they refer to.
template <int D>
struct Kv4State {
  f32x4 o[D / 16];              // [4 g + e]: channels 64 g + 4 (4 g4 + r) + e
  f32x4 corr[D / 64];           // (the same in all rows)
  float l, m;
};

// Maximum over the four lanes of a column (lanes l16 + 16 g4).
__device__ __forceinline__ float column_max(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Memory and the waits around it, in the order that they are written in.
__device__ __forceinline__ void kv4_fence() { asm volatile("" ::: "memory"); }

// The wave's 16 C pairs (pair0 on) against the piece's blocks, `side` waves beside each other on each
// of them.  With C = 2 both tiles of pairs take the codes as they were unpacked once.
template <int D, int C, class Lds>
__device__ __forceinline__ void kv4_wave(const Kv4Args& a, const Kv4Piece& x, int h, int pair0, int side,
                                         Lds& lds, Kv4State<D> (&st)[C]) {
  constexpr int kG = D / 64;
  using P = Kv4Page<D>;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, wave = wave_id();
  const int group = a.hq / a.hkv, pairs = x.rows * group;
  const float c = a.scale * kLog2e, tau = fminf(kRescaleLog2 / c, 1e30f);   // (finite at any scale)
  const Kv4Unpack unpack;

  // ---- copies ---------------------------------------------------------------------------------
  const int pages = (x.kv_len + 15) / 16;
  const int32_t* table = a.tables + (size_t)x.s * a.max_blocks;
  const size_t stride = (size_t)a.hkv * P::kBytes;
  const char* kc = (const char*)a.k_cache + (size_t)h * P::kBytes;
  const char* vc = (const char*)a.v_cache + (size_t)h * P::kBytes;
  // The lane's 16 bytes of a page (two pages where D = 64).  D = 128: each four lanes' in an order
  // of their own, so that 16 lanes that read every fourth piece find them in all banks.
  const int piece = kG == 2 ? 16 * ((lane & ~3) | ((lane - g4) & 3)) : 16 * (lane & 31);
  const char* pc = (lane / (16 * kG) % 2 ? vc : kc) + P::kParams + lane % (16 * kG) * 4;
  // Behind the last block that one is copied again, so that the number of loads on their way is
  // known.  Page ids come through the scalar cache, a block before they are used.
  int next[2];
  auto find = [&](int blk) {               // (behind the last page: that one again)
#pragma unroll
    for (int j = 0; j < 2; ++j) next[j] = kv4_uniform(table, min(2 * min(blk, x.b1 - 1) + j, pages - 1));
  };
  auto copy = [&](int stage) {
    Kv4Block<D>& to = lds.ring[stage][wave];
    const size_t id0 = (size_t)next[0] * stride, id1 = (size_t)next[1] * stride;
    if constexpr (kG == 2) {
      dma16_stream(kc + id0 + piece, to.k);
      dma16_stream(kc + id1 + piece, to.k + 8 * D);
      dma4_stream(pc + id0, to.p);
      dma4_stream(pc + id1, to.p + 64);
      dma16_stream(vc + id0 + piece, to.v);
      dma16_stream(vc + id1 + piece, to.v + 8 * D);
    } else {
      const size_t id = lane < 32 ? id0 : id1;
      dma16_stream(kc + id + piece, to.k);
      dma4_stream(pc + id, to.p);
      dma16_stream(vc + id + piece, to.v);
    }
  };
  if (x.b0 < x.b1) {
#pragma unroll
    for (int i = 0; i < kQStages - 1; ++i) {
      find(x.b0 + i * kQWaves + wave);
      copy(i);
    }
    find(x.b0 + (kQStages - 1) * kQWaves + wave);
  }

  int last[C];                             // the last key that the lane's column sees
  bf16x8 q[C][2 * kG];
  bf16x8 qz[C][kG];                        // minus the sum of q, in three parts
#pragma unroll
  for (int t = 0; t < C; ++t) {
    const int pair = min(pair0 + 16 * t + l16, pairs - 1), row = pair / group;
    last[t] = x.kv_len - x.rows + row;
    const bf16_t* src = (const bf16_t*)a.q + ((size_t)(x.qb + row) * a.hq + h * group + pair % group) * D;
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const u32x4 y = load16(src + 64 * g + 16 * g4 + 8 * w);
        q[t][2 * g + w] = as_bf16x8(y);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum += __uint_as_float(y[i] << 16) + __uint_as_float(y[i] & 0xffff0000u);
      }
      sum += wave_xor(sum, 16);
      sum += wave_xor(sum, 32);
      const float part0 = (float)(__bf16)-sum, part1 = (float)(__bf16)(-sum - part0);
      const float on = g4 == 0 ? 1.f : 0.f;
      qz[t][g] =
          to_bf16x8(part0 * on, part1 * on, (-sum - part0 - part1) * on, 0.f, 0.f, 0.f, 0.f, 0.f);
      st[t].corr[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    st[t].l = 0.f;
    st[t].m = -INFINITY;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) st[t].o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // where the lane's operands stand in a page's codes
  const int at = kG == 2 ? 16 * (4 * l16 + ((g4 + (l16 >> 2)) & 3)) : 8 * (4 * l16 + g4);
  auto block = [&](const Kv4Block<D>& r, int b, auto masked_t) {
    constexpr bool masked = decltype(masked_t)::value;
    const int key0 = kQKeys * b;
    const uint32_t* params = r.p;
    // ---- S^T = K Q^T ---------------------------------------------------------------
    float sc[C][8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t code[2 * kG];
      kv4_read(code, r.k + 8 * D * j + at);
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const uint32_t kz = params[kv4_place<D>(j, 0, g) + l16];
        const uint32_t zz = __builtin_amdgcn_perm(kz, kz, 0x01000100u);
        f32x4 acc[C];
#pragma unroll
        for (int t = 0; t < C; ++t)
          acc[t] = mfma16(kv4_operand(zz, zz, zz, zz), qz[t][g], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t y = code[2 * g + w];
          const bf16x8 k = kv4_operand(unpack(y, 0), unpack(y, 1), unpack(y, 2), unpack(y, 3));
#pragma unroll
          for (int t = 0; t < C; ++t) acc[t] = mfma16(k, q[t][2 * g + w], acc[t]);
        }
        const u32x4 kp = *reinterpret_cast<const u32x4*>(params + kv4_place<D>(j, 0, g) + 4 * g4);
#pragma unroll
        for (int t = 0; t < C; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float s = kv4_scale(kp[i]);
            sc[t][4 * j + i] = g == 0 ? s * acc[t][i] : fmaf(s, acc[t][i], sc[t][4 * j + i]);
          }
      }
    }
    u32x4 vp[2][kG];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < kG; ++g)
        vp[j][g] = *reinterpret_cast<const u32x4*>(params + kv4_place<D>(j, 1, g) + 4 * g4);
    uint32_t v[2][2 * kG];
#pragma unroll
    for (int j = 0; j < 2; ++j) kv4_read(v[j], r.v + 8 * D * j + at);
    // ---- masks: keys that a row does not see, and slots behind the last key -----------
    if constexpr (masked) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = key0 + 16 * (i / 4) + 4 * g4 + i % 4;
#pragma unroll
        for (int t = 0; t < C; ++t)
          if (key > last[t]) sc[t][i] = -INFINITY;
#pragma unroll
        for (int g = 0; g < kG; ++g) {     // (zero points alike for all columns: none that is NaN)
          const uint32_t y = key < x.kv_len ? vp[i / 4][g][i % 4] : 0;
          vp[i / 4][g][i % 4] = (y & 0x7f80u) == 0x7f80u ? y & 0xffff0000u : y;
        }
      }
    }
    // ---- softmax ------------------------------------------------------------------------
#pragma unroll
    for (int t = 0; t < C; ++t) {
      float top = sc[t][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[t][i]);
      top = column_max(top);
      if (wave_any(top > st[t].m + tau)) {
        const float m = fmaxf(st[t].m, top);
        const float alpha = st[t].m == -INFINITY ? 0.f : fast_exp2((st[t].m - m) * c);
        st[t].l *= alpha;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) st[t].o[i] *= alpha;
#pragma unroll
        for (int g = 0; g < kG; ++g) st[t].corr[g] *= alpha;
        st[t].m = m;
      }
      const float ref = st[t].m == -INFINITY ? 0.f : -st[t].m * c;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sc[t][i] = fast_exp2(fmaf(sc[t][i], c, ref));
        st[t].l += sc[t][i];
      }
    }
    // ---- O^T += V^T P^T ---------------------------------------------------------------------
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      bf16x8 pf[C];
#pragma unroll
      for (int t = 0; t < C; ++t) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = sc[t][i] * kv4_scale(vp[i / 4][g][i % 4]);
        if constexpr (masked) {            // (the scale of a key not seen may be NaN)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (key0 + 16 * (i / 4) + 4 * g4 + i % 4 > last[t]) y[i] = 0.f;
        }
        pf[t] = to_bf16x8(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
      }
      uint32_t w[4], zz[4];                // two keys' units of group g, and their zero points
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 pr = vp[i / 2][g];
        zz[i] = __builtin_amdgcn_perm(pr[i % 2 * 2 + 1], pr[i % 2 * 2], 0x05040100u);
        if constexpr (kG == 1)
          w[i] = v[i / 2][i % 2];
        else
          w[i] = __builtin_amdgcn_perm(v[i / 2][i % 2 * 2 + 1], v[i / 2][i % 2 * 2],
                                       g == 0 ? 0x05040100u : 0x07060302u);
      }
#pragma unroll
      for (int t = 0; t < C; ++t)
        st[t].corr[g] = mfma16(kv4_operand(zz[0], zz[1], zz[2], zz[3]), pf[t], st[t].corr[g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x8 vv = kv4_operand(unpack(w[0], e), unpack(w[1], e), unpack(w[2], e), unpack(w[3], e));
#pragma unroll
        for (int t = 0; t < C; ++t) st[t].o[4 * g + e] = mfma16(vv, pf[t], st[t].o[4 * g + e]);
      }
    }
  };
  // Blocks base .. base + 3 stand in stage `stage`.  Waits for the wave's own copies (and, where waves
  // share blocks, for the others'), then starts those of the stage that all are done with.
  int stage = 0;
  auto turn = [&] {
    kv4_fence();
    __builtin_amdgcn_s_waitcnt(0x0070 | (Kv4Block<D>::kOps * (kQStages - 2)));   // and lgkmcnt(0)
    if (side > 1) __builtin_amdgcn_s_barrier();
    kv4_fence();
  };
  auto refill = [&](int base) {
    copy(stage == 0 ? kQStages - 1 : stage - 1);
    find(base + kQStages * kQWaves + wave);
  };
  const int open = (x.kv_len - x.rows + 1) / kQKeys;     // blocks that all rows see whole
  auto blocks = [&](int& base, int to, auto masked_t) {
    for (; base < to; base += kQWaves) {
      turn();
      refill(base);
      for (int j = wave / side; j < kQWaves && base + j < x.b1; j += kQWaves / side)
        block(lds.ring[stage][j], base + j, masked_t);
      stage = stage == kQStages - 1 ? 0 : stage + 1;
    }
  };
  // (two loops: the compiler would make one of two variants in a loop, with the codes of a
  // block unpacked before it knows which)
  int base = x.b0;
  blocks(base, min(x.b1, open) - kQWaves + 1, std::false_type());
  blocks(base, x.b1, std::true_type());
  kv4_fence();
  __builtin_amdgcn_s_waitcnt(0);           // (copies that nobody waited for)
  kv4_fence();
#pragma unroll
  for (int t = 0; t < C; ++t) {
    st[t].l += wave_xor(st[t].l, 16);
    st[t].l += wave_xor(st[t].l, 32);
#pragma unroll
    for (int g = 0; g < kG; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) st[t].o[4 * g + e] -= st[t].corr[g];
  }
}

// x of the lanes 4 (R = 4) or 8 (R = 2, 4) before this one in its 16, around.
template <int kBy>
__device__ __forceinline__ float kv4_turned(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + kBy, 0xf, 0xf, false));
}
template <int R>
__device__ __forceinline__ float kv4_class_sum(float x) {
  if constexpr (R == 4) x += kv4_turned<4>(x);
  return x + kv4_turned<8>(x);
}

// Up to 16 / R pairs (R = 2, 4) against the blocks from x.b0 + 2 wave on, two of every eight.  Of the 16
// columns R each are a pair's: class jl = l16 / (16 / R) of them has the scores of pages jl, jl + R, ..
// (of the four that the wave has at a time; the matrix unit gives all columns all pages' scores, of
// which a lane takes its own), so that softmax works on no score twice, and columns of O^T that hold
// their classes' shares.  While four pages are worked on, the wave's next four are on their way.
template <int D, int R>
__device__ __forceinline__ void kv4_wave_few(const Kv4Args& a, const Kv4Piece& x, int h,
                                             Kv4Four<D>* lds, Kv4State<D>& st) {
  constexpr int kG = D / 64, kTurns = 4 / R, kCols = 16 / R;
  using P = Kv4Page<D>;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, wave = wave_id();
  const int jl = l16 / kCols;
  const int group = a.hq / a.hkv, pairs = x.rows * group;
  const float c = a.scale * kLog2e, tau = fminf(kRescaleLog2 / c, 1e30f);   // (finite at any scale)
  const Kv4Unpack unpack;

  // ---- copies ---------------------------------------------------------------------------------
  const int pages = min((x.kv_len + 15) / 16, 2 * x.b1);
  const int32_t* table = a.tables + (size_t)x.s * a.max_blocks;
  const size_t stride = (size_t)a.hkv * P::kBytes;
  const char* kc = (const char*)a.k_cache + (size_t)h * P::kBytes;
  const char* vc = (const char*)a.v_cache + (size_t)h * P::kBytes;
  const int piece = kG == 2 ? 16 * ((lane & ~3) | ((lane - g4) & 3)) : 16 * (lane & 31);
  const int param = P::kParams + lane % (16 * kG) * 4;
  int next[4];
  auto find = [&](int page) {              // (behind the last page: that one again)
#pragma unroll
    for (int j = 0; j < 4; ++j) next[j] = kv4_uniform(table, min(page + j, pages - 1));
  };
  auto pick = [](bool first, size_t a, size_t b) { return first ? a : b; };
  auto copy = [&](const char* cache, char* codes, uint32_t* params) {
    size_t id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) id[j] = (size_t)next[j] * stride;
    if constexpr (kG == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) dma16_stream(cache + id[j] + piece, codes + 8 * D * j);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        dma4_stream(cache + pick(lane < 32, id[2 * j], id[2 * j + 1]) + param, params + 64 * j);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        dma16_stream(cache + pick(lane < 32, id[2 * j], id[2 * j + 1]) + piece, codes + 16 * D * j);
      dma4_stream(cache + pick(lane < 32, pick(lane < 16, id[0], id[1]), pick(lane < 48, id[2], id[3])) +
                      param, params);
    }
  };
  int page = 2 * x.b0 + 4 * wave;
  const int end = 2 * x.b1;
  if (page < end) {
    find(page);
    copy(kc, lds[0].k, lds[0].kp);
    copy(vc, lds[0].v, lds[0].vp);
    find(page + 4 * kQWaves);
    copy(kc, lds[1].k, lds[1].kp);
    copy(vc, lds[1].v, lds[1].vp);
    find(page + 8 * kQWaves);
  }

  const int pair = min(l16 % kCols, pairs - 1), row = pair / group;
  const int last = min(x.kv_len - x.rows + row, kQKeys * x.b1 - 1);   // the last key of the lane's column
  const bf16_t* src = (const bf16_t*)a.q + ((size_t)(x.qb + row) * a.hq + h * group + pair % group) * D;
  bf16x8 q[2 * kG];
  bf16x8 qz[kG];                           // minus the sum of q, in three parts
#pragma unroll
  for (int g = 0; g < kG; ++g) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const u32x4 y = load16(src + 64 * g + 16 * g4 + 8 * w);
      q[2 * g + w] = as_bf16x8(y);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum += __uint_as_float(y[i] << 16) + __uint_as_float(y[i] & 0xffff0000u);
    }
    sum += wave_xor(sum, 16);
    sum += wave_xor(sum, 32);
    const float part0 = (float)(__bf16)-sum, part1 = (float)(__bf16)(-sum - part0);
    const float on = g4 == 0 ? 1.f : 0.f;
    qz[g] = to_bf16x8(part0 * on, part1 * on, (-sum - part0 - part1) * on, 0.f, 0.f, 0.f, 0.f, 0.f);
    st.corr[g] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  st.l = 0.f;
  st.m = -INFINITY;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) st.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int at = kG == 2 ? 16 * (4 * l16 + ((g4 + (l16 >> 2)) & 3)) : 8 * (4 * l16 + g4);

  auto taken = [&] {                       // what was read from LDS is in registers: it is filled again
    kv4_fence();
    __builtin_amdgcn_s_waitcnt(0xC07F);
    kv4_fence();
  };
  auto four = [&](Kv4Four<D>& r, auto masked_t) {
    constexpr bool masked = decltype(masked_t)::value;
    kv4_fence();
    __builtin_amdgcn_s_waitcnt(0x0F70 | Kv4Four<D>::kOps);     // (those of the next four may be out)
    kv4_fence();
    // ---- S^T = K Q^T -------------------------------------------------------------------------
    float sc[kTurns][4];
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        f32x4 mine = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const int pg = t * R + j;
          uint32_t code[2];
          kv4_read(code, r.k + 8 * D * pg + at + 8 * g);
          const uint32_t z = r.kp[(pg * kG + g) * 16 + l16], zz = __builtin_amdgcn_perm(z, z, 0x01000100u);
          // (a product of 16 channels would do, but an accumulator that passes from that shape to the
          // other needs a wait, which the compiler leaves out: half of such sums were wrong where the
          // two follow at once, none with 16 cycles between them)
          f32x4 acc = mfma16(kv4_operand(zz, zz, zz, zz), qz[g], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t y = code[w];
            acc = mfma16(kv4_operand(unpack(y, 0), unpack(y, 1), unpack(y, 2), unpack(y, 3)),
                         q[2 * g + w], acc);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[i] = j == 0 || jl == j ? acc[i] : mine[i];
        }
        const u32x4 kp = *reinterpret_cast<const u32x4*>(r.kp + ((t * R + jl) * kG + g) * 16 + 4 * g4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = kv4_scale(kp[i]);
          sc[t][i] = g == 0 ? s * mine[i] : fmaf(s, mine[i], sc[t][i]);
        }
      }
    taken();
    copy(kc, r.k, r.kp);
    // ---- softmax -------------------------------------------------------------------------------
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (masked && 16 * (page + t * R + jl) + 4 * g4 + i > last) sc[t][i] = -INFINITY;
        top = fmaxf(top, sc[t][i]);
      }
    if constexpr (R == 4) top = fmaxf(top, kv4_turned<4>(top));
    top = fmaxf(top, kv4_turned<8>(top));
    top = column_max(top);
    if (wave_any(top > st.m + tau)) {
      const float m = fmaxf(st.m, top);
      const float alpha = st.m == -INFINITY ? 0.f : fast_exp2((st.m - m) * c);
      st.l *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) st.o[i] *= alpha;
#pragma unroll
      for (int g = 0; g < kG; ++g) st.corr[g] *= alpha;
      st.m = m;
    }
    const float ref = st.m == -INFINITY ? 0.f : -st.m * c;
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[t][i] = fast_exp2(fmaf(sc[t][i], c, ref));
        st.l += sc[t][i];
      }
    // ---- O^T += V^T P^T ------------------------------------------------------------------------
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      u32x2 p[kTurns];                     // p', four keys of the lane's page
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const u32x4 vp = *reinterpret_cast<const u32x4*>(r.vp + ((t * R + jl) * kG + g) * 16 + 4 * g4);
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = sc[t][i] * kv4_scale(vp[i]);
          // (the scale of a key not seen may be NaN)
          if (masked && 16 * (page + t * R + jl) + 4 * g4 + i > last) y[i] = 0.f;
        }
        p[t] = __builtin_bit_cast(u32x2, to_bf16x4(y[0], y[1], y[2], y[3]));
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) {        // pages 2 m and 2 m + 1
        u32x4 b;
        uint32_t w[4], zz[4];              // two keys' units of group g, and their zero points
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int j = 2 * m + i;
          const u32x4 vz = *reinterpret_cast<const u32x4*>(r.vp + (j * kG + g) * 16 + 4 * g4);
          uint32_t v[2 * kG];
          kv4_read(v, r.v + 8 * D * j + at);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            b[2 * i + e] = jl == j % R ? p[j / R][e] : 0;
            uint32_t z0 = vz[2 * e], z1 = vz[2 * e + 1];
            if (masked) {                  // (zero points alike for all columns: none that is NaN)
              const int key = 16 * (page + j) + 4 * g4 + 2 * e;
              if (key >= x.kv_len || (z0 & 0x7f80u) == 0x7f80u) z0 = 0;
              if (key + 1 >= x.kv_len || (z1 & 0x7f80u) == 0x7f80u) z1 = 0;
            }
            zz[2 * i + e] = __builtin_amdgcn_perm(z1, z0, 0x05040100u);
            if constexpr (kG == 1)
              w[2 * i + e] = v[e];
            else
              w[2 * i + e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e],
                                                   g == 0 ? 0x05040100u : 0x07060302u);
          }
        }
        const bf16x8 pf = as_bf16x8(b);
        st.corr[g] = mfma16(kv4_operand(zz[0], zz[1], zz[2], zz[3]), pf, st.corr[g]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st.o[4 * g + e] = mfma16(kv4_operand(unpack(w[0], e), unpack(w[1], e), unpack(w[2], e),
                                               unpack(w[3], e)),
                                   pf, st.o[4 * g + e]);
      }
    }
    taken();
    copy(vc, r.v, r.vp);
    page += 4 * kQWaves;
    find(page + 8 * kQWaves);
  };
  // pages that all rows see whole, and that are the piece's
  const int whole = min((x.kv_len - x.rows + 1) / 16, end);
  int stage = 1;
  while (page + 4 <= whole) four(lds[stage ^= 1], std::false_type());
  while (page < end) four(lds[stage ^= 1], std::true_type());
  kv4_fence();
  __builtin_amdgcn_s_waitcnt(0);           // (copies that nobody waited for)
  kv4_fence();
  st.l = kv4_class_sum<R>(st.l);
  st.l += wave_xor(st.l, 16);
  st.l += wave_xor(st.l, 32);
#pragma unroll
  for (int g = 0; g < kG; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        st.o[4 * g + e][r] = kv4_class_sum<R>(st.o[4 * g + e][r] - st.corr[g][r]);
}

// Join of a cut tile's pieces: piece p's partials are at place 2 (first + p), + 1 for p = 0.  A wave has
// kRows rows' reads on their way at a time, of eight pieces each.
template <int D, int kRows>
__device__ __forceinline__ void kv4_join(const Kv4Args& a, const Kv4Piece& x, int h) {
  const int C = a.cols;
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63, group = a.hq / a.hkv;
  const int have = min(kQPairs, x.rows * group - x.tile * kQPairs);
  auto place = [&](int p) { return ((size_t)(2 * (x.first + p) + (p == 0)) * a.hkv + h) * C; };
  auto request = [&](float (&y)[8][kPer], int i, int p0) {
#pragma unroll
    for (int p = 0; p < 8; ++p)
      load_coherent_vec<kPer>(a.part_o + (place(min(p0 + p, x.n - 1)) + i) * D + lane * kPer, y[p]);
  };
  for (int i0 = wave_id(); i0 < have; i0 += kRows * kQWaves) {
    float lse[kRows], y[kRows][8][kPer];
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int i = min(i0 + t * kQWaves, have - 1);
      lse[t] = lane < x.n ? load_coherent(a.part_lse + place(lane) + i) : -INFINITY;
      request(y[t], i, 0);
    }
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int i = i0 + t * kQWaves;
      if (i >= have) break;
      float top = lse[t];
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) top = fmaxf(top, wave_xor(top, m));
      const float w = lse[t] == -INFINITY ? 0.f : fast_exp2(lse[t] - top);
      float sum = w;
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) sum += wave_xor(sum, m);
      float acc[kPer] = {};
      for (int p0 = 0; p0 < x.n; p0 += 8) {
        if (p0 > 0) request(y[t], i, p0);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
          const float wp = __uint_as_float(
              __builtin_amdgcn_readlane(__float_as_uint(w), min(p0 + p, kWave - 1)));
#pragma unroll
          for (int e = 0; e < kPer; ++e) acc[e] += p0 + p >= x.n || wp == 0.f ? 0.f : wp * y[t][p][e];
        }
      }
      const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
      const int pair = x.tile * kQPairs + i;
      bf16_t* o = (bf16_t*)a.o + ((size_t)(x.qb + pair / group) * a.hq + h * group + pair % group) * D;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const __bf16 z = (__bf16)(acc[e] * inv);
        o[lane * kPer + e] = __builtin_bit_cast(bf16_t, z);
      }
    }
  }
}

template <int D, int R, int C>
__device__ __forceinline__ void kv4_piece(const Kv4Args& a, const Kv4Piece& x, int h, Kv4Lds<D, R, C>& lds) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, wave = wave_id();
  const int group = a.hq / a.hkv, pair0 = x.tile * kQPairs, have = min(x.rows * group - pair0, kQPairs);
  // the waves: `side` of them beside each other, of 16 C pairs each
  const int side = C == 1 ? 1 : kv4_side(have), mine = wave % side;
  const float c = a.scale * kLog2e;
  auto keep = [&](const Kv4State<D>& st, int t) {
    if (l16 < 16 / R) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          lds.o[wave][16 * t + l16][64 * (i / 4) + 4 * (4 * g4 + r) + i % 4] = st.o[i][r];
      if (g4 == 0) {
        lds.m[wave][16 * t + l16] = st.m;
        lds.l[wave][16 * t + l16] = st.l;
      }
    }
  };
  // (waves beside each other may differ in their number of tiles; either way they pass the same number of
  // barriers: one for every kQWaves of the piece's blocks, and one behind them)
  if (C == 2 && have > 16 * (2 * mine + 1)) {
    if constexpr (C == 2) {
      Kv4State<D> st[2];
      kv4_wave<D, 2>(a, x, h, pair0 + 32 * mine, side, lds, st);
      __syncthreads();                     // (the blocks make room for the states)
      keep(st[0], 0);
      keep(st[1], 1);
    }
  } else {
    Kv4State<D> st[1];
    if constexpr (R == 1)
      kv4_wave<D, 1>(a, x, h, pair0 + 32 * mine, side, lds, st);
    else
      kv4_wave_few<D, R>(a, x, h, lds.four[wave], st[0]);
    __syncthreads();
    keep(st[0], 0);
  }
  __syncthreads();
  // (a wave has some rows' reads on their way at a time: one after another a row takes a microsecond)
  auto join = [&](auto side_t) {
    constexpr int kSide = decltype(side_t)::value, kStates = kQWaves / kSide;
    constexpr int kRows = R == 1 ? 4 : 4 / R;
    for (int i0 = wave; i0 < have; i0 += kRows * kQWaves) {
      float m[kRows][kStates], l[kRows][kStates], y[kRows][kStates][kPer];
#pragma unroll
      for (int t = 0; t < kRows; ++t) {
        const int i = min(i0 + t * kQWaves, have - 1), row = i % (16 * C), w0 = i / (16 * C);
#pragma unroll
        for (int k = 0; k < kStates; ++k) {
          const int w = w0 + k * kSide;
          m[t][k] = lds.m[w][row];
          l[t][k] = lds.l[w][row];
#pragma unroll
          for (int e = 0; e < kPer; ++e) y[t][k][e] = lds.o[w][row][lane * kPer + e];
        }
      }
#pragma unroll
      for (int t = 0; t < kRows; ++t) {
        const int i = i0 + t * kQWaves, pair = pair0 + i;
        if (i >= have) break;
        float top = m[t][0], sum = 0.f, acc[kPer] = {};
#pragma unroll
        for (int k = 1; k < kStates; ++k) top = fmaxf(top, m[t][k]);
#pragma unroll
        for (int k = 0; k < kStates; ++k) {
          const float f = m[t][k] == -INFINITY ? 0.f : fast_exp2((m[t][k] - top) * c);
          sum += m[t][k] == -INFINITY ? l[t][k] : f * l[t][k];
#pragma unroll
          for (int e = 0; e < kPer; ++e) acc[e] += f * y[t][k][e];
        }
        // (a sum that is NaN, from keys that are, stays: the row is NaN)
        const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
        if (x.n == 1) {
          bf16_t* o =
              (bf16_t*)a.o + ((size_t)(x.qb + pair / group) * a.hq + h * group + pair % group) * D;
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            const __bf16 z = (__bf16)(acc[e] * inv);
            o[lane * kPer + e] = __builtin_bit_cast(bf16_t, z);
          }
        } else {
          const size_t at = ((size_t)(2 * (x.first + x.p) + (x.p == 0)) * a.hkv + h) * a.cols + i;
#pragma unroll
          for (int e = 0; e < kPer; ++e)
            store_coherent(a.part_o + at * D + lane * kPer + e, acc[e] * inv);
          if (lane == 0)
            store_coherent(a.part_lse + at, sum > 0.f   ? top * c + __log2f(sum)
                                            : sum == sum ? -INFINITY
                                                         : sum);
        }
      }
    }
  };
  if (side == 1)
    join(std::integral_constant<int, 1>());
  else
    join(std::integral_constant<int, 2>());
  if (x.n == 1) return;
  // Every partial has gone out with device-coherent stores; once they have completed one
  // arrival is counted, and the workgroup that counts the last joins and clears the counter.
  wait_all_memory();
  __syncthreads();
  int* count = a.arrivals + (size_t)x.first * a.hkv + h;
  if (threadIdx.x == 0)
    lds.flag = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (lds.flag != x.n - 1) return;
  kv4_join<D, C == 2 ? 8 : 4 / R>(a, x, h);
  if (threadIdx.x == 0) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Pairs a sequence: up to 16 / R, or, with C = 2, any number.
template <int D, int R, int C>
__global__ __launch_bounds__(64 * kQWaves, 2) void kv4_decode_kernel(Kv4Args a) {
  __shared__ Kv4Lds<D, R, C> lds;
  const int h = blockIdx.x % a.hkv, unit = blockIdx.x / a.hkv;
  Kv4Plan plan;
  if (a.units > 0) kv4_plan(a, lds, plan);
  for (int at = 0;;) {
    Kv4Piece x;
    if (a.units > 0) {
      x = kv4_find(a, lds, plan, unit, at);
      if (x.s < 0) return;
      at = x.next;
      if (x.p < 0) continue;
    } else {                               // a workgroup for each tile
      x.s = unit / a.tiles;
      x.tile = unit % a.tiles;
      kv4_sequence(a, x.s, x.qb, x.rows, x.kv_len);
      if (x.tile * kQPairs >= x.rows * (a.hq / a.hkv)) return;
      x.b0 = x.p = x.first = 0;
      x.b1 = kv4_blocks(x.kv_len);
      x.n = 1;
    }
    kv4_piece<D, R, C>(a, x, h, lds);
    if (a.units == 0) return;
  }
}

}  // namespace

Kv4Shape kv4_shape(int num_seqs, int max_rows, int hq, int hkv, int max_blocks) {
  const int64_t pairs = (int64_t)max_rows * (hq / hkv);
  Kv4Shape t;
  t.cols = (int)std::min<int64_t>(pairs, kQPairs);
  t.tiles = (int)((pairs + kQPairs - 1) / kQPairs);
  t.units = num_seqs <= kKv4PlanSeqs ? std::max(kQWorkgroups / hkv, 1) : 0;
  // (counters; places among all blocks are counted in 32 bits; without pages there is nothing to cut)
  if (max_blocks == 0 || (int64_t)t.units * hkv > kKv4Counters ||
      (double)num_seqs * t.tiles * (max_blocks / 2 + 1 + kQStart) * kQMaxWeight > 1e9)
    t.units = 0;
  return t;
}

int64_t kv4_grid(const Kv4Shape& t, int num_seqs, int hkv) {
  return t.units > 0 ? (int64_t)t.units * hkv : (int64_t)num_seqs * t.tiles * hkv;
}

namespace {

template <int D>
void launch_kv4_d(const Kv4Args& a, const Kv4Shape& t, hipStream_t stream) {
  const dim3 grid((unsigned)kv4_grid(t, a.num_seqs, a.hkv)), block(64 * kQWaves);
  if (t.cols <= 4)
    kv4_decode_kernel<D, 4, 1><<<grid, block, 0, stream>>>(a);
  else if (t.cols <= 8)
    kv4_decode_kernel<D, 2, 1><<<grid, block, 0, stream>>>(a);
  else if (t.cols <= 16)
    kv4_decode_kernel<D, 1, 1><<<grid, block, 0, stream>>>(a);
  else
    kv4_decode_kernel<D, 1, 2><<<grid, block, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_kv4(const Kv4Args& a, const Kv4Shape& t, hipStream_t stream) {
  a.d == 64 ? launch_kv4_d<64>(a, t, stream) : launch_kv4_d<128>(a, t, stream);
  return hipGetLastError();
}

}  // namespace rag
