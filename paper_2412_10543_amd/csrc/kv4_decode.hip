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
// Blocks of two pages (32 keys) are copied straight into LDS, kQStages - 1 of them ahead, with
// 16 bytes a lane and lanes in the pages' order, parameters with a load of their lines: a load that
// finds a line still on its way holds up all behind it (64 sequences of 2.6k to 10.3k keys: 98 us
// with the codes loaded as the matrix operands have them, 113 with the parameters' lines read
// where they are needed).  Each of a workgroup's four waves copies every fourth block.  Up to 16
// pairs, each attends the blocks that it has copied; for up to 32, two and two do with 16 pairs
// each every second block; for up to 64 all four do every block.  They join their states through
// LDS.  As many workgroups as the chip takes at a time get even shares of all sequences' blocks;
// a sequence that is cut writes partial outputs and log-sum-exps, which the last of its
// workgroups to finish joins.
#include "common.h"
#include "kv4.h"
#include "serve.h"

#include <type_traits>

namespace rag {

namespace {

constexpr int kQWaves = 4;
constexpr int kQKeys = 32;                 // keys of a block
constexpr int kQPairs = 16 * kQWaves;      // pairs of a tile, at most
constexpr int kQMinBlocks = 8;             // blocks of a share, at least
constexpr int kQStart = 6;                 // blocks that the start of a tile counts for
constexpr int kQMaxPieces = 64;            // of a tile (one lane each in the join)
constexpr int kQWorkgroups = 512;          // about two a CU

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

#ifndef STAGES
#define STAGES 3
#endif
constexpr int kQStages = STAGES;

// A block in LDS: K codes of its two pages, V codes, parameters [page][K, V][group][token].
template <int D>
struct Kv4Block {
  char k[16 * D], v[16 * D];
  uint32_t p[D];
  static constexpr int kOps = D == 128 ? 6 : 3;      // loads that fill one
};

template <int D>
struct Kv4Lds {
  union {
    Kv4Block<D> ring[kQStages][kQWaves];
    float o[kQWaves][16][D + 4];
  };
  float m[kQWaves][16], l[kQWaves][16];
  int start[kKv4PlanSeqs], span[kKv4PlanSeqs], len[kKv4PlanSeqs];   // (a thread's own four each)
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

__device__ __forceinline__ void kv4_sequence(const Kv4Args& a, int s, int& qb, int& rows, int& kv) {
  qb = a.cu_q != nullptr ? a.cu_q[s] : s;
  rows = a.cu_q != nullptr ? a.cu_q[s + 1] - qb : 1;
  kv = min(a.kv_lens[s], a.max_blocks * 16);
}

__device__ __forceinline__ int kv4_blocks(int kv_len) {
  return (max(kv_len, 0) + kQKeys - 1) / kQKeys;
}

// The sequences' places in one row of all blocks, kQStart more in front of each tile.
template <class Lds>
__device__ __forceinline__ void kv4_plan(const Kv4Args& a, Lds& lds, Kv4Plan& plan) {
  const int group = a.hq / a.hkv;
  int sum = 0, longest = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = threadIdx.x * 4 + i;
    int tiles = 0, len = 0;
    if (s < a.num_seqs) {
      int qb, rows, kv;
      kv4_sequence(a, s, qb, rows, kv);
      tiles = (max(rows, 0) * group + kQPairs - 1) / kQPairs;
      len = kv4_blocks(kv) + kQStart;
    }
    lds.start[s] = sum;
    lds.span[s] = tiles * len;
    lds.len[s] = len;
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
  for (int i = 0; i < 4; ++i) lds.start[threadIdx.x * 4 + i] += before;
  // (a tile is cut into at most kQMaxPieces)
  plan.share = max(max((plan.total + a.units - 1) / a.units, kQMinBlocks),
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
    if (off >= 0 && off < lds.span[s]) {
      Kv4Piece x;
      x.s = s;
      x.tile = off / lds.len[s];
      const int t0 = lds.start[s] + x.tile * lds.len[s], t1 = t0 + lds.len[s];
      x.b0 = max(g - t0 - kQStart, 0);
      x.b1 = max(min(to, t1) - t0 - kQStart, 0);
      x.first = t0 / plan.share;
      x.n = (t1 - 1) / plan.share - x.first + 1;
      x.p = unit - x.first;
      x.next = min(to, t1) - from;
      kv4_sequence(a, x.s, x.qb, x.rows, x.kv_len);
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

// The wave's 16 pairs (pair0 on) against the piece's blocks, `side` waves beside each other on each
// of them; a wave whose pairs are none copies its blocks for the others.
template <int D>
__device__ __forceinline__ void kv4_wave(const Kv4Args& a, const Kv4Piece& x, int h, int pair0, int side,
                                         Kv4Lds<D>& lds, Kv4State<D>& st) {
  constexpr int kG = D / 64;
  using P = Kv4Page<D>;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, wave = wave_id();
  const int group = a.hq / a.hkv, pairs = x.rows * group;
  const float c = a.scale * kLog2e, tau = kRescaleLog2 / c;
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
      dma16(kc + id0 + piece, (bf16_t*)to.k);
      dma16(kc + id1 + piece, (bf16_t*)(to.k + 8 * D));
      dma4(pc + id0, to.p);
      dma4(pc + id1, to.p + 64);
      dma16(vc + id0 + piece, (bf16_t*)to.v);
      dma16(vc + id1 + piece, (bf16_t*)(to.v + 8 * D));
    } else {
      const size_t id = lane < 32 ? id0 : id1;
      dma16(kc + id + piece, (bf16_t*)to.k);
      dma4(pc + id, to.p);
      dma16(vc + id + piece, (bf16_t*)to.v);
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

  const int pair = min(pair0 + l16, pairs - 1), row = pair / group;
  const int last = x.kv_len - x.rows + row;        // the last key that the lane's column sees
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

  // where the lane's operands stand in a page's codes
  const int at = kG == 2 ? 16 * (4 * l16 + ((g4 + (l16 >> 2)) & 3)) : 8 * (4 * l16 + g4);
  auto block = [&](const Kv4Block<D>& r, int b, auto masked_t) {
    constexpr bool masked = decltype(masked_t)::value;
    const int key0 = kQKeys * b;
    const uint32_t* params = r.p;
    // ---- S^T = K Q^T ---------------------------------------------------------------
    float sc[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t code[2 * kG];
      kv4_read(code, r.k + 8 * D * j + at);
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const uint32_t kz = params[kv4_place<D>(j, 0, g) + l16];
        const uint32_t zz = __builtin_amdgcn_perm(kz, kz, 0x01000100u);
        f32x4 acc = mfma16(kv4_operand(zz, zz, zz, zz), qz[g], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t y = code[2 * g + w];
          acc = mfma16(kv4_operand(unpack(y, 0), unpack(y, 1), unpack(y, 2), unpack(y, 3)),
                       q[2 * g + w], acc);
        }
        const u32x4 kp = *reinterpret_cast<const u32x4*>(params + kv4_place<D>(j, 0, g) + 4 * g4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = kv4_scale(kp[i]);
          sc[4 * j + i] = g == 0 ? s * acc[i] : fmaf(s, acc[i], sc[4 * j + i]);
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
        if (key > last) sc[i] = -INFINITY;
#pragma unroll
        for (int g = 0; g < kG; ++g) {     // (zero points alike for all columns: none that is NaN)
          const uint32_t y = key < x.kv_len ? vp[i / 4][g][i % 4] : 0;
          vp[i / 4][g][i % 4] = (y & 0x7f80u) == 0x7f80u ? y & 0xffff0000u : y;
        }
      }
    }
    // ---- softmax ------------------------------------------------------------------------
    float top = sc[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i]);
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
    for (int i = 0; i < 8; ++i) {
      sc[i] = fast_exp2(fmaf(sc[i], c, ref));
      st.l += sc[i];
    }
    // ---- O^T += V^T P^T ---------------------------------------------------------------------
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = sc[i] * kv4_scale(vp[i / 4][g][i % 4]);
      if constexpr (masked) {              // (the scale of a key not seen may be NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (key0 + 16 * (i / 4) + 4 * g4 + i % 4 > last) y[i] = 0.f;
      }
      const bf16x8 pf = to_bf16x8(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
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
      st.corr[g] = mfma16(kv4_operand(zz[0], zz[1], zz[2], zz[3]), pf, st.corr[g]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        st.o[4 * g + e] = mfma16(kv4_operand(unpack(w[0], e), unpack(w[1], e), unpack(w[2], e),
                                             unpack(w[3], e)),
                                 pf, st.o[4 * g + e]);
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
  const bool active = pair0 < pairs;
  const int open = (x.kv_len - x.rows + 1) / kQKeys;     // blocks that all rows see whole
  auto blocks = [&](int& base, int to, auto masked_t) {
    for (; base < to; base += kQWaves) {
      turn();
      refill(base);
      if (active)
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
  st.l += wave_xor(st.l, 16);
  st.l += wave_xor(st.l, 32);
#pragma unroll
  for (int g = 0; g < kG; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[4 * g + e] -= st.corr[g];
}

// Join of a cut tile's pieces: piece p's partials are at place 2 (first + p), + 1 for p = 0.
template <int D>
__device__ __forceinline__ void kv4_join(const Kv4Args& a, const Kv4Piece& x, int h) {
  const int C = a.cols;
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63, group = a.hq / a.hkv;
  const int have = min(kQPairs, x.rows * group - x.tile * kQPairs);
  auto place = [&](int p) { return ((size_t)(2 * (x.first + p) + (p == 0)) * a.hkv + h) * C; };
  for (int i = threadIdx.x >> 6; i < have; i += kQWaves) {
    const float lse = lane < x.n ? load_coherent(a.part_lse + place(lane) + i) : -INFINITY;
    float top = lse;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) top = fmaxf(top, wave_xor(top, m));
    const float w = lse == -INFINITY ? 0.f : fast_exp2(lse - top);
    float sum = w;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += wave_xor(sum, m);
    float acc[kPer] = {};
    for (int p = 0; p < x.n; ++p) {
      float y[kPer];
      load_coherent_vec<kPer>(a.part_o + (place(p) + i) * D + lane * kPer, y);
      const float wp = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p));
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += wp == 0.f ? 0.f : wp * y[e];
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
    const int pair = x.tile * kQPairs + i;
    bf16_t* o = (bf16_t*)a.o + ((size_t)(x.qb + pair / group) * a.hq + h * group + pair % group) * D;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const __bf16 y = (__bf16)(acc[e] * inv);
      o[lane * kPer + e] = __builtin_bit_cast(bf16_t, y);
    }
  }
}

template <int D>
__device__ __forceinline__ void kv4_piece(const Kv4Args& a, const Kv4Piece& x, int h, Kv4Lds<D>& lds) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, wave = wave_id();
  const int group = a.hq / a.hkv, pair0 = x.tile * kQPairs, have = min(x.rows * group - pair0, kQPairs);
  // the waves: `side` column tiles of 16 pairs beside each other
  const int side = have <= 16 ? 1 : have <= 32 ? 2 : 4, mine = wave % side;
  const float c = a.scale * kLog2e;
  {
    Kv4State<D> st;
    kv4_wave<D>(a, x, h, pair0 + 16 * mine, side, lds, st);
    __syncthreads();                       // (the blocks make room for the states)
    if (16 * mine < have) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          lds.o[wave][l16][64 * (i / 4) + 4 * (4 * g4 + r) + i % 4] = st.o[i][r];
      if (g4 == 0) {
        lds.m[wave][l16] = st.m;
        lds.l[wave][l16] = st.l;
      }
    }
  }
  __syncthreads();
  for (int i = wave; i < have; i += kQWaves) {
    const int pair = pair0 + i, row = i % 16;
    float top = -INFINITY, sum = 0.f, acc[kPer] = {};
    for (int w = i / 16; w < kQWaves; w += side) top = fmaxf(top, lds.m[w][row]);
    for (int w = i / 16; w < kQWaves; w += side) {
      const float m = lds.m[w][row], f = m == -INFINITY ? 0.f : fast_exp2((m - top) * c);
      sum += m == -INFINITY ? lds.l[w][row] : f * lds.l[w][row];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += f * lds.o[w][row][lane * kPer + e];
    }
    // (a sum that is NaN, from keys that are, stays: the row is NaN)
    const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
    if (x.n == 1) {
      bf16_t* o = (bf16_t*)a.o + ((size_t)(x.qb + pair / group) * a.hq + h * group + pair % group) * D;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const __bf16 y = (__bf16)(acc[e] * inv);
        o[lane * kPer + e] = __builtin_bit_cast(bf16_t, y);
      }
    } else {
      const size_t at = ((size_t)(2 * (x.first + x.p) + (x.p == 0)) * a.hkv + h) * a.cols + i;
#pragma unroll
      for (int e = 0; e < kPer; ++e) store_coherent(a.part_o + at * D + lane * kPer + e, acc[e] * inv);
      if (lane == 0)
        store_coherent(a.part_lse + at, sum > 0.f   ? top * c + __log2f(sum)
                                        : sum == sum ? -INFINITY
                                                     : sum);
    }
  }
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
  kv4_join<D>(a, x, h);
  if (threadIdx.x == 0) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

#ifndef OCC
#define OCC 2
#endif
template <int D>
__global__ __launch_bounds__(64 * kQWaves, OCC) void kv4_decode_kernel(Kv4Args a) {
  __shared__ Kv4Lds<D> lds;
  const int h = blockIdx.x % a.hkv, unit = blockIdx.x / a.hkv;
  Kv4Plan plan;
  if (a.units > 0) kv4_plan(a, lds, plan);
  for (int at = 0;;) {
    Kv4Piece x;
    if (a.units > 0) {
      x = kv4_find(a, lds, plan, unit, at);
      if (x.s < 0) return;
      at = x.next;
    } else {                               // a workgroup for each tile
      x.s = unit / a.tiles;
      x.tile = unit % a.tiles;
      kv4_sequence(a, x.s, x.qb, x.rows, x.kv_len);
      if (x.tile * kQPairs >= x.rows * (a.hq / a.hkv)) return;
      x.b0 = x.p = x.first = 0;
      x.b1 = kv4_blocks(x.kv_len);
      x.n = 1;
    }
    kv4_piece<D>(a, x, h, lds);
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
  // (counters; places among all blocks are counted in 32 bits)
  if ((int64_t)t.units * hkv > kKv4Counters ||
      (double)num_seqs * t.tiles * (max_blocks / 2 + 1 + kQStart) > 1e9)
    t.units = 0;
  return t;
}

int64_t kv4_grid(const Kv4Shape& t, int num_seqs, int hkv) {
  return t.units > 0 ? (int64_t)t.units * hkv : (int64_t)num_seqs * t.tiles * hkv;
}

hipError_t launch_kv4(const Kv4Args& a, const Kv4Shape& t, hipStream_t stream) {
  const dim3 grid((unsigned)kv4_grid(t, a.num_seqs, a.hkv)), block(64 * kQWaves);
  if (a.d == 64)
    kv4_decode_kernel<64><<<grid, block, 0, stream>>>(a);
  else
    kv4_decode_kernel<128><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rag
