// Attention of trees of drafted tokens to a paged KV cache (gfx950): the
// queries of a sequence's n drafted nodes, its last n keys, see every key
// before them and the nodes that their mask names.
//
// A unit is (piece of a sequence's keys, kv head, 128 rows): its rows are (node, q
// head of the group) pairs, node by node, so that every K/V byte is read once for
// 128 of them.  The pieces are cut on the GPU from the sequences' lengths: as many
// workgroups as the chip takes at a time get even shares of all blocks, which may
// end in one sequence and begin in another (tree_share); where a sequence has
// several pieces, they write normalised partial outputs and their log-sum-exp, which
// a second kernel joins.
//
// Measured (32 q / 8 kv heads of 128): 48 sequences of 700 to 10,304 keys and 5 to
// 12 nodes 149 us, K/V at 4.6 TB/s (HBM); 16 of 2,600 to 10,300 keys and 64 nodes 117
// us, 695 TFLOP/s (the tile loop 104 of them, the join 13); one of 4,782
// and 25 nodes 19.8 us: 15.2 for pieces of 8 or 9 blocks, of which the chain of
// lengths, page ids, first copies and queries takes 4, and 4.4 for the join.
#include "common.h"
#include "draft.h"
#include "masked_tile.h"

namespace rag {

namespace {

constexpr int kTrRows = 32 * kMtWaves;
// Blocks of a share, at least: a unit's start, end and join cost about
// as much as eight.  One sequence of 4,782 keys, 32 q / 8 kv heads, 25 nodes: 19.9 us;
// cut down to 4 blocks 19.7, for twice the partials, to 16 23.6, to 32 36.2.
constexpr int kTrMinBlocks = 8;

// With sequences for a chipful of units, or more, nothing is cut where the tables have
// fewer blocks than this (the join's launch would cost more: 64 sequences of 500 to
// 1500 keys and 8 nodes 61 us, cut 73; 256 of 1000 keys 199, cut 211).
constexpr int kTrLongBlocks = 64;

// Blocks that the start of a sequence in a unit counts for.  40 sequences of 600 keys
// and one of 20,000, 12 nodes: 51 us; with 3 blocks 60, with 6 or 14 57 (more short
// sequences are cut, or the long one less); 63 of 500 and one of 30,000, 8 nodes: 70,
// with 3, 6 or 14 71, 69 and 72; 96 of 700 to 10,304 and 200 of 2,048 keys the same.
// (Against a quota of blocks a piece and sequences apart: 48 of 700 to 10,304 keys
// 161 -> 149 us, 96 of them 519 -> 437, 63 and one 80 -> 70, but 200 of 2,048 325 -> 338.)
constexpr int kTrStart = 10;

// What the lane's row sees.
struct TreeRows {
  const uint64_t* mask;         // its node's words, the first two of them loaded
  uint64_t w0, w1;
  int prior, n, words;          // keys before the nodes; nodes; words per node
  __device__ __forceinline__ FullBlocks full_blocks(const KeySpans& sp) const {
    return {max(prior - sp.a0, 0) / kMtKeys, 0, 0};
  }
  __device__ __forceinline__ uint64_t word(int w) const {
    // (w is the same for the wave; a load waits for every copy in flight)
    if (w < 0 || w >= words) return 0;
    return w == 0 ? w0 : w == 1 ? w1 : mask[w];
  }
  __device__ __forceinline__ uint32_t seen(int k0) const {
    const int j0 = k0 - prior;                   // node of the block's first key (may be < 0)
    const int w = j0 >> 6, b = j0 & 63;
    uint64_t x = word(w) >> b;
    if (b > 32) x |= word(w + 1) << (64 - b);
    const uint32_t nodes = (uint32_t)x & low_bits(n - j0);
    return low_bits(-j0) | (nodes & ~low_bits(-j0));
  }
};

// The rows of a unit (one item): (node, q head of the group) pairs r0 + 32 wave on.
template <int D>
struct TreeSrc {
  const TreeArgs& a;
  static constexpr int count = 1;
  int qb, n, group, h0, r0, kv_len, n_sp;
  size_t unit;                  // of the partials
  KeySpans spans;
  TreeRows rows;
  // Row r of the wave's 32 is pair `pair(r)` of the sequence and kv head.
  __device__ __forceinline__ int pair(int r) const { return r0 + 32 * wave_id() + r; }
  __device__ __forceinline__ size_t at(int r) const {     // its element offset in q and o
    const int x = min(pair(r), n * group - 1);
    return ((size_t)(qb + x / group) * a.hq + h0 + x % group) * D;
  }
  __device__ __forceinline__ void fetch(int) {}
  __device__ __forceinline__ KeySpans settle(int) {
    const int x = min(pair(opaque_lane() & 31), n * group - 1);
    rows.mask = a.mask + (size_t)(qb + x / group) * a.mask_words;
    rows.prior = kv_len - n;
    rows.n = n;
    rows.words = a.mask_words;
    rows.w0 = rows.mask[0];
    rows.w1 = rows.mask[min(1, a.mask_words - 1)];
    return spans;
  }
  __device__ __forceinline__ const bf16_t* q(int, int r) const { return (const bf16_t*)a.q + at(r); }
  __device__ __forceinline__ void store(int, const PfState<D>& st, float l, float scale,
                                        bf16_t* io) const {
    if (n_sp == 1) {
      mt_store<D>(st, io, [&](int r) {
        return pair(r) < n * group ? (bf16_t*)a.o + at(r) : (bf16_t*)nullptr;
      });
      return;
    }
    const size_t first = unit * a.part_rows + 32 * wave_id();
    mt_store_f32<D>(st, io, [&](int r) {
      return pair(r) < n * group ? a.part_o + (first + r) * D : (float*)nullptr;
    });
    const float lse = mt_lse(st, l, scale);
    const int r = opaque_lane();
    if (r < 32 && pair(r) < n * group) a.part_lse[first + r] = lse;
  }
};

}  // namespace

// Blocks of a sequence with n nodes and kv_len keys.
__device__ __forceinline__ int tree_blocks(const TreeArgs& a, int n, int kv_len) {
  return n <= 0 ? 0 : (min(kv_len, a.max_blocks * 16) + kMtKeys - 1) / kMtKeys;
}

// Blocks [b0, b1) of sequence s (-1: no more), the p-th of its n pieces, and their
// place among the partials where n > 1; `first` for the join (tree_place).
struct TreePiece {
  int s, p, n, b0, b1, first;
  int qb, nodes, kv_len;        // of sequence s
  int next;                     // where in the unit the next piece starts
};

// The place of a sequence's piece p.
__device__ __forceinline__ int tree_place(const TreeArgs& a, int first, int p) {
  return a.splits > 0 ? first + p : 2 * (first + p) + (p == 0);
}

// With a number of splits given every sequence is cut into that many (or its
// blocks), and unit s * splits + p is sequence s's p-th piece.
__device__ __forceinline__ TreePiece tree_even(const TreeArgs& a, int unit, int at) {
  TreePiece t;
  t.s = unit / a.splits;
  t.p = unit % a.splits;
  t.first = unit - t.p;
  t.qb = uniform_load(a.cu_q, t.s);
  t.nodes = uniform_load(a.cu_q, t.s + 1) - t.qb;
  t.kv_len = uniform_load(a.kv_lens, t.s);
  const int64_t blocks = tree_blocks(a, t.nodes, t.kv_len);
  t.n = min(a.splits, max((int)blocks, 1));
  t.b0 = (int)(blocks * t.p / t.n);
  t.b1 = (int)(blocks * (t.p + 1) / t.n);
  t.next = 1;
  if (t.p >= t.n || at > 0) t.s = -1;
  return t;
}

// Inclusive prefix sums over the wave's lanes.
__device__ __forceinline__ int tree_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return x;
}

// Otherwise (at most kTreePlanSeqs sequences) all sequences' blocks, kTrStart more in
// front of each for what its start costs, stand in one row that is cut into even
// shares, one a unit: a unit has the end of a sequence, whole ones and the
// beginning of one, of which the first and the last may have partials (places 2 unit
// and 2 unit + 1).  The piece at `at` of the unit's share; wave-parallel, one lane per
// sequence, and every wave finds the same.
// The shares count key blocks, for the row blocks of max_nodes alike: where most trees
// are far smaller, the workgroups of the other row blocks have nothing to do (48 trees of
// up to 12 nodes, 32 q / 8 kv heads: 150 us, with max_nodes 64 192, with 128 311).  More
// than kTreePlanSeqs sequences (four a lane) would take a scan of a second level: 256 of
// 1,000 keys and one of 30,000 take 752 us, with one fewer 253.
template <int kChunks>
__device__ __forceinline__ TreePiece tree_share(const TreeArgs& a, int unit, int at) {
  const int lane = opaque_lane();
  int end[kChunks], len[kChunks], qb[kChunks], qe[kChunks], kv[kChunks], longest = 0, total = 0;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int s = c * kWave + lane, x = min(s, a.num_seqs - 1);
    qb[c] = a.cu_q[x];
    qe[c] = a.cu_q[x + 1];
    kv[c] = a.kv_lens[x];
    const int bl = s < a.num_seqs ? tree_blocks(a, qe[c] - qb[c], kv[c]) : 0;
    len[c] = bl > 0 ? bl + kTrStart : 0;
    longest = max(longest, len[c]);
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    end[c] = total + tree_scan(len[c]);
    total = __builtin_amdgcn_readlane(end[c], 63);
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) longest = max(longest, __shfl_xor(longest, m, kWave));
  // (of kTreeMaxSplits units at most that a sequence touches)
  const int share = max(max((total + a.units - 1) / a.units, kTrMinBlocks),
                        (longest + kTreeMaxSplits - 3) / (kTreeMaxSplits - 2));
  const int from = unit * share, to = min(from + share, total);
  TreePiece t{-1, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  const int g = from + at;
  if (from >= total || g >= to) return t;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const uint64_t here = __builtin_amdgcn_ballot_w64(g >= end[c] - len[c] && g < end[c]);
    if (here != 0) {
      const int l = __builtin_ctzll(here);
      const int e = __builtin_amdgcn_readlane(end[c], l);
      const int b = e - __builtin_amdgcn_readlane(len[c], l) + kTrStart;   // of its blocks
      t.s = c * kWave + l;
      t.first = b / share;
      t.n = (e - 1) / share - t.first + 1;
      t.p = unit - t.first;
      t.b0 = max(g - b, 0);
      t.b1 = max(min(e, to) - b, 0);
      t.next = min(e, to) - from;
      t.qb = __builtin_amdgcn_readlane(qb[c], l);
      t.nodes = __builtin_amdgcn_readlane(qe[c], l) - t.qb;
      t.kv_len = __builtin_amdgcn_readlane(kv[c], l);
    }
  }
  return t;
}

// Unit order: the row blocks of one (piece, kv head) follow each other on one XCD,
// whose L2 then serves their K/V.
template <int D, int kChunks>
__global__ __launch_bounds__(64 * kMtWaves, 2) void tree_kernel(TreeArgs a) {
  __shared__ __attribute__((aligned(16))) MtLds<D> lds;
  const int group = a.hq / a.hkv;
  int xcd, local;
  xcd_slot(blockIdx.x, xcd, local);
  const int rb = local % a.row_blocks;
  const int stream = xcd + kNumXcd * (local / a.row_blocks);
  const int kvh = stream % a.hkv, unit = stream / a.hkv;
  if (unit >= a.units) return;
#pragma unroll 1
  for (int at = 0;;) {
    TreePiece t;
    if constexpr (kChunks == 0) t = tree_even(a, unit, at); else t = tree_share<kChunks>(a, unit, at);
    const int s = __builtin_amdgcn_readfirstlane(t.s);
    if (s < 0) return;
    at = __builtin_amdgcn_readfirstlane(t.next);
    const int p = __builtin_amdgcn_readfirstlane(t.p), n_sp = __builtin_amdgcn_readfirstlane(t.n);
    const int b0 = __builtin_amdgcn_readfirstlane(t.b0), b1 = __builtin_amdgcn_readfirstlane(t.b1);
    if (b0 >= b1) continue;                      // (its start only, or no key)
    if (p == 0 && rb == 0 && kvh == 0 && threadIdx.x == 0 && a.part_of != nullptr)
      reinterpret_cast<int2*>(a.part_of)[s] = int2{t.first, t.n};   // for the join
    TreeSrc<D> src{a};
    src.qb = __builtin_amdgcn_readfirstlane(t.qb);
    src.n = __builtin_amdgcn_readfirstlane(t.nodes);
    src.r0 = rb * kTrRows;
    const int nk = min(__builtin_amdgcn_readfirstlane(t.kv_len), a.max_blocks * 16);
    if (src.r0 >= src.n * group) continue;
    src.n_sp = n_sp;
    src.unit = ((size_t)__builtin_amdgcn_readfirstlane(tree_place(a, t.first, p)) * a.hkv + kvh) *
                   a.row_blocks + rb;
    src.group = group;
    src.h0 = kvh * group;
    src.kv_len = nk;
    src.spans = KeySpans{b0 * kMtKeys, b1 - b0, 0, 0};
    const PagedDmaKV<D> kv{(const bf16_t*)a.k_cache + (size_t)kvh * 16 * D,
                           (const bf16_t*)a.v_cache + (size_t)kvh * 16 * D,
                           a.tables + (size_t)s * a.max_blocks, (size_t)a.hkv * 16 * D};
    masked_items<D>(src, kv, nk, a.scale, lds);
    __syncthreads();                             // (the next piece takes the same LDS)
  }
}

// o = sum_i 2^(lse_i - m) o_i / sum_i 2^(lse_i - m): one wave per kRows (node, q head)
// pairs.  Small launches are one chain of reads long, with a wave a pair (one tree of 25
// nodes, 32 heads: 19.8 us a call, by fours 22.1); where the waves would come in several
// rounds, four pairs share the chain (tree_join_rows: 16 trees of 64 nodes in about 3
// pieces 115.5 us a call, with a wave a pair 118.2).
template <int D, int kRows>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  constexpr int kPer = D / 64;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int per = (a.max_nodes * a.hq + 4 * kRows - 1) / (4 * kRows);   // workgroups of a sequence
  const int s = blockIdx.x / per;
  const int qb = uniform_load(a.cu_q, s), n = uniform_load(a.cu_q, s + 1) - qb;
  const int i0 = (blockIdx.x % per * 4 + wave) * kRows;   // the first (node, head) of the sequence
  if (i0 >= n * a.hq) return;
  if (uniform_load(a.kv_lens, s) <= 0) return;
  const int first = uniform_load(a.part_of, 2 * s), n_sp = uniform_load(a.part_of, 2 * s + 1);
  if (n_sp <= 1) return;
  const int group = a.hq / a.hkv;
  const size_t stride = (size_t)a.hkv * a.row_blocks * a.part_rows;     // rows between places
  size_t row[kRows];                             // in a place
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int i = min(i0 + j, n * a.hq - 1), node = i / a.hq, head = i % a.hq, kvh = head / group;
    const int r = node * group + head % group;   // row of the unit's row blocks
    row[j] = ((size_t)kvh * a.row_blocks + r / kTrRows) * a.part_rows + r % kTrRows;
  }
  // kBatch pieces requested at a time, the first beside the log-sum-exps.
  constexpr int kBatch = kRows == 1 ? 8 : 4;
  float lse[kRows], x[kRows][kBatch][kPer];
#pragma unroll
  for (int j = 0; j < kRows; ++j)
    lse[j] = lane < n_sp ? a.part_lse[row[j] + tree_place(a, first, lane) * stride] : -INFINITY;
  auto request = [&](int k0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (k0 + b < n_sp) {
        const float* po = a.part_o + tree_place(a, first, k0 + b) * stride * D + lane * kPer;
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
          for (int e = 0; e < kPer; ++e) x[j][b][e] = po[row[j] * D + e];
      }
  };
  request(0);
  float w[kRows], inv[kRows], acc[kRows][kPer] = {};
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    float mx = lse[j];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) mx = fmaxf(mx, wave_xor(mx, m));
    // (a NaN among them stays one: fmaxf drops it, the difference below does not)
    w[j] = lse[j] == -INFINITY ? 0.f : fast_exp2((lse[j] - mx) * kLog2e);
    float den = w[j];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) den += wave_xor(den, m);
    inv[j] = den == 0.f ? 0.f : 1.f / den;
  }
  for (int k0 = 0; k0 < n_sp; k0 += kBatch) {
    if (k0 > 0) request(k0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (k0 + b < n_sp) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
          const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w[j]), k0 + b));
#pragma unroll
          for (int e = 0; e < kPer; ++e) acc[j][e] += wk * x[j][b][e];
        }
      }
  }
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    if (i0 + j >= n * a.hq) break;
    bf16_t* o = (bf16_t*)a.o + ((size_t)qb * a.hq + i0 + j) * D + lane * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const __bf16 v = (__bf16)(acc[j][e] * inv[j]);
      o[e] = __builtin_bit_cast(bf16_t, v);
    }
  }
}

// Pairs of a wave of the join: four where there are more than 256 CUs hold waves for.
static int tree_join_rows(const TreeArgs& a) {
  return (int64_t)a.num_seqs * a.max_nodes * a.hq > 256 * 32 ? 4 : 1;
}

// Workgroups that are on the chip at a time (the LDS of two a CU, three at D = 64).
static int64_t tree_places(int d) { return (d == 64 ? 3 : 2) * 256; }

// Key blocks of the longest sequence.
static int64_t tree_longest(int max_blocks) { return ((int64_t)max_blocks + 1) / 2; }

TreeShape tree_shape(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks,
                     int requested) {
  TreeShape t{};
  const int64_t rows = (int64_t)max_nodes * (hq / hkv);
  t.row_blocks = (int)((rows + kTrRows - 1) / kTrRows);
  t.part_rows = (int)std::min<int64_t>(rows, kTrRows);
  const int64_t blocks = tree_longest(max_blocks);
  // (the plan's sums are 32-bit)
  if (requested > 0 || num_seqs > kTreePlanSeqs || num_seqs * (blocks + kTrStart) >= 1 << 30) {
    t.splits = (int)std::max<int64_t>(1, std::min<int64_t>({requested, kTreeMaxSplits, blocks}));
    t.units = t.places = (int64_t)num_seqs * t.splits;
    return t;
  }
  t.splits = 0;
  // As many units as are on the chip at a time.
  int64_t n = std::max<int64_t>(1, tree_places(d) / ((int64_t)hkv * t.row_blocks));
  n = std::min(n, num_seqs * std::max<int64_t>(1, blocks / kTrMinBlocks));
  if (n <= num_seqs && blocks < kTrLongBlocks) {                 // nothing to cut
    t.splits = 1;
    n = num_seqs;
  }
  t.units = n;
  t.places = 2 * n;
  return t;
}

size_t tree_partial_rows(const TreeShape& t, int hkv) {
  return t.splits == 1 ? 0 : (size_t)t.places * hkv * t.row_blocks * t.part_rows;
}

// No less than tree_partial_rows of a launch of these sizes or of smaller ones.  (The
// launch's own number goes up and down: with more rows the same workgroups make fewer
// units, and with more sequences none may be cut.)  Its units are limited as in
// tree_shape, by the chip and by the blocks; in each limit, times hkv * row_blocks, the
// sizes only add.
size_t tree_partial_rows_upto(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks,
                              int requested) {
  const TreeShape t = tree_shape(num_seqs, max_nodes, hq, hkv, d, max_blocks, requested);
  if (requested > 0) return tree_partial_rows(t, hkv);           // (adds with the sizes by itself)
  const int64_t pieces = tree_longest(max_blocks) / kTrMinBlocks;
  if (pieces <= 1) return 0;                                     // no sequence is ever cut
  const int64_t streams = (int64_t)hkv * t.row_blocks;
  const int64_t units = std::min(std::max(tree_places(d), streams),
                                 std::min(num_seqs, kTreePlanSeqs) * pieces * streams);
  return (size_t)(2 * units) * t.part_rows;
}

static int64_t tree_join_grid(const TreeArgs& a) {
  const int rows = 4 * tree_join_rows(a);
  return (int64_t)a.num_seqs * (((int64_t)a.max_nodes * a.hq + rows - 1) / rows);
}
static int64_t tree_units_grid(int64_t units, int hkv, int row_blocks) {
  return (units * hkv + kNumXcd - 1) / kNumXcd * kNumXcd * row_blocks;
}

int64_t tree_grid(const TreeShape& t, const TreeArgs& a) {
  return std::max(tree_units_grid(t.units, a.hkv, t.row_blocks),
                  t.splits == 1 ? 0 : tree_join_grid(a));        // (the larger of the launches)
}

template <int D>
static hipError_t launch_tree_d(const TreeArgs& a, hipStream_t stream) {
  const int64_t grid = tree_units_grid(a.units, a.hkv, a.row_blocks);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a);
  };
  if (a.splits > 0)
    go(tree_kernel<D, 0>);
  else if (a.num_seqs <= kWave)
    go(tree_kernel<D, 1>);
  else
    go(tree_kernel<D, kTreePlanSeqs / kWave>);
  if (a.part_o != nullptr) {
    auto join = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)tree_join_grid(a)), dim3(256), 0, stream, a);
    };
    tree_join_rows(a) == 4 ? join(tree_join_kernel<D, 4>) : join(tree_join_kernel<D, 1>);
  }
  return hipGetLastError();
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t stream) {
  return a.d == 64 ? launch_tree_d<64>(a, stream) : launch_tree_d<128>(a, stream);
}

}  // namespace rag
