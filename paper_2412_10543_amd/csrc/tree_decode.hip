// Attention of trees of drafted tokens to a paged KV cache (gfx950): the
// queries of a sequence's n drafted nodes, its last n keys, see every key
// before them and the nodes that their mask names.
//
// A unit is (piece of a sequence's keys, kv head, 128 rows): its rows are (node, q
// head of the group) pairs, node by node, so that every K/V byte is read once for
// 128 of them.  The pieces are cut on the GPU from the sequences' lengths, about
// as many units as the chip takes at a time and about equally long (tree_plan);
// where a sequence has several, they write normalised partial outputs and their
// log-sum-exp, which a second kernel joins.
//
// Measured (32 q / 8 kv heads of 128): 48 sequences of 700 to 10,304 keys and 5 to
// 12 nodes 156 us, K/V at 4.4 TB/s (HBM); 16 of 2,600 to 10,300 keys and 64 nodes 125
// us, 650 TFLOP/s (the tile loop, and pieces that are not all equal); one of 4,782
// and 25 nodes 19.8 us: 16.0 for pieces of 8 or 9 blocks, of which the chain of
// lengths, page ids, first copies and queries takes 4, and 4.4 for the join.
#include "common.h"
#include "draft.h"
#include "masked_tile.h"

namespace rag {

namespace {

constexpr int kTrRows = 32 * kMtWaves;
constexpr int kTrPlanSeqs = 256;     // sequences whose pieces are cut from their lengths
// Blocks that a piece is cut for, at least: a unit's start, end and join cost about
// as much as eight.  One sequence of 8192 keys, 32 q / 8 kv heads, 32 nodes: 19.9 us;
// cut down to 4 blocks 22.4, to 16 23.5, to 32 34.8.
constexpr int kTrMinBlocks = 8;

// With sequences for a chipful of units, or more, those are cut that are longer than
// twice an even share of a chipful, where the tables have at least this many blocks
// (or the join's launch would cost more): 63 sequences of 500 keys and one of 30,000,
// 8 nodes, 76 us (uncut 584); 64 of 4,096 keys 203 (198), 32 of 2,000 to 8,000 and 64
// nodes 227 (223; cut from one even share on 235).
constexpr int kTrLongBlocks = 64;

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

// Piece `pi` of the launch: sequence s (-1: there is no such piece), the p-th of
// its n pieces; `first` its first one's place among the partials (where n > 1).
struct TreePiece {
  int s, p, n, first;
  int qb, nodes, kv_len;        // of sequence s
};

// With a number of splits given every sequence is cut into that many (or its
// blocks), and piece s * splits + p is sequence s's p-th.
__device__ __forceinline__ TreePiece tree_piece_even(const TreeArgs& a, int pi) {
  TreePiece t;
  t.s = pi / a.splits;
  t.p = pi % a.splits;
  t.first = pi - t.p;
  t.qb = uniform_load(a.cu_q, t.s);
  t.nodes = uniform_load(a.cu_q, t.s + 1) - t.qb;
  t.kv_len = uniform_load(a.kv_lens, t.s);
  t.n = min(a.splits, max(tree_blocks(a, t.nodes, t.kv_len), 1));
  if (t.p >= t.n) t.s = -1;
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

// Otherwise (at most kTrPlanSeqs sequences) into pieces of at most a quota of blocks,
// from an even share of them on the smallest tried for which the pieces are at most
// a.pieces.  Wave-parallel, one lane per sequence; every wave finds the same.
template <int kChunks>
__device__ __forceinline__ TreePiece tree_plan(const TreeArgs& a, int pi) {
  const int lane = threadIdx.x & 63;
  int bl[kChunks], np[kChunks], pf[kChunks], qb[kChunks], qe[kChunks], kv[kChunks], longest = 0;
  float total = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int s = c * kWave + lane;
    const int x = min(s, a.num_seqs - 1);
    qb[c] = a.cu_q[x];
    qe[c] = a.cu_q[x + 1];
    kv[c] = a.kv_lens[x];
    bl[c] = tree_blocks(a, qe[c] - qb[c], kv[c]);
    if (s >= a.num_seqs) bl[c] = 0;
    longest = max(longest, bl[c]);
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c)
    total += (float)(uint32_t)__builtin_amdgcn_readlane(tree_scan(bl[c]), 63);
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) longest = max(longest, __shfl_xor(longest, m, kWave));
  // (single precision: every wave forms the same numbers, and any cut is a valid one)
  float q = fmaxf((float)kTrMinBlocks, fmaxf(total / (float)a.share,
                                             (float)longest / (float)kTreeMaxSplits));
  for (;;) {
    const float rq = 1.f / q;
    int count = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      np[c] = bl[c] > 0 ? min(max((int)ceilf((float)bl[c] * rq - 1e-3f), 1), kTreeMaxSplits) : 0;
      const int incl = tree_scan(np[c]);
      pf[c] = count + incl - np[c];
      count += __builtin_amdgcn_readlane(incl, 63);
    }
    // (from the longest on every sequence is one piece: at most num_seqs <= pieces)
    if (count <= a.pieces || q > (float)longest) break;
    q = fmaxf(q * 1.0625f, q + 1.f);
  }
  // Only sequences of several pieces have partials: a piece more than its share each,
  // which is more than one, so at most 2 a.share of them.
  int place[kChunks], places = 0;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int cut = np[c] > 1 ? np[c] : 0, incl = tree_scan(cut);
    place[c] = places + incl - cut;
    places += __builtin_amdgcn_readlane(incl, 63);
  }
  TreePiece t{-1, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const uint64_t at = __builtin_amdgcn_ballot_w64(pi >= pf[c] && pi < pf[c] + np[c]);
    if (at != 0) {
      const int l = __builtin_ctzll(at);
      t.s = c * kWave + l;
      t.first = __builtin_amdgcn_readlane(place[c], l);
      t.n = __builtin_amdgcn_readlane(np[c], l);
      t.p = pi - __builtin_amdgcn_readlane(pf[c], l);
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
  const int kvh = stream % a.hkv, pi = stream / a.hkv;
  if (pi >= a.pieces) return;
  TreePiece t;
  if constexpr (kChunks == 0) t = tree_piece_even(a, pi); else t = tree_plan<kChunks>(a, pi);
  const int s = __builtin_amdgcn_readfirstlane(t.s);
  if (s < 0) return;
  const int p = __builtin_amdgcn_readfirstlane(t.p), n_sp = __builtin_amdgcn_readfirstlane(t.n);
  if (p == 0 && rb == 0 && kvh == 0 && threadIdx.x == 0 && a.part_of != nullptr)
    reinterpret_cast<int2*>(a.part_of)[s] = int2{t.first, t.n};   // for the join
  TreeSrc<D> src{a};
  src.qb = __builtin_amdgcn_readfirstlane(t.qb);
  src.n = __builtin_amdgcn_readfirstlane(t.nodes);
  src.r0 = rb * kTrRows;
  const int nk = min(__builtin_amdgcn_readfirstlane(t.kv_len), a.max_blocks * 16);
  if (src.r0 >= src.n * group || nk <= 0) return;
  src.n_sp = n_sp;
  src.unit = ((size_t)(t.first + p) * a.hkv + kvh) * a.row_blocks + rb;
  src.group = group;
  src.h0 = kvh * group;
  src.kv_len = nk;
  const int64_t blocks = (nk + kMtKeys - 1) / kMtKeys;
  const int b0 = (int)(blocks * p / n_sp), b1 = (int)(blocks * (p + 1) / n_sp);
  src.spans = KeySpans{b0 * kMtKeys, b1 - b0, 0, 0};
  const PagedDmaKV<D> kv{(const bf16_t*)a.k_cache + (size_t)kvh * 16 * D,
                         (const bf16_t*)a.v_cache + (size_t)kvh * 16 * D,
                         a.tables + (size_t)s * a.max_blocks, (size_t)a.hkv * 16 * D};
  masked_items<D>(src, kv, nk, a.scale, lds);
}

// o = sum_i 2^(lse_i - m) o_i / sum_i 2^(lse_i - m): one wave per (node, q head).
template <int D>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  constexpr int kPer = D / 64;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int per = (a.max_nodes * a.hq + 3) / 4;  // workgroups of a sequence
  const int s = blockIdx.x / per;
  const int qb = uniform_load(a.cu_q, s), n = uniform_load(a.cu_q, s + 1) - qb;
  const int i = blockIdx.x % per * 4 + wave;     // (node, head) of the sequence
  if (i >= n * a.hq) return;
  if (uniform_load(a.kv_lens, s) <= 0) return;
  const int first = uniform_load(a.part_of, 2 * s), n_sp = uniform_load(a.part_of, 2 * s + 1);
  if (n_sp <= 1) return;
  const int group = a.hq / a.hkv, node = i / a.hq, head = i % a.hq, kvh = head / group;
  const int r = node * group + head % group;     // row of the unit's row blocks
  const size_t stride = (size_t)a.hkv * a.row_blocks * a.part_rows;     // rows between pieces
  const size_t row = (((size_t)first * a.hkv + kvh) * a.row_blocks + r / kTrRows) * a.part_rows +
                     r % kTrRows;
  // kBatch pieces requested at a time, the first beside the log-sum-exps.
  constexpr int kBatch = 8;
  const float lse = lane < n_sp ? a.part_lse[row + lane * stride] : -INFINITY;
  const float* po = a.part_o + row * D + lane * kPer;
  float x[kBatch][kPer];
  auto request = [&](int k0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[b][e] = po[min(k0 + b, n_sp - 1) * stride * D + e];
  };
  request(0);
  float mx = lse;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) mx = fmaxf(mx, wave_xor(mx, m));
  // (a NaN among them stays one: fmaxf drops it, the difference below does not)
  const float w = lse == -INFINITY ? 0.f : fast_exp2((lse - mx) * kLog2e);
  float den = w;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) den += wave_xor(den, m);
  const float inv = den == 0.f ? 0.f : 1.f / den;
  float acc[kPer] = {};
  for (int k0 = 0; k0 < n_sp; k0 += kBatch) {
    if (k0 > 0) request(k0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const float wk = __uint_as_float(
          __builtin_amdgcn_readlane(__float_as_uint(w), min(k0 + b, n_sp - 1)));
      if (k0 + b < n_sp) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] += wk * x[b][e];
      }
    }
  }
  bf16_t* o = (bf16_t*)a.o + ((size_t)qb * a.hq + i) * D + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const __bf16 b = (__bf16)(acc[e] * inv);
    o[e] = __builtin_bit_cast(bf16_t, b);
  }
}

TreeShape tree_shape(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks,
                     int requested) {
  TreeShape t{};
  const int64_t rows = (int64_t)max_nodes * (hq / hkv);
  t.row_blocks = (int)((rows + kTrRows - 1) / kTrRows);
  t.part_rows = (int)std::min<int64_t>(rows, kTrRows);
  const int64_t blocks = ((int64_t)max_blocks + 1) / 2;          // of the longest sequence
  if (requested > 0 || num_seqs > kTrPlanSeqs) {
    t.splits = (int)std::max<int64_t>(1, std::min<int64_t>({requested, kTreeMaxSplits, blocks}));
    t.pieces = t.places = (int64_t)num_seqs * t.splits;
    return t;
  }
  t.splits = 0;
  // As many units as are on the chip at a time (the LDS of two workgroups a CU, three
  // at D = 64).
  const int64_t units = (d == 64 ? 3 : 2) * 256;
  int64_t n = std::max<int64_t>(1, units / ((int64_t)hkv * t.row_blocks));
  n = std::min(n, num_seqs * std::max<int64_t>(1, blocks / kTrMinBlocks));
  n = std::min<int64_t>(n, (int64_t)num_seqs * kTreeMaxSplits);
  if (n > num_seqs) {
    t.share = t.pieces = t.places = n;
  } else if (blocks >= kTrLongBlocks) {
    t.share = (n + 1) / 2;
    t.pieces = num_seqs + t.share;
    t.places = 2 * t.share;
  } else {
    t.pieces = num_seqs;
  }
  if (t.pieces == num_seqs) t.splits = 1;                        // nothing to cut
  return t;
}

size_t tree_partial_rows(const TreeShape& t, int hkv) {
  return t.splits == 1 ? 0 : (size_t)t.places * hkv * t.row_blocks * t.part_rows;
}

static int64_t tree_join_grid(const TreeArgs& a) {
  return (int64_t)a.num_seqs * (((int64_t)a.max_nodes * a.hq + 3) / 4);
}
static int64_t tree_units_grid(int64_t pieces, int hkv, int row_blocks) {
  return (pieces * hkv + kNumXcd - 1) / kNumXcd * kNumXcd * row_blocks;
}

int64_t tree_grid(const TreeShape& t, const TreeArgs& a) {
  return std::max(tree_units_grid(t.pieces, a.hkv, t.row_blocks),
                  t.splits == 1 ? 0 : tree_join_grid(a));        // (the larger of the launches)
}

template <int D>
static hipError_t launch_tree_d(const TreeArgs& a, hipStream_t stream) {
  const int64_t grid = tree_units_grid(a.pieces, a.hkv, a.row_blocks);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a);
  };
  if (a.splits > 0)
    go(tree_kernel<D, 0>);
  else if (a.num_seqs <= kWave)
    go(tree_kernel<D, 1>);
  else
    go(tree_kernel<D, kTrPlanSeqs / kWave>);
  if (a.part_o != nullptr)
    hipLaunchKernelGGL(tree_join_kernel<D>, dim3((unsigned)tree_join_grid(a)), dim3(256), 0,
                       stream, a);
  return hipGetLastError();
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t stream) {
  return a.d == 64 ? launch_tree_d<64>(a, stream) : launch_tree_d<128>(a, stream);
}

}  // namespace rag
