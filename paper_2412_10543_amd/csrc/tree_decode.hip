// Attention of trees of drafted tokens to a paged KV cache (gfx950): the
// queries of a sequence's n drafted nodes, its last n keys, see every key
// before them and the nodes that their mask names.
//
// A unit is (sequence, kv head, 128 rows, piece of the pages): its rows are the
// (node, q head of the group) pairs, node by node, so that every K/V byte is
// read once for all of them.  Pieces of one sequence write normalised partial
// outputs and their log-sum-exp, which a second kernel joins.
#include "common.h"
#include "draft.h"
#include "masked_tile.h"

namespace rag {

namespace {

constexpr int kTrRows = 32 * kMtWaves;

// What the lane's row sees.
struct TreeRows {
  const uint64_t* mask;         // its node's words
  int prior, n, words;          // keys before the nodes; nodes; words per node
  __device__ __forceinline__ FullBlocks full_blocks(const KeySpans& sp) const {
    return {max(prior - sp.a0, 0) / kMtKeys, 0, 0};
  }
  __device__ __forceinline__ uint64_t word(int w) const {
    return w >= 0 && w < words ? mask[w] : 0;
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
  int qb, n, group, h0, r0, kv_len, sp, n_sp;
  KeySpans spans;
  TreeRows rows;
  __device__ __forceinline__ int row() const {
    return r0 + 32 * wave_id() + (opaque_lane() & 31);
  }
  __device__ __forceinline__ size_t out() const {         // (query row, q head)
    const int r = min(row(), n * group - 1);
    return (size_t)(qb + r / group) * a.hq + h0 + r % group;
  }
  __device__ __forceinline__ void fetch(int) {}
  __device__ __forceinline__ KeySpans settle(int) {
    rows.mask = a.mask + (size_t)(qb + min(row(), n * group - 1) / group) * a.mask_words;
    rows.prior = kv_len - n;
    rows.n = n;
    rows.words = a.mask_words;
    return spans;
  }
  __device__ __forceinline__ const bf16_t* q(int) const { return (const bf16_t*)a.q + out() * D; }
  __device__ __forceinline__ void store(int, const PfState<D>& st, float l, float scale) const {
    const bool valid = row() < n * group;
    const size_t x = out();
    if (n_sp == 1) {
      mt_store<D>(st, (bf16_t*)a.o + x * D, valid);
      return;
    }
    const float lse = mt_lse(st, l, scale);
    if (!valid) return;
    const int half = opaque_lane() >> 5;
    float* o = a.part_o + (x * a.num_splits + sp) * D + 4 * half;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(o + 32 * dt + 8 * g) =
            f32x4{st.oacc[dt][4 * g], st.oacc[dt][4 * g + 1], st.oacc[dt][4 * g + 2],
                  st.oacc[dt][4 * g + 3]};
    if (half == 0) a.part_lse[x * a.num_splits + sp] = lse;
  }
};

struct TreeCoord {
  int s, kvh, rb, sp;
};

}  // namespace

// Unit order: the row blocks of one (sequence, kv head, piece) follow each other
// on one XCD, whose L2 then serves their K/V.
__device__ __forceinline__ bool tree_coord(const TreeArgs& a, int row_blocks, TreeCoord& t) {
  int xcd, local;
  xcd_slot(blockIdx.x, xcd, local);
  t.rb = local % row_blocks;
  const int64_t stream = xcd + (int64_t)kNumXcd * (local / row_blocks);
  const int64_t pairs = (int64_t)a.num_seqs * a.hkv;
  if (stream >= pairs * a.num_splits) return false;
  t.sp = (int)(stream / pairs);
  const int pr = (int)(stream % pairs);
  t.s = pr / a.hkv;
  t.kvh = pr % a.hkv;
  return true;
}

// Pieces that a sequence of kv_len keys is cut into, of pps pages each.
__device__ __forceinline__ int tree_pieces(const TreeArgs& a, int kv_len, int& pps) {
  pps = max(1, (a.max_blocks + a.num_splits - 1) / a.num_splits);
  pps = (pps + 1) & ~1;                          // whole blocks of 32 keys
  return max(1, ((kv_len + 15) / 16 + pps - 1) / pps);
}

template <int D>
__global__ __launch_bounds__(64 * kMtWaves, 2) void tree_kernel(TreeArgs a) {
  __shared__ __attribute__((aligned(16))) MtLds<D> lds;
  const int group = a.hq / a.hkv;
  TreeCoord t;
  if (!tree_coord(a, (a.max_nodes * group + kTrRows - 1) / kTrRows, t)) return;
  TreeSrc<D> src{a};
  src.qb = uniform_load(a.cu_q, t.s);
  src.n = uniform_load(a.cu_q, t.s + 1) - src.qb;
  src.r0 = t.rb * kTrRows;
  if (src.r0 >= src.n * group) return;
  const int nk = min(uniform_load(a.kv_lens, t.s), a.max_blocks * 16);
  int pps;
  src.n_sp = tree_pieces(a, nk, pps);
  if (t.sp >= src.n_sp || nk <= 0) return;
  src.sp = t.sp;
  src.group = group;
  src.h0 = t.kvh * group;
  src.kv_len = nk;
  const int k0 = t.sp * pps * 16, k1 = min(nk, k0 + pps * 16);
  src.spans = KeySpans{k0, (k1 - k0 + kMtKeys - 1) / kMtKeys, 0, 0};
  const PagedDmaKV<D> kv{(const bf16_t*)a.k_cache + (size_t)t.kvh * 16 * D,
                         (const bf16_t*)a.v_cache + (size_t)t.kvh * 16 * D,
                         a.tables + (size_t)t.s * a.max_blocks, (size_t)a.hkv * 16 * D};
  masked_items<D>(src, kv, nk, a.scale, lds);
}

// o = sum_i 2^(lse_i - m) o_i / sum_i 2^(lse_i - m): one wave per (node, q head).
template <int D>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  constexpr int kPer = D / 64;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int per = (a.max_nodes * a.hq + 3) / 4;  // workgroups of a sequence
  const int s = blockIdx.x / per;
  const int qb = a.cu_q[s], n = a.cu_q[s + 1] - qb;
  const int i = blockIdx.x % per * 4 + wave;     // (node, head) of the sequence
  if (i >= n * a.hq) return;
  const int nk = min(a.kv_lens[s], a.max_blocks * 16);
  int pps;
  const int n_sp = tree_pieces(a, nk, pps);
  if (n_sp == 1) return;
  const size_t row = (size_t)qb * a.hq + i;
  const float lse = lane < n_sp ? a.part_lse[row * a.num_splits + lane] : -INFINITY;
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
  const float* po = a.part_o + row * a.num_splits * D + lane * kPer;
  for (int k = 0; k < n_sp; ++k) {
    const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), k));
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] += wk * po[(size_t)k * D + e];
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const __bf16 b = (__bf16)(acc[e] * inv);
    ((bf16_t*)a.o)[row * D + lane * kPer + e] = __builtin_bit_cast(bf16_t, b);
  }
}

static int tree_row_blocks(int max_nodes, int group) {
  return (int)(((int64_t)max_nodes * group + kTrRows - 1) / kTrRows);
}

int tree_splits(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks, int requested) {
  (void)d;
  const int64_t units = (int64_t)num_seqs * hkv * std::max(1, tree_row_blocks(max_nodes, hq / hkv));
  int64_t n = requested > 0 ? requested : (512 + units - 1) / units;
  if (requested <= 0) n = std::min<int64_t>(n, std::max(1, max_blocks / 16));
  n = std::max<int64_t>(1, std::min<int64_t>({n, (int64_t)kTreeMaxSplits, (int64_t)(max_blocks + 1) / 2}));
  return (int)n;
}

static int64_t tree_join_grid(const TreeArgs& a) {
  return (int64_t)a.num_seqs * (((int64_t)a.max_nodes * a.hq + 3) / 4);
}

int64_t tree_grid(const TreeArgs& a) {
  const int64_t streams = (int64_t)a.num_seqs * a.hkv * a.num_splits;
  const int64_t units =
      (streams + kNumXcd - 1) / kNumXcd * kNumXcd * tree_row_blocks(a.max_nodes, a.hq / a.hkv);
  return std::max(units, a.num_splits > 1 ? tree_join_grid(a) : 0);   // (the larger of the launches)
}

template <int D>
static hipError_t launch_tree_d(const TreeArgs& a, hipStream_t stream) {
  const int64_t streams = (int64_t)a.num_seqs * a.hkv * a.num_splits;
  const int64_t grid =
      (streams + kNumXcd - 1) / kNumXcd * kNumXcd * tree_row_blocks(a.max_nodes, a.hq / a.hkv);
  hipLaunchKernelGGL(tree_kernel<D>, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a);
  if (a.num_splits > 1)
    hipLaunchKernelGGL(tree_join_kernel<D>, dim3((unsigned)tree_join_grid(a)), dim3(256), 0,
                       stream, a);
  return hipGetLastError();
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t stream) {
  return a.d == 64 ? launch_tree_d<64>(a, stream) : launch_tree_d<128>(a, stream);
}

}  // namespace rag
