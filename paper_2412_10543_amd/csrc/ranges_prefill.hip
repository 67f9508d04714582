// Packed variable-length attention with a key range per query row (gfx950): the
// row at position p of its sequence sees the keys j < shared and the keys
// start <= j <= p.  Documents that do not see one another, prefixes seen by
// every row, windows with a few first keys.
//
// A workgroup is one tile of query rows of up to four heads of a GQA group, as
// in the causal prefill; it visits the key tiles of two spans only: up to its
// rows' largest `shared`, and from their smallest `start` to their last
// position.
//
// Measured (32 q / 8 kv heads of 128): 16 prompts of 5 to 20 documents of 400 to
// 512 tokens and 64 query rows 0.88 ms, 567 TFLOP/s of visible pairs, matrix
// cores 34%, vector issue 40% and LDS 23% busy: the waves' chains of one slot
// after another, and the starts and ends of tiles of 14 blocks, bound it.  One
// prompt of nine documents 88 us: its query's tiles, 150 blocks at 0.6 us one
// after another (the others are done after 58).  Those tiles cut in two halves of
// keys by pairs of waves, joined in LDS, took 86 with rings of two blocks (the batch
// 1007 us) and 90 with a CU for each workgroup and rings of four.
#include <climits>

#include "common.h"
#include "draft.h"
#include "masked_tile.h"

namespace rag {

namespace {

// Tiles of every sequence that are dispatched first: those of a prompt's query, which
// sees all its documents, would end a launch alone.  16 prompts of 5 to 20 documents
// and 64 query rows (three tiles of 32): one first 1072 us, two 1010, four 877, six 878,
// eight 882; 128 query rows (five tiles): one 1161, two 1090, four 1117, six 976, eight
// 979.
constexpr int kRgLast = 6;
// Of the others a workgroup takes kRgItems where there are at least kRgMany (eight
// for each place of the GPU): 21800 tiles of 14 blocks 916 us one by one, 880 by twos,
// 885 by fours; the same prompts with windows of 512 keys 1196, 1160 and 1170; but 1024
// rows with 8192 keys 142 us one by one, 257 and 503.
constexpr int kRgItems = 2;
constexpr int64_t kRgMany = 4096;

// Maximum over the wave of values from 0 on.
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));   // row_shr:1
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));   // row_shr:2
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));   // row_shr:4
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));   // row_shr:8
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // row_bcast:15
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // row_bcast:31
  return __builtin_amdgcn_readlane(x, 63);
}

// What a row sees: keys below shared, and start..last (start kNoStart: none).
constexpr int kNoStart = 1 << 30;
struct RowRange {
  int shared, start;
};
__device__ __forceinline__ RowRange row_range(int2 r, int last, int nk) {
  return {min(max(r.x, 0), nk), r.y > last || last < 0 ? kNoStart : max(r.y, 0)};
}

// The lane's row, and for the tile's rows what makes a block full.
struct RangeRows {
  RowRange r;
  int last;
  int shared_min, start_max, last_min;
  __device__ __forceinline__ FullBlocks full_blocks(const KeySpans& sp) const {
    const int by = sp.nb > 0 ? sp.na - sp.b0 / kMtKeys : 0;
    return {min(shared_min / kMtKeys, sp.na), (start_max + kMtKeys - 1) / kMtKeys + by,
            (last_min + 1) / kMtKeys + by};
  }
  __device__ __forceinline__ uint32_t seen(int k0) const {
    return low_bits(r.shared - k0) | (low_bits(last + 1 - k0) & ~low_bits(r.start - k0));
  }
};

// Smallest and largest of a value from 0 on over the wave; mostly it is one.
__device__ __forceinline__ void wave_bounds(int x, int y, int& lo, int& hi) {
  lo = hi = __builtin_amdgcn_readfirstlane(x);
  if (__builtin_amdgcn_ballot_w64(x != lo || y != lo) != 0) {
    lo = INT_MAX - wave_max(INT_MAX - min(x, y));
    hi = wave_max(max(x, y));
  }
}

// Query tiles t0, t0 + 1, ... of one sequence and head group.
template <int D>
struct RangeSrc {
  using Rows = RangeRows;
  const RangesArgs& a;
  int count, t0, qb, nq, nk, h0, hw, tile_rows;
  Rows rows;
  int2 own, some, more;         // ranges of the lane's row, and of the tile's rows
  __device__ __forceinline__ int row(int m) const {
    return (t0 + m) * tile_rows + 32 * (wave_id() / hw) + (opaque_lane() & 31);
  }
  __device__ __forceinline__ int2 range(int r) const {
    return reinterpret_cast<const int2*>(a.ranges)[qb + min(r, nq - 1)];
  }
  __device__ __forceinline__ void fetch(int m) {
    own = range(row(m));
    if (tile_rows > 32) some = range((t0 + m) * tile_rows + opaque_lane());
    if (tile_rows > 64) more = range((t0 + m) * tile_rows + 64 + opaque_lane());
  }
  __device__ __forceinline__ int last_key(int r) const {   // of row r's own range
    return min(nk - nq + min(r, nq - 1), nk - 1);
  }
  __device__ __forceinline__ KeySpans settle(int m) {
    const int r0 = (t0 + m) * tile_rows;
    rows.last = last_key(row(m));
    rows.r = row_range(own, rows.last, nk);
    RowRange lo = rows.r, hi = rows.r;           // the tile's rows
    auto join = [&](int2 r, int i) {
      const RowRange x = row_range(r, last_key(r0 + i), nk);
      lo = {min(lo.shared, x.shared), min(lo.start, x.start)};
      hi = {max(hi.shared, x.shared), max(hi.start, x.start)};
    };
    if (tile_rows > 32) join(some, opaque_lane());
    if (tile_rows > 64) join(more, 64 + opaque_lane());
    int shared_max, start_min;
    wave_bounds(lo.shared, hi.shared, rows.shared_min, shared_max);
    wave_bounds(lo.start, hi.start, start_min, rows.start_max);
    rows.last_min = last_key(r0);
    return key_spans(shared_max, start_min, last_key(r0 + tile_rows - 1) + 1);
  }
  // Element offset of row r of the wave's 32, of item m; its row of the sequence.
  __device__ __forceinline__ int seq_row(int m, int r) const {
    return (t0 + m) * tile_rows + 32 * (wave_id() / hw) + r;
  }
  __device__ __forceinline__ size_t at(int m, int r) const {
    return ((size_t)(qb + min(seq_row(m, r), nq - 1)) * a.hq + h0 + wave_id() % hw) * D;
  }
  __device__ __forceinline__ const bf16_t* q(int m, int r) const {
    return (const bf16_t*)a.q + at(m, r);
  }
  __device__ __forceinline__ void store(int m, const PfState<D>& st, float l, float scale,
                                        bf16_t* io) const {
    mt_store<D>(st, io, [&](int r) {
      return seq_row(m, r) < nq ? (bf16_t*)a.o + at(m, r) : (bf16_t*)nullptr;
    });
    if (a.lse != nullptr) {
      const float lse = mt_lse(st, l, scale);
      const int r = row(m);
      if (opaque_lane() < 32 && r < nq)
        a.lse[(size_t)(h0 + wave_id() % hw) * uniform_load(a.cu_q, a.num_seqs) + qb + r] = lse;
    }
  }
};

}  // namespace

// Workgroups of a (sequence, kv head, head group): min(n_qt, kRgLast) for the last
// tiles, one each, dispatched first for all of them (a prompt's query sees all its
// documents, and nothing else would even out a launch that ends with it); then one
// for every `items` others.
__host__ __device__ constexpr int ranges_groups(int n_qt, int items) {
  return n_qt <= kRgLast ? n_qt : kRgLast + (n_qt - kRgLast + items - 1) / items;
}

// Where the kv heads divide among the XCDs, each has all sequences' tiles of its own
// heads and their K/V in its L2 (16 prompts of 5 to 20 documents, 32 q / 8 kv heads: 878
// us, with tiles round the XCDs one by one 914; 16 / 16 heads 812 and 844).  Elsewhere
// that would give the XCDs other sequences, and other amounts of work, and tiles go round
// them.  4 prompts of 5 to 20 chunks with prefixes, tiles round the XCDs and not: 8 q / 1
// kv heads 704 and 1764 us, 32 / 2 2762 and 3921, 32 / 4 2791 and 3893, 24 / 6 2178 and
// 2587; with windows 87 and 180, 311 and 361, 333 and 360, 259 and 257; with documents 209
// and 213, 264 and 287, 272 and 295, 229 and 224; 16 prompts of documents 261 and 275, 980
// and 956, 998 and 975, 782 and 761.
__host__ __device__ constexpr int ranges_parts(int hkv) { return hkv % kNumXcd == 0 ? kNumXcd : 1; }

template <int D>
__global__ __launch_bounds__(64 * kMtWaves, 2) void ranges_kernel(RangesArgs a, int n_qt, int items) {
  __shared__ __attribute__((aligned(16))) MtLds<D> lds;
  const int group = a.hq / a.hkv, hw = pf_heads_per_wg(group), ng = group / hw;
  const int parts = ranges_parts(a.hkv);
  const int xcd = blockIdx.x % parts;
  int local = blockIdx.x / parts;
  const int streams = (a.num_seqs * a.hkv + parts - 1) / parts;       // per XCD
  const int hg = local % ng;
  local /= ng;
  const int first = min(n_qt, kRgLast) * streams;
  int j, stream, count = 1;
  if (local < first) {
    j = local / streams;
    stream = xcd + parts * (local % streams);
  } else {
    const int per = ranges_groups(n_qt, items) - kRgLast;
    j = kRgLast + (local - first) % per * items;
    count = items;
    stream = xcd + parts * ((local - first) / per);
  }
  if (stream >= a.num_seqs * a.hkv) return;
  const int s = stream / a.hkv, kvh = stream % a.hkv;
  const int qb = uniform_load(a.cu_q, s), kb = uniform_load(a.cu_k, s);
  const int nq = uniform_load(a.cu_q, s + 1) - qb, nk = uniform_load(a.cu_k, s + 1) - kb;
  const int rows = pf_rows_per_tile(group, kMtWaves);
  // tiles j .. j + count - 1 from the sequence's end, in ascending order
  const int last = (nq + rows - 1) / rows - 1 - j;
  if (last < 0) return;
  RangeSrc<D> src{a};
  src.count = min(count, last + 1);
  src.t0 = last + 1 - src.count;
  src.qb = qb;
  src.nq = nq;
  src.nk = nk;
  src.h0 = kvh * group + hg * hw;
  src.hw = hw;
  src.tile_rows = rows;
  if (nk <= 0) {                                 // no key: nothing to copy from
    PfState<D> st;
    pf_reset(st);
    for (int m = 0; m < src.count; ++m) src.store(m, st, 0.f, a.scale, lds.io[wave_id()]);
    return;
  }
  const DenseKV kv{(const bf16_t*)a.k + ((size_t)kb * a.hkv + kvh) * D,
                   (const bf16_t*)a.v + ((size_t)kb * a.hkv + kvh) * D, (size_t)a.hkv * D};
  masked_items<D>(src, kv, nk, a.scale, lds);
}

static int ranges_tiles(const RangesArgs& a) {
  const int rows = pf_rows_per_tile(a.hq / a.hkv, kMtWaves);
  return (int)((a.max_seqlen_q + (int64_t)rows - 1) / rows);
}

static int ranges_items(const RangesArgs& a) {
  if (const int forced = pf_items_override()) return forced;
  const int group = a.hq / a.hkv, ng = group / pf_heads_per_wg(group);
  const int64_t tiles = (int64_t)(ranges_tiles(a) - kRgLast) * a.num_seqs * a.hkv * ng;
  return tiles >= kRgMany ? kRgItems : 1;
}

static int64_t ranges_grid_of(const RangesArgs& a, int items) {
  const int group = a.hq / a.hkv;
  const int64_t streams = (int64_t)a.num_seqs * a.hkv;
  const int parts = ranges_parts(a.hkv);
  return (streams + parts - 1) / parts * parts * ranges_groups(ranges_tiles(a), items) *
         (group / pf_heads_per_wg(group));
}

int64_t ranges_grid(const RangesArgs& a) { return ranges_grid_of(a, 1); }

hipError_t launch_ranges(const RangesArgs& a, hipStream_t stream) {
  const int items = ranges_items(a);
  const int64_t grid = ranges_grid_of(a, items);
  if (grid == 0) return hipSuccess;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a,
                       ranges_tiles(a), items);
  };
  a.d == 64 ? go(ranges_kernel<64>) : go(ranges_kernel<128>);
  return hipGetLastError();
}

}  // namespace rag
