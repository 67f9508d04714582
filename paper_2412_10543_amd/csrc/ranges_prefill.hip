// Packed variable-length attention with a key range per query row (gfx950): the
// row at position p of its sequence sees the keys j < shared and the keys
// start <= j <= p.  Documents that do not see one another, prefixes seen by
// every row, windows with a few first keys.
//
// A workgroup is one tile of query rows of up to four heads of a GQA group, as
// in the causal prefill; it visits the key tiles of two spans only: up to its
// rows' largest `shared`, and from their smallest `start` to their last
// position.
#include <climits>

#include "common.h"
#include "draft.h"
#include "masked_tile.h"

namespace rag {

namespace {

constexpr int kRgLast = 4;       // tiles of every sequence that are dispatched first

// The lane's row, and for the wave what makes a block full.
struct RangeRows {
  int shared, start, last;      // keys below shared, and start..last
  int shared_min, start_max, last_min;           // of the wave's rows
  __device__ __forceinline__ FullBlocks full_blocks(const KeySpans& sp) const {
    const int lo = (start_max + kMtKeys - 1) / kMtKeys, hi = (last_min + 1) / kMtKeys;
    return {min(shared_min / kMtKeys, sp.na), sp.nb > 0 ? lo + sp.na - sp.b0 / kMtKeys : lo,
            (uint32_t)max(hi - lo, 0)};
  }
  __device__ __forceinline__ uint32_t seen(int k0) const {
    return low_bits(shared - k0) | (low_bits(last + 1 - k0) & ~low_bits(start - k0));
  }
};

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
__device__ __forceinline__ int wave_min(int x) { return INT_MAX - wave_max(INT_MAX - x); }

}  // namespace

template <int D>
__global__ __launch_bounds__(64 * kMtWaves, 2) void ranges_kernel(RangesArgs a, int n_qt) {
  __shared__ __attribute__((aligned(16))) bf16_t kring[kMtRing * BlockLayout<D>::kElems];
  __shared__ __attribute__((aligned(16))) bf16_t vring[kMtRing * BlockLayout<D>::kElems];
  __shared__ int span[3][kMtWaves];
  const int group = a.hq / a.hkv, hw = pf_heads_per_wg(group), ng = group / hw;
  // The last kRgLast tiles of every sequence first: a prompt's query sees all its
  // documents, and nothing else would even out a launch that ends with it.
  int xcd, local;
  xcd_slot(blockIdx.x, xcd, local);
  const int streams = (a.num_seqs * a.hkv + kNumXcd - 1) / kNumXcd;   // per XCD
  const int hg = local % ng;
  local /= ng;
  const int head_n = min(n_qt, kRgLast) * streams;
  int j, stream;
  if (local < head_n) {
    j = local / streams;
    stream = xcd + kNumXcd * (local % streams);
  } else {
    j = kRgLast + (local - head_n) % (n_qt - kRgLast);
    stream = xcd + kNumXcd * ((local - head_n) / (n_qt - kRgLast));
  }
  if (stream >= a.num_seqs * a.hkv) return;
  const int s = stream / a.hkv, kvh = stream % a.hkv, h0 = kvh * group + hg * hw;
  const int qb = uniform_load(a.cu_q, s), kb = uniform_load(a.cu_k, s);
  const int nq = uniform_load(a.cu_q, s + 1) - qb, nk = uniform_load(a.cu_k, s + 1) - kb;
  const int rows = pf_rows_per_tile(group, kMtWaves);
  const int q0 = ((nq + rows - 1) / rows - 1 - j) * rows;
  if (q0 < 0) return;
  const int wave = wave_id(), lane = threadIdx.x & 63, half = lane >> 5;
  const int r = q0 + 32 * (wave / hw) + (lane & 31);
  const int rc = min(r, nq - 1), head = h0 + wave % hw;
  const int2 rg = reinterpret_cast<const int2*>(a.ranges)[qb + rc];
  PfState<D> st;
  mt_load_q<D>(st, (const bf16_t*)a.q + ((size_t)(qb + rc) * a.hq + head) * D);
  RangeRows rr;
  rr.last = min(nk - nq + rc, nk - 1);
  rr.shared = min(max(rg.x, 0), nk);
  rr.start = max(rg.y, 0);
  if (rr.start > rr.last) {                      // nothing of its own
    rr.start = nk;
    rr.last = -1;
  }
  rr.shared_min = wave_min(rr.shared);
  rr.start_max = wave_max(rr.start);
  rr.last_min = wave_min(rr.last + 1) - 1;
  const int shared_max = wave_max(rr.shared), start_min = wave_min(rr.start);
  const int last_max = wave_max(rr.last + 1) - 1;
  if (lane == 0) {
    span[0][wave] = shared_max;
    span[1][wave] = start_min;
    span[2][wave] = last_max;
  }
  __syncthreads();
  int a1 = 0, b0 = nk, b1 = 0;
#pragma unroll
  for (int w = 0; w < kMtWaves; ++w) {
    a1 = max(a1, span[0][w]);
    b0 = min(b0, span[1][w]);
    b1 = max(b1, span[2][w] + 1);
  }
  const DenseKV kv{(const bf16_t*)a.k + ((size_t)kb * a.hkv + kvh) * D,
                   (const bf16_t*)a.v + ((size_t)kb * a.hkv + kvh) * D, (size_t)a.hkv * D};
  const KeySpans sp = key_spans(__builtin_amdgcn_readfirstlane(a1),
                                __builtin_amdgcn_readfirstlane(b0),
                                __builtin_amdgcn_readfirstlane(b1));
  masked_tile<D>(rr, kv, sp, 0, sp.blocks(), nk, a.scale, kring, vring, st);
  const float lse = mt_finish<D>(st, a.scale);
  mt_store<D>(st, (bf16_t*)a.o + ((size_t)(qb + r) * a.hq + head) * D, r < nq);
  if (a.lse != nullptr && half == 0 && r < nq)
    a.lse[(size_t)head * uniform_load(a.cu_q, a.num_seqs) + qb + r] = lse;
}

int64_t ranges_grid(const RangesArgs& a) {
  const int group = a.hq / a.hkv, rows = pf_rows_per_tile(group, kMtWaves);
  const int64_t n_qt = (a.max_seqlen_q + (int64_t)rows - 1) / rows;
  const int64_t streams = (int64_t)a.num_seqs * a.hkv;
  return (streams + kNumXcd - 1) / kNumXcd * kNumXcd * n_qt * (group / pf_heads_per_wg(group));
}

hipError_t launch_ranges(const RangesArgs& a, hipStream_t stream) {
  const int group = a.hq / a.hkv, rows = pf_rows_per_tile(group, kMtWaves);
  const int n_qt = (a.max_seqlen_q + rows - 1) / rows;
  const int64_t grid = ranges_grid(a);
  if (grid == 0) return hipSuccess;
  if (a.d == 64)
    hipLaunchKernelGGL(ranges_kernel<64>, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a, n_qt);
  else
    hipLaunchKernelGGL(ranges_kernel<128>, dim3((unsigned)grid), dim3(64 * kMtWaves), 0, stream, a, n_qt);
  return hipGetLastError();
}

}  // namespace rag
