// Pages of a paged KV cache, kept on the GPU (gfx950):
//   pages_kernel  block tables, slot mapping and free stack from the lengths
//                 that the rows hold and are to hold
//   keep_kernel   the K/V rows of accepted drafted tokens moved to the end of
//                 their sequence
// Both move a few bytes per token; a call's time is its launch and its chain of
// dependent reads (64 rows that grow by 1 to 64 tokens 6.3 us a call, 640 that get 576
// each 6.7; 1 and 256 accepted paths 5.2, of which the kernel 2.6 and 3.7; an empty
// launch takes 3.6).
#include <algorithm>

#include "common.h"
#include "draft.h"

namespace rag {

namespace {

constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / kWave;
constexpr int kPgRows = 4;                       // consecutive rows of a thread, at a time
constexpr int kPgSlots = 4 * kPgThreads;         // slots per workgroup, four a thread
// Sums stop here: any count above what a call can grant is as good as another,
// and two of them still fit 32 bits.
constexpr uint32_t kPgMany = 1u << 30;

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kPgMany); }

__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t x) {
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));  // row_shr:1
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));  // row_shr:2
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));  // row_shr:4
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));  // row_shr:8
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));  // row_bcast:15
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));  // row_bcast:31
  return x;
}

}  // namespace

// Every workgroup forms the same prefix sums over the rows (from the caches;
// a launch that shared them would need a second kernel or a wait) and fills its
// own share of the slots.  A page's table entry is written by the thread that
// has the page's first token; the pages themselves follow from the sums, so no
// workgroup reads what another writes: page number j that is taken is entry
// n + P - 1 - j of the stack with the P given pages behind its n.
// A chain of latencies: the lengths, the sums, a row's search, its page's id.
__global__ __launch_bounds__(kPgThreads) void pages_kernel(PagesArgs a) {
  // sums of the rows above: tokens added, pages taken, pages given back [S + 1];
  // tokens held [S]
  extern __shared__ uint32_t sums[];
  __shared__ uint32_t wave_sum[2][3][kPgWaves];
  __shared__ int cut;
  const int S = a.num_seqs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t* tok = sums;
  uint32_t* grow = tok + S + 1;
  uint32_t* give = grow + S + 1;
  int* old = reinterpret_cast<int*>(give + S + 1);
  const int cap = a.max_blocks * 16;             // (max_blocks is below 2^27)
  const int n_free = min(max(*a.num_free, 0), a.num_blocks);
  uint32_t base[3] = {0, 0, 0};
  if (tid == 0) {
    cut = S;
    tok[0] = grow[0] = give[0] = 0;
  }
  for (int r0 = 0, turn = 0; r0 < S; r0 += kPgRows * kPgThreads, turn ^= 1) {
    const int r = r0 + kPgRows * tid;
    int o[kPgRows], n[kPgRows];
#pragma unroll
    for (int k = 0; k < kPgRows; ++k) {
      const int x = min(r + k, S - 1);
      o[k] = a.old_lens[x];
      n[k] = a.new_lens[x];
    }
    uint32_t s[3][kPgRows];                      // inclusive
    uint32_t run[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < kPgRows; ++k) {
      o[k] = min(max(o[k], 0), cap);
      n[k] = max(n[k], 0);
      const bool real = r + k < S;
      const int held = (o[k] + 15) >> 4, want = (int)(((uint32_t)n[k] + 15) >> 4);
      const uint32_t v[3] = {real ? min((uint32_t)max(n[k] - o[k], 0), kPgMany) : 0u,
                             real ? (uint32_t)max(want - held, 0) : 0u,
                             real ? (uint32_t)max(held - want, 0) : 0u};
#pragma unroll
      for (int i = 0; i < 3; ++i) s[i][k] = run[i] = sat_add(run[i], v[i]);
    }
    uint32_t upto[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      upto[i] = wave_scan_sat(run[i]);
      if (lane == 63) wave_sum[turn][i][wave] = upto[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint32_t before = base[i], all = base[i];
#pragma unroll
      for (int w = 0; w < kPgWaves; ++w) {
        if (w < wave) before = sat_add(before, wave_sum[turn][i][w]);
        all = sat_add(all, wave_sum[turn][i][w]);
      }
      base[i] = all;
      // (the lane's own rows leave the wave's sum up to it: below the limit sums are
      // exact, and at it the difference does not matter: rows there do not fit)
      const uint32_t up = __shfl_up(upto[i], 1, kWave);
      if (lane > 0) before = sat_add(before, up);
      uint32_t* to = i == 0 ? tok : i == 1 ? grow : give;
#pragma unroll
      for (int k = 0; k < kPgRows; ++k)
        if (r + k < S) to[r + k + 1] = sat_add(before, s[i][k]);
    }
#pragma unroll
    for (int k = 0; k < kPgRows; ++k)
      if (r + k < S) old[r + k] = o[k];
  }
  __syncthreads();
  // Rows grow up to the first that does not fit.
  const uint32_t avail = min((uint32_t)n_free + give[S], (uint32_t)a.num_blocks);
  for (int r = tid; r < S; r += kPgThreads) {
    const uint32_t t0 = tok[r], t1 = tok[r + 1], g0 = grow[r], g1 = grow[r + 1];
    if (t1 == t0 && t0 < kPgMany) continue;      // adds nothing
    // (sums at the limit fit neither; below it a row's pages are g1 - g0 more)
    const bool fits = g1 <= avail && t1 <= (uint32_t)a.max_new_tokens &&
                      (uint32_t)((old[r] + 15) >> 4) + (g1 - g0) <= (uint32_t)a.max_blocks;
    if (!fits) atomicMin(&cut, r);
  }
  __syncthreads();
  const int F = cut;
  const int total = (int)tok[F];                 // (all of it granted: at most max_new_tokens)
  const uint32_t taken = grow[F];
  const int left = (int)(avail - min(taken, avail));

  // page x of the stack with the given pages behind it
  auto pile = [&](int x) -> int {
    if (x < n_free) return a.stack[x];
    const uint32_t g = (uint32_t)(x - n_free);
    int lo = 0, hi = S - 1;                      // the row that gave it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (give[mid] <= g) lo = mid; else hi = mid - 1;
    }
    const int at = ((old[lo] + 15) >> 4) - (int)(give[lo + 1] - g);   // behind what it keeps
    return a.tables[(size_t)lo * a.max_blocks + min(max(at, 0), a.max_blocks - 1)];
  };

  // ---- slots ----------------------------------------------------------------
  const int i0 = blockIdx.x * kPgSlots + 4 * tid;
  if (i0 < a.max_new_tokens) {
    int out[4] = {-1, -1, -1, -1};
    if (i0 < total) {
      int lo = 0, hi = F - 1;                    // the row of slot i0
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int)tok[mid] <= i0) lo = mid; else hi = mid - 1;
      }
      int row = lo, page = -1, id = 0;
      int o = old[row];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + e;
        if (i >= total) break;
        while ((int)tok[row + 1] <= i) {
          ++row;
          page = -1;
          o = old[row];
        }
        const int t = o + (i - (int)tok[row]), p = t >> 4, held = (o + 15) >> 4;
        if (p != page) {
          page = p;
          if (p < held) {
            id = a.tables[(size_t)row * a.max_blocks + p];
          } else {
            id = pile((int)avail - 1 - ((int)grow[row] + p - held));
            if ((t & 15) == 0) a.tables[(size_t)row * a.max_blocks + p] = id;
          }
        }
        out[e] = id * 16 + (t & 15);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i0 + e < a.max_new_tokens) a.slots[i0 + e] = out[e];
  }
  // ---- given pages that stay on the stack ------------------------------------
  for (int x = n_free + blockIdx.x * kPgThreads + tid; x < left; x += gridDim.x * kPgThreads)
    a.stack[x] = pile(x);
  // ---- lengths, offsets, counts ------------------------------------------------
  for (int r = blockIdx.x * kPgThreads + tid; r <= S; r += gridDim.x * kPgThreads) {
    a.cu_new[r] = (int)tok[min(r, F)];
    if (r < S) {
      const int o = a.old_lens[r], n = a.new_lens[r];
      a.lens_out[r] = r < F || n < o ? max(n, 0) : o;
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    *a.num_free_out = left;
    *a.num_granted = F;
  }
}

// Workgroups for the slots, and for the pages given back (of which the host knows
// only that the pool has no more), at most one a CU: a row of 36000 tokens that ends
// leaves 2250 (16 rows of 20,000 to 36,000 tokens that end beside 48 that get up to 8
// more: 8.4 us, with workgroups for the slots alone 76).
int64_t pages_grid(const PagesArgs& a) {
  const int64_t slots = ((int64_t)a.max_new_tokens + kPgSlots - 1) / kPgSlots;
  const int64_t pages = ((int64_t)a.num_blocks + kPgSlots - 1) / kPgSlots;
  return std::max<int64_t>({1, slots, std::min<int64_t>(pages, 256)});
}

hipError_t launch_pages(const PagesArgs& a, hipStream_t stream) {
  const size_t lds = (4 * (size_t)a.num_seqs + 3) * sizeof(uint32_t);
  hipLaunchKernelGGL(pages_kernel, dim3((unsigned)pages_grid(a)), dim3(kPgThreads), lds, stream, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// One workgroup per (row, kv head): 256 / (2 D/8) accepted nodes at a time, the
// K half and the V half of the threads, each 16 bytes of one row.  All of a
// pass's reads are done before its writes (a node's place may be another's
// source); later passes read behind everything written before, as kept is
// strictly increasing: kept[j] >= j.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a) {
  constexpr int kCh = D / 8, kNodes = 256 / (2 * kCh);
  const int s = blockIdx.x / a.hkv, h = blockIdx.x % a.hkv;
  const int n = min(a.num_kept[s], a.max_kept), base = a.base_lens[s];
  const int32_t* table = a.tables + (size_t)s * a.max_blocks;
  const int c = threadIdx.x % kCh, side = (threadIdx.x / kCh) & 1, node = threadIdx.x / (2 * kCh);
  bf16_t* cache = (bf16_t*)(side ? a.v_cache : a.k_cache);
  const int64_t cap = (int64_t)a.max_blocks * 16;
  auto at = [&](int key) {
    return cache + (((size_t)table[key >> 4] * a.hkv + h) * 16 + (key & 15)) * D + c * 8;
  };
  for (int i0 = 0; i0 < n; i0 += kNodes) {
    const int i = i0 + node;
    const int from = i < n ? a.kept[(size_t)s * a.max_kept + i] : -1;
    const int64_t src = (int64_t)base + from, dst = (int64_t)base + i;
    const bool move = from >= 0 && from != i && base >= 0 && src < cap && dst < cap;
    u32x4 x = {0, 0, 0, 0};
    if (move) x = load16(at((int)src));
    wait_all_memory();
    __syncthreads();
    if (move) *reinterpret_cast<u32x4*>(at((int)dst)) = x;
    __syncthreads();
  }
}

int64_t keep_grid(const KeepArgs& a) { return (int64_t)a.num_seqs * a.hkv; }

hipError_t launch_keep(const KeepArgs& a, hipStream_t stream) {
  const int64_t grid = keep_grid(a);
  if (grid == 0 || a.max_kept == 0) return hipSuccess;
  if (a.d == 64)
    hipLaunchKernelGGL(keep_kernel<64>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(keep_kernel<128>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace rag
