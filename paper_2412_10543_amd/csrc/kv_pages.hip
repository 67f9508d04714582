// Pages of a paged KV cache, kept on the GPU (gfx950):
//   pages_kernel  block tables, slot mapping and free stack from the lengths
//                 that the rows hold and are to hold
//   keep_kernel   the K/V rows of accepted drafted tokens moved to the end of
//                 their sequence
// Both move a few bytes per token; a call's time is its launch and its chain of
// dependent reads.
#include "common.h"
#include "draft.h"

namespace rag {

namespace {

constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / kWave;
constexpr int kPgSlots = 4 * kPgThreads;         // slots per workgroup, four a thread
// Sums stop here: any count above what a call can grant is as good as another,
// and two of them still fit 32 bits.
constexpr uint32_t kPgMany = 1u << 30;

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kPgMany); }

__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const uint32_t y = __shfl_up(x, d, kWave);
    if (lane >= d) x = sat_add(x, y);
  }
  return x;
}

// What row r is to gain or give back.
struct RowChange {
  uint32_t grow, give, tokens;  // pages taken, pages given back, tokens added
  int want;                     // pages it is to hold
};

__device__ __forceinline__ RowChange row_change(const PagesArgs& a, int r) {
  const int cap = a.max_blocks * 16;             // (max_blocks is below 2^27)
  const int o = min(max(a.old_lens[r], 0), cap), n = max(a.new_lens[r], 0);
  const int held = (o + 15) >> 4;
  RowChange c;
  c.want = (int)(((uint32_t)n + 15) >> 4);
  c.grow = (uint32_t)max(c.want - held, 0);
  c.give = (uint32_t)max(held - c.want, 0);
  c.tokens = (uint32_t)max(n - o, 0);
  return c;
}

}  // namespace

// Every workgroup forms the same prefix sums over the rows (from the caches;
// a launch that shared them would need a second kernel or a wait) and fills its
// own share of the slots.  A page's table entry is written by the thread that
// has the page's first token; the pages themselves follow from the sums, so no
// workgroup reads what another writes: page number j that is taken is entry
// n + P - 1 - j of the stack with the P given pages behind its n.
__global__ __launch_bounds__(kPgThreads) void pages_kernel(PagesArgs a) {
  extern __shared__ uint32_t sums[];             // tok [S + 1], grow [S + 1], give [S + 1]
  __shared__ uint32_t wave_sum[3][kPgWaves];
  __shared__ int cut;
  const int S = a.num_seqs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t* tok = sums;
  uint32_t* grow = tok + S + 1;
  uint32_t* give = grow + S + 1;
  uint32_t base[3] = {0, 0, 0};
  if (tid == 0) cut = S;
  for (int r0 = 0; r0 < S; r0 += kPgThreads) {
    const int r = r0 + tid;
    RowChange c{0, 0, 0, 0};
    if (r < S) c = row_change(a, r);
    const uint32_t v[3] = {min(c.tokens, kPgMany), c.grow, c.give};
    uint32_t incl[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      incl[i] = wave_scan_sat(v[i]);
      if (lane == 63) wave_sum[i][wave] = incl[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint32_t before = base[i];
#pragma unroll
      for (int w = 0; w < kPgWaves; ++w) {
        if (w == wave && r < S) {
          // (inclusive sums at r + 1: entry r is then the sum of the rows above)
          (i == 0 ? tok : i == 1 ? grow : give)[r + 1] = sat_add(before, incl[i]);
        }
        before = sat_add(before, wave_sum[i][w]);
      }
      base[i] = before;
    }
    __syncthreads();
  }
  if (tid == 0) tok[0] = grow[0] = give[0] = 0;
  __syncthreads();
  // Rows grow up to the first that does not fit.
  const int n_free = min(max(*a.num_free, 0), a.num_blocks);
  const uint32_t given = give[S];
  const uint32_t avail = min((uint32_t)n_free + given, (uint32_t)a.num_blocks);
  for (int r = tid; r < S; r += kPgThreads) {
    if (tok[r + 1] == tok[r] && tok[r] < kPgMany) continue;    // adds nothing
    if (row_change(a, r).tokens == 0) continue;
    const bool fits = grow[r + 1] <= avail && tok[r + 1] <= (uint32_t)a.max_new_tokens &&
                      row_change(a, r).want <= a.max_blocks;
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
    const int want = max(row_change(a, lo).want, 0) + (int)(g - give[lo]);
    return a.tables[(size_t)lo * a.max_blocks + min(want, a.max_blocks - 1)];
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
      int o = min(max(a.old_lens[row], 0), a.max_blocks * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + e;
        if (i >= total) break;
        while ((int)tok[row + 1] <= i) {
          ++row;
          page = -1;
          o = min(max(a.old_lens[row], 0), a.max_blocks * 16);
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

int64_t pages_grid(const PagesArgs& a) {
  return a.max_new_tokens > 0 ? ((int64_t)a.max_new_tokens + kPgSlots - 1) / kPgSlots : 1;
}

hipError_t launch_pages(const PagesArgs& a, hipStream_t stream) {
  const size_t lds = 3 * ((size_t)a.num_seqs + 1) * sizeof(uint32_t);
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
