// Keys and values of sequences in a 4-bit paged cache, back as packed bf16 rows
// (gfx950): what a prefill over keys that are in the cache already takes.
//
// HBM-bound, by the rows written.  A wave takes one page of one kv head: a lane has 16
// bytes of K codes (one key, 32 channels) and 16 of V codes (four keys, 8 channels)
// in one load each.
#include "common.h"
#include "kv4.h"
#include "serve.h"

namespace rag {

namespace {

constexpr int kRdWaves = 4;

// s (c - z), two codes of a register, as two bf16.
__device__ __forceinline__ uint32_t kv4_value2(uint32_t w, int p, float s, float zz) {
  const uint32_t x = kv4_pair(w, p);
  const float a = (__uint_as_float(x << 16) - zz) * s;
  const float b = (__uint_as_float(x & 0xffff0000u) - zz) * s;
  const bf16x2 o = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, o);
}

// Sequence s's pages stand at the places (cu[s] / 16) + s on, which leaves room for all of
// them: its rows fall on at most cu[s+1]/16 - cu[s]/16 + 1 pages.
template <int D>
__global__ __launch_bounds__(64 * kRdWaves) void kv4_read_kernel(Kv4ReadArgs a) {
  using P = Kv4Page<D>;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  const int64_t unit = (int64_t)blockIdx.x * kRdWaves + wave_id();
  const int place = (int)(unit / a.hkv), h = (int)(unit % a.hkv);
  if (place >= (a.num_rows >> 4) + a.num_seqs) return;
  int lo = 0, hi = a.num_seqs - 1;                 // the last sequence that starts at or before
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((a.cu_k[mid] >> 4) + mid <= place) lo = mid; else hi = mid - 1;
  }
  const int first = a.cu_k[lo], n = min(a.cu_k[lo + 1], a.num_rows) - first;
  const int page = place - (first >> 4) - lo;
  if (page < 0 || 16 * page >= n || page >= a.max_blocks) return;
  const int left = min(n - 16 * page, 16);
  const int id = a.tables[(size_t)lo * a.max_blocks + page];
  const size_t at = ((size_t)id * a.hkv + h) * P::kBytes;
  const char* kp = (const char*)a.k_cache + at;
  const char* vp = (const char*)a.v_cache + at;
  const size_t row = (size_t)(first + 16 * page), stride = (size_t)a.hkv * D;
  bf16_t* ko = (bf16_t*)a.k + row * stride + (size_t)h * D;
  bf16_t* vo = (bf16_t*)a.v + row * stride + (size_t)h * D;

  if (l16 < left) {                                // K: key l16, channels 16 g4 .. of each group
#pragma unroll
    for (int g = 0; g < P::kGroups; ++g) {
      const uint32_t pr = *(const uint32_t*)(kp + P::param(l16, g));
      const float s = kv4_scale(pr), zz = kv4_zero(pr);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t x = *(const uint32_t*)(kp + P::k_word(l16, 8 * g + 2 * g4 + w));
        u32x4 o;
#pragma unroll
        for (int p = 0; p < 4; ++p) o[p] = kv4_value2(x, p, s, zz);
        *reinterpret_cast<u32x4*>(ko + l16 * stride + 64 * g + 16 * g4 + 8 * w) = o;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {                    // V: keys 4 g4 + t, channels 4 l16 .. of each group
    const int key = 4 * g4 + t;
    if (key >= left) continue;
#pragma unroll
    for (int g = 0; g < P::kGroups; ++g) {
      const uint32_t pr = *(const uint32_t*)(vp + P::param(key, g));
      const float s = kv4_scale(pr), zz = kv4_zero(pr);
      const uint32_t x = *(const uint16_t*)(vp + P::v_unit(key, l16, g));
      // nibbles (0, 1) and (2, 3) in the halves of a word
      u32x2 o;
      o[0] = kv4_value2((x & 0xf) | (x & 0xf0) << 12, 0, s, zz);
      o[1] = kv4_value2((x >> 8 & 0xf) | (x & 0xf000) << 4, 0, s, zz);
      *reinterpret_cast<u32x2*>(vo + key * stride + 64 * g + 4 * l16) = o;
    }
  }
}

}  // namespace

int64_t kv4_read_grid(const Kv4ReadArgs& a) {
  return (((int64_t)(a.num_rows >> 4) + a.num_seqs) * a.hkv + kRdWaves - 1) / kRdWaves;
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)kv4_read_grid(a)), block(64 * kRdWaves);
  if (a.d == 64)
    kv4_read_kernel<64><<<grid, block, 0, stream>>>(a);
  else
    kv4_read_kernel<128><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rag
