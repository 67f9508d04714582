// Keys and values of sequences in a 4-bit paged cache, back as packed bf16 rows
// (gfx950): what a prefill over keys that are in the cache already takes.
//
// HBM-bound, by the rows written (24,600 keys of 8 heads of 128: 29 us, 4.5 TB/s of codes and
// rows; 131,072 keys 142, 4.8 TB/s).  A wave takes one page of one kv head: a lane has 16 bytes of K
// codes (one key, 16 channels of each group) and 16 of V codes (four keys, four channels of each
// group), each load in the page's order, and one or two parameters, which reach the lanes that
// need them by shuffles.  (Two, four or eight heads a wave, one after another with the next one's page
// on its way, are slower from 24,600 keys on: 66,000 keys 66 us, with them 74, 77, 85; 524,288 keys
// 560, with them 584 to 591.)
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
  constexpr int kG = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kRdWaves + wave_id();
  const int place = (int)(unit / a.hkv), h = (int)(unit % a.hkv);
  if (place >= (a.num_rows >> 4) + a.num_seqs) return;
  // the last sequence that starts at or before the place (one at least does)
  int s = -1;
  for (int s0 = 0; s0 < a.num_seqs; s0 += kWave) {
    const int x = min(s0 + lane, a.num_seqs - 1);
    s += __popcll(__builtin_amdgcn_ballot_w64(s0 + lane < a.num_seqs && (a.cu_k[x] >> 4) + x <= place));
  }
  if (s < 0) return;
  const int first = a.cu_k[s], n = min(a.cu_k[s + 1], a.num_rows) - first;
  const int page = place - (first >> 4) - s;
  if (page < 0 || 16 * page >= n || page >= a.max_blocks) return;
  const int left = min(n - 16 * page, 16);
  const size_t id = (size_t)a.tables[(size_t)s * a.max_blocks + page] * a.hkv + h;
  const size_t row = (size_t)(first + 16 * page), stride = (size_t)a.hkv * D;
  // K: the lane's key and 16-channel chunk; V: its unit and four keys
  const int l4 = lane >> 2, t4 = lane & 3;

  const char* kp = (const char*)a.k_cache + id * P::kBytes;
  const char* vp = (const char*)a.v_cache + id * P::kBytes;
  uint32_t k[2 * kG], v[2 * kG];
  if constexpr (kG == 2) {
    const u32x4 x = load16_stream(kp + 16 * lane), y = load16_stream(vp + 16 * lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[i] = x[i];
      v[i] = y[i];
    }
  } else {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(kp + 8 * lane));
    const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(vp + 8 * lane));
    k[0] = x[0];
    k[1] = x[1];
    v[0] = y[0];
    v[1] = y[1];
  }
  // K's parameters in the first 16 kG lanes, V's in the next
  const int at = P::kParams + 4 * (lane & (16 * kG - 1));
  const uint32_t params = *reinterpret_cast<const uint32_t*>((lane & (16 * kG) ? vp : kp) + at);
  // (all requested before the first is used: the compiler would move K's codes under the branch of their
  // stores, behind the parameters, 2 to 10% longer)
#pragma unroll
  for (int i = 0; i < 2 * kG; ++i) asm volatile("" : "+v"(k[i]), "+v"(v[i]));

  bf16_t* ko = (bf16_t*)a.k + row * stride + (size_t)h * D;
  bf16_t* vo = (bf16_t*)a.v + row * stride + (size_t)h * D;
#pragma unroll
  for (int g = 0; g < kG; ++g) {                   // K: channels 64 g + 16 t4 ..
    const uint32_t pr = __shfl(params, 16 * g + l4, kWave);
    const float sc = kv4_scale(pr), zz = kv4_zero(pr);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      u32x4 o;
#pragma unroll
      for (int p = 0; p < 4; ++p) o[p] = kv4_value2(k[2 * g + w], p, sc, zz);
      if (l4 < left) *reinterpret_cast<u32x4*>(ko + l4 * stride + 64 * g + 16 * t4 + 8 * w) = o;
    }
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)                      // V: keys 4 t4 + t, channels 64 g + 4 l4 ..
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      const uint32_t pr = __shfl(params, 16 * (kG + g) + 4 * t4 + t, kWave);
      const float sc = kv4_scale(pr), zz = kv4_zero(pr);
      // the unit's four nibbles, two in the halves of a word each
      const uint32_t word = v[kG == 2 ? t : t / 2], x = (kG == 2 ? g : t % 2) ? word >> 16 : word & 0xffff;
      u32x2 o;
      o[0] = kv4_value2((x & 0xf) | (x & 0xf0) << 12, 0, sc, zz);
      o[1] = kv4_value2((x >> 8 & 0xf) | (x & 0xf000) << 4, 0, sc, zz);
      if (4 * t4 + t < left)
        *reinterpret_cast<u32x2*>(vo + (4 * t4 + t) * stride + 64 * g + 4 * l4) = o;
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
