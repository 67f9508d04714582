// Keys and values of sequences in a 4-bit paged cache, back as packed bf16 rows
// (gfx950): what a prefill over keys that are in the cache already takes.
//
// HBM-bound, by the rows written (24,600 keys of 8 heads of 128: 30 us, 4.3 TB/s of codes and
// rows).  A wave takes one page of a few kv heads, one after another: a lane has 16 bytes of K
// codes (one key, 16 channels of each group) and 16 of V codes (four keys, four channels of each
// group), each load in the page's order, and one or two parameters, which reach the lanes that
// need them by shuffles.
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
__global__ __launch_bounds__(64 * kRdWaves) void kv4_read_kernel(Kv4ReadArgs a, int heads) {
  using P = Kv4Page<D>;
  constexpr int kG = D / 64;
  const int lane = threadIdx.x & 63;
  const int parts = (a.hkv + heads - 1) / heads;   // of a page
  const int64_t unit = (int64_t)blockIdx.x * kRdWaves + wave_id();
  const int place = (int)(unit / parts), h0 = (int)(unit % parts) * heads;
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
  const size_t id = (size_t)a.tables[(size_t)s * a.max_blocks + page] * a.hkv;
  const size_t row = (size_t)(first + 16 * page), stride = (size_t)a.hkv * D;
  // K: the lane's key and 16-channel chunk; V: its unit and four keys
  const int l4 = lane >> 2, t4 = lane & 3;

  struct Page {
    uint32_t k[2 * kG], v[2 * kG], p;
  };
  auto load = [&](Page& r, int h) {
    const char* kp = (const char*)a.k_cache + (id + h) * P::kBytes;
    const char* vp = (const char*)a.v_cache + (id + h) * P::kBytes;
    if constexpr (kG == 2) {
      const u32x4 x = load16_stream(kp + 16 * lane), y = load16_stream(vp + 16 * lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r.k[i] = x[i];
        r.v[i] = y[i];
      }
    } else {
      const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(kp + 8 * lane));
      const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(vp + 8 * lane));
      r.k[0] = x[0];
      r.k[1] = x[1];
      r.v[0] = y[0];
      r.v[1] = y[1];
    }
    // K's parameters in the first 16 kG lanes, V's in the next
    const int w = lane & (16 * kG - 1);
    r.p = *reinterpret_cast<const uint32_t*>((lane & (16 * kG) ? vp : kp) + P::kParams + 4 * w);
  };
  auto store = [&](const Page& r, int h) {
    bf16_t* ko = (bf16_t*)a.k + row * stride + (size_t)h * D;
    bf16_t* vo = (bf16_t*)a.v + row * stride + (size_t)h * D;
#pragma unroll
    for (int g = 0; g < kG; ++g) {                 // K: channels 64 g + 16 t4 ..
      const uint32_t pr = __shfl(r.p, 16 * g + l4, kWave);
      const float sc = kv4_scale(pr), zz = kv4_zero(pr);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        u32x4 o;
#pragma unroll
        for (int p = 0; p < 4; ++p) o[p] = kv4_value2(r.k[2 * g + w], p, sc, zz);
        if (l4 < left)
          *reinterpret_cast<u32x4*>(ko + l4 * stride + 64 * g + 16 * t4 + 8 * w) = o;
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)                    // V: keys 4 t4 + t, channels 64 g + 4 l4 ..
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const uint32_t pr = __shfl(r.p, 16 * (kG + g) + 4 * t4 + t, kWave);
        const float sc = kv4_scale(pr), zz = kv4_zero(pr);
        // the unit's four nibbles, two in the halves of a word each
        const uint32_t word = r.v[kG == 2 ? t : t / 2], x = (kG == 2 ? g : t % 2) ? word >> 16 : word & 0xffff;
        u32x2 o;
        o[0] = kv4_value2((x & 0xf) | (x & 0xf0) << 12, 0, sc, zz);
        o[1] = kv4_value2((x >> 8 & 0xf) | (x & 0xf000) << 4, 0, sc, zz);
        if (4 * t4 + t < left)
          *reinterpret_cast<u32x2*>(vo + (4 * t4 + t) * stride + 64 * g + 4 * l4) = o;
      }
  };
  const int end = min(h0 + heads, a.hkv);
  Page next;
  load(next, h0);
  for (int h = h0; h < end; ++h) {
    const Page r = next;
    if (h + 1 < end) load(next, h + 1);
    store(r, h);
  }
}

// kv heads of a wave: as many as leave the GPU kRdFill waves (24,600 keys of 8 heads of 128: 30.6 us;
// with 4096 34.2, 1024 37.4).
constexpr int64_t kRdFill = 8192;

int read_heads(const Kv4ReadArgs& a) {
  const int64_t places = (int64_t)(a.num_rows >> 4) + a.num_seqs;
  int heads = std::min(a.hkv, 8);
  while (heads > 1 && places * ((a.hkv + heads - 1) / heads) < kRdFill) heads /= 2;
  return heads;
}

}  // namespace

int64_t kv4_read_grid(const Kv4ReadArgs& a) {
  const int heads = read_heads(a), parts = (a.hkv + heads - 1) / heads;
  return (((int64_t)(a.num_rows >> 4) + a.num_seqs) * parts + kRdWaves - 1) / kRdWaves;
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)kv4_read_grid(a)), block(64 * kRdWaves);
  const int heads = read_heads(a);
  if (a.d == 64)
    kv4_read_kernel<64><<<grid, block, 0, stream>>>(a, heads);
  else
    kv4_read_kernel<128><<<grid, block, 0, stream>>>(a, heads);
  return hipGetLastError();
}

}  // namespace rag
