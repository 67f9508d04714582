// Between the projection of a batch of new tokens and their attention (gfx950):
// the RMS norm of each head of Q and K, the rotation of both by the tokens'
// positions, and the K and V rows' way into the paged cache, in bf16 or in 4 bits,
// in one pass over the projection's output.
//
//   norm      y = x w / sqrt(mean(x^2) + eps), over the D channels of a head
//   rotation  (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of channels
//             (i, i + R/2), or (2 i, 2 i + 1); channels from R on stay
// Both in fp32, rounded once, to bf16; 4-bit codes (kv4.h) are made of the rounded
// values, so that they are those of a bf16 cache.
//
// HBM-bound: 8,200 tokens of 32 q / 8 kv heads of 128 with packed K and V 46 us, 4.6 TB/s; 6,665 into 4
// bits 44, 3.3 TB/s, with the vector units busy for 69% (minima, codes and their places).  64 tokens take
// 4.0 us in bf16 and 4.6 in 4 bits, one launch's latencies.  A wave
// holds 64 / (D/8) head rows at a time, 16 bytes a lane, and walks over the heads of one token with its
// angles in registers, so that neither the rows nor the angles are read twice and a head's sum of
// squares stays in DPP rows of 8 or 16 lanes.
#include "common.h"
#include "kv4.h"
#include "serve.h"

namespace rag {

namespace {

constexpr int kRpWaves = 4;
// Steps whose rows are requested at a time (8,200 tokens, 32 q / 8 kv heads of 128: 47.8 us; with
// one 50.3, two 49.2, four 48.5).
constexpr int kRpAhead = 3;
// Workgroups that a token's rows are spread over waves for (4096: 50.5 us).
constexpr int kRpFill = 1024;

__device__ __forceinline__ void unpack8(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(x[i] << 16);
    f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
}

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), kCtrl, 0xf, 0xf, false));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e;        // lanes of a quad
constexpr int kMirror8 = 0x141, kMirror16 = 0x140, kTurn8 = 0x128;

// Sum over the D/8 lanes of a row.
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<kXor1>(x);
  x += dpp<kXor2>(x);
  x += dpp<kMirror8>(x);
  if constexpr (D == 128) x += dpp<kMirror16>(x);
  return x;
}

// Minimum over the 8 lanes of a group of 64 channels.
__device__ __forceinline__ float group_min(float x) {
  x = fminf(x, dpp<kXor1>(x));
  x = fminf(x, dpp<kXor2>(x));
  return fminf(x, dpp<kMirror8>(x));
}

// The lane's eight channels (chunk j of the row) of a token's K or V row, to its page.
template <int D>
__device__ __forceinline__ void store_kv4(u32x4 x, bool key, char* page, int token, int j) {
  using P = Kv4Page<D>;
  float f[8], c[8];
  unpack8(x, f);
  float lo = 0.f, hi = 0.f;
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, f[i]);
    hi = fminf(hi, -f[i]);
    finite &= fabsf(f[i]) < INFINITY;
  }
  lo = group_min(lo);
  hi = -group_min(hi);
  finite = group_min(finite ? 1.f : 0.f) > 0.f;
  const Kv4Scale sc(lo, hi, finite);
  sc.codes(f, c);
  // (four nibbles are a whole float below 2^16)
  auto nibbles = [](float a, float b, float d, float e) {
    return (uint32_t)fmaf(fmaf(fmaf(e, 16.f, d), 16.f, b), 16.f, a);
  };
  uint32_t word, at;
  if (key) {
    word = nibbles(c[0], c[2], c[4], c[6]) | nibbles(c[1], c[3], c[5], c[7]) << 16;
    at = P::k_word(token, j);
  } else {
    const uint32_t first = nibbles(c[0], c[1], c[2], c[3]), second = nibbles(c[4], c[5], c[6], c[7]);
    word = first | second << 16;
    at = P::v_unit(token, 2 * (j % 8), j / 8);
  }
  if constexpr (D == 128) {                        // both groups' unit i of a token in one word
    const uint32_t give = j < 8 ? word >> 16 : word << 16;
    const uint32_t got = __builtin_amdgcn_update_dpp(0, give, kTurn8, 0xf, 0xf, false);
    if (!key) {
      word = j < 8 ? (word & 0xffff) | got : (word & 0xffff0000u) | got;
      at = P::v_unit(token, 2 * (j % 8) + j / 8, 0);
    }
    *reinterpret_cast<uint32_t*>(page + at) = word;
  } else if (key) {
    *reinterpret_cast<uint32_t*>(page + at) = word;
  } else {
    *reinterpret_cast<uint16_t*>(page + at) = (uint16_t)word;
    *reinterpret_cast<uint16_t*>(page + P::v_unit(token, 2 * j + 1, 0)) = (uint16_t)(word >> 16);
  }
  if (j % 8 == 0) *reinterpret_cast<uint32_t*>(page + P::param(token, j / 8)) = sc.param();
}

// Workgroup: kRpWaves waves, each a token (x) and a share of its head rows (y).  kRpAhead steps' rows
// are requested before the first of them is worked on.
template <int D, bool kKv4>
__global__ __launch_bounds__(64 * kRpWaves) void rope_kernel(RopeArgs a) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;
  const int lane = threadIdx.x & 63, j = lane % kLanes;
  const int64_t t = (int64_t)blockIdx.x * kRpWaves + wave_id();
  if (t >= a.num_tokens) return;
  const int q_rows = a.q != nullptr ? a.hq : 0, rows = q_rows + 2 * a.hkv;
  const int steps = (rows + kRows - 1) / kRows;
  auto row_at = [&](int it) {
    const int r = min(it * kRows + lane / kLanes, rows - 1);
    const bf16_t* src = r < q_rows           ? (const bf16_t*)a.q + t * a.q_stride + (size_t)r * D
                        : r < q_rows + a.hkv ? (const bf16_t*)a.k + t * a.k_stride + (size_t)(r - q_rows) * D
                                             : (const bf16_t*)a.v + t * a.v_stride +
                                                   (size_t)(r - q_rows - a.hkv) * D;
    return src + j * 8;
  };
  u32x4 next[kRpAhead];
#pragma unroll
  for (int i = 0; i < kRpAhead; ++i)
    next[i] = load16(row_at(min((int)(blockIdx.y + i * gridDim.y), steps - 1)));

  const int slot = a.slots != nullptr ? a.slots[t] : 0;
  if (slot < 0) return;                              // padding token
  // the pair's other channel is in chunk `other`; angles of the lane's eight channels
  const int half = a.rot / 16;                       // chunks of R/2 channels
  const bool turned = a.positions != nullptr && j < a.rot / 8;
  int other = j;
  float c[8], s[8];
  if (turned) {
    // (a position outside the table is a broken precondition; it reads the last row)
    const int pos = (int)min((uint32_t)a.positions[t], (uint32_t)(a.max_position - 1));
    const float* row = a.cos_sin + (size_t)pos * a.rot;
    if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = row[4 * j + i / 2];
        s[i] = row[a.rot / 2 + 4 * j + i / 2] * (i % 2 ? 1.f : -1.f);
      }
    } else {
      other = j < half ? j + half : j - half;
      const float* p = row + 8 * (j < half ? j : other);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = p[i];
        s[i] = p[a.rot / 2 + i] * (j < half ? -1.f : 1.f);
      }
    }
  }
  u32x4 wq[2], wk[2];                                // weights of the lane's chunk and of the other
  if (a.q_weight != nullptr) {
    wq[0] = load16((const bf16_t*)a.q_weight + j * 8);
    wq[1] = load16((const bf16_t*)a.q_weight + other * 8);
  }
  if (a.k_weight != nullptr) {
    wk[0] = load16((const bf16_t*)a.k_weight + j * 8);
    wk[1] = load16((const bf16_t*)a.k_weight + other * 8);
  }

  auto step = [&](int it, u32x4 x) {
    const int r = it * kRows + lane / kLanes;
    const bool is_q = r < q_rows, is_k = !is_q && r < q_rows + a.hkv, has = r < rows;
    const int h = is_q ? r : is_k ? r - q_rows : r - q_rows - a.hkv;
    const bool normed = is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr;
    float f[8], g[8];
    unpack8(x, f);
    // the other channels, by the wave's quickest way
    u32x4 y = x;
    if (a.positions != nullptr && !a.interleaved) {
      if (D == 128 && half == kLanes / 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_update_dpp(0, x[i], kTurn8, 0xf, 0xf, false);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __shfl(x[i], lane - j + other, kWave);
      }
    }
    unpack8(y, g);
    if (a.q_weight != nullptr || a.k_weight != nullptr) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
      const float n = 1.f / sqrtf(row_sum<D>(sum) * (1.f / D) + a.eps);
      if (normed) {
        float wf[8], wg[8];
        unpack8(is_q ? wq[0] : wk[0], wf);
        unpack8(is_q ? wq[1] : wk[1], wg);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = f[i] * n * wf[i];
          g[i] = g[i] * n * wg[i];
        }
      }
    }
    if (turned && (is_q || is_k)) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = fmaf(f[i], c[i], (a.interleaved ? f[i ^ 1] : g[i]) * s[i]);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = o[i];
    }
    if (normed || (turned && (is_q || is_k)))        // (others are copied bit by bit)
      x = as_u32x4(to_bf16x8(f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]));
    if (is_q) {
      *reinterpret_cast<u32x4*>((bf16_t*)a.q_out + ((size_t)t * a.hq + h) * D + j * 8) = x;
    } else if (has) {
      bf16_t* out = (bf16_t*)(is_k ? a.k_out : a.v_out);
      if (out != nullptr)
        *reinterpret_cast<u32x4*>(out + ((size_t)t * a.hkv + h) * D + j * 8) = x;
      if (a.slots != nullptr) {
        char* cache = (char*)(is_k ? a.k_cache : a.v_cache);
        const size_t page = (size_t)(slot >> 4) * a.hkv + h;
        if constexpr (kKv4)                          // (the lanes of a row take this together)
          store_kv4<D>(x, is_k, cache + page * Kv4Page<D>::kBytes, slot & 15, j);
        else
          *reinterpret_cast<u32x4*>((bf16_t*)cache + (page * 16 + (slot & 15)) * D + j * 8) = x;
      }
    }
  };
  for (int it = blockIdx.y; it < steps; it += kRpAhead * gridDim.y) {
    u32x4 x[kRpAhead];
#pragma unroll
    for (int i = 0; i < kRpAhead; ++i) x[i] = next[i];
    if (it + (int)(kRpAhead * gridDim.y) < steps) {
#pragma unroll
      for (int i = 0; i < kRpAhead; ++i)
        next[i] = load16(row_at(min(it + (int)((kRpAhead + i) * gridDim.y), steps - 1)));
    }
#pragma unroll
    for (int i = 0; i < kRpAhead; ++i)
      if (it + i * (int)gridDim.y < steps) step(it + i * (int)gridDim.y, x[i]);
  }
}

int rope_steps(const RopeArgs& a) {
  const int rows = (a.q != nullptr ? a.hq : 0) + 2 * a.hkv, per = kWave / (a.d / 8);
  return (rows + per - 1) / per;
}

dim3 rope_dim(const RopeArgs& a) {
  const unsigned x = (unsigned)((a.num_tokens + (int64_t)kRpWaves - 1) / kRpWaves);
  const int steps = rope_steps(a);
  int y = 1;
  while (y < steps && (int64_t)x * y < kRpFill) ++y;
  return dim3(x, (unsigned)std::min(y, 65535));
}

}  // namespace

int64_t rope_grid(const RopeArgs& a) {
  const dim3 g = rope_dim(a);
  return (int64_t)g.x * g.y;
}

hipError_t launch_rope(const RopeArgs& a, bool kv4, hipStream_t stream) {
  const dim3 grid = rope_dim(a), block(64 * kRpWaves);
  if (grid.x == 0) return hipSuccess;
  if (a.d == 64)
    kv4 ? rope_kernel<64, true><<<grid, block, 0, stream>>>(a)
        : rope_kernel<64, false><<<grid, block, 0, stream>>>(a);
  else
    kv4 ? rope_kernel<128, true><<<grid, block, 0, stream>>>(a)
        : rope_kernel<128, false><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rag
