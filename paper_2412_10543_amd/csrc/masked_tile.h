// Attention of one tile of query rows to a list of key spans, with a mask per
// row, for gfx950: kWaves waves of 32 rows each over shared 64-key tiles.
//
// Method: exact tiled attention with an online softmax, on the pieces of
// prefill_tile.h (S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16,
// one query row per lane).  What differs from the causal prefill:
//   * the key tiles are those of two spans (KeySpans), so that keys between
//     them cost nothing;
//   * a 32-key block is full (no mask), partial (a 32-bit word per lane says
//     which of its keys the lane's row sees) or, for a wave, empty (skipped);
//   * a row may see no key at all: output 0, log-sum-exp -inf;
//   * values of keys that a row does not see never reach it, whatever they
//     are: in a partial block a NaN or an infinity times a weight of 0 would.
#pragma once

#include "common.h"
#include "prefill_tile.h"

namespace rag {

// Keys [0, a1) and [b0, b1) in 64-key tiles; b0 is a multiple of 64 with
// b0 >= a1, or the second span is empty.
struct KeySpans {
  int na, nb;                   // tiles of each
  int b0;
  __device__ __forceinline__ int tiles() const { return na + nb; }
  __device__ __forceinline__ int key0(int t) const {
    return t < na ? t * kPfBN : b0 + (t - na) * kPfBN;
  }
};

__device__ __forceinline__ KeySpans key_spans(int a1, int b0, int b1) {
  KeySpans k;
  k.b0 = 0;
  k.nb = 0;
  const int b0t = b0 & ~(kPfBN - 1);
  if (b1 > b0 && b0t <= a1) {                    // one span
    a1 = max(a1, b1);
  } else if (b1 > b0) {
    k.b0 = b0t;
    k.nb = (b1 - b0t + kPfBN - 1) / kPfBN;
  }
  k.na = a1 > 0 ? (a1 + kPfBN - 1) / kPfBN : 0;
  return k;
}

// Bits of a word for the keys below n of a block of 32 (n counts from its first).
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
}

// Keys of the block that the lane's row does not see (seen: one bit per key).
__device__ __forceinline__ void mt_mask(f32x16& s, uint32_t seen) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint32_t mine = seen >> (4 * half);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const int key = 8 * (j >> 2) + (j & 3);      // + 4 * half
    if (!((mine >> key) & 1)) s[j] = -INFINITY;
  }
}

// O^T += V^T P^T over the 32 keys 32*H of a stage, where some rows do not see
// some keys: with finite values as in a full block; else key by key, each for
// the rows that see it.
template <int D, int H>
__device__ __forceinline__ void mt_pv_partial(PfState<D>& st, const ChunkLayout<D>& lay,
                                              const bf16_t* __restrict__ stage,
                                              const bf16x8 (&p)[2], uint32_t seen) {
  const bf16_t* vst = stage + kPfBN * D;
  uint32_t odd = 0;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    const int rw = 32 * H + 16 * s2;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const u32x4 v = as_u32x4(join_bf16x8(lds_read_tr4(vst + lay.v_off(rw, dt)),
                                           lds_read_tr4(vst + lay.v_off(rw + 8, dt))));
#pragma unroll
      for (int e = 0; e < 4; ++e) {              // an exponent of all ones in either half
        odd |= (v[e] & 0x7f800000u) == 0x7f800000u;
        odd |= (v[e] & 0x7f80u) == 0x7f80u;
      }
    }
  }
  if (__builtin_expect(!wave_any(odd != 0), 1)) {
    pf_pv<D, H>(st, lay, stage, p);
    return;
  }
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float own = (float)p[s2][i], other = wave_xor(own, 32);
#pragma unroll 1
      for (int hf = 0; hf < 2; ++hf) {
        const int key = 16 * s2 + 8 * (i >> 2) + 4 * hf + (i & 3);
        if (!((seen >> key) & 1)) continue;
        const float w = hf == half ? own : other;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const bf16_t* v = vst + 2048 * dt + 32 * (32 * H + key) + 8 * (j >> 2) + 4 * half + (j & 3);
            st.oacc[dt][j] += w * __uint_as_float((uint32_t)*v << 16);
          }
      }
    }
  }
}

// One 32-key block of a staged tile.
template <int D, int H, class Rows>
__device__ __forceinline__ void mt_block(PfState<D>& st, const ChunkLayout<D>& lay,
                                         const bf16_t* __restrict__ stage, const Rows& rows,
                                         int k0, float c) {
  uint32_t seen = 0xffffffffu;
  const bool full = rows.full(k0);
  if (!full) {
    seen = rows.seen(k0);
    if (!wave_any(seen != 0)) return;
  }
  f32x16 s = pf_qk<D, H>(st, lay, stage);
  if (!full) mt_mask(s, seen);
  bf16x8 p[2];
  float sum = pf_weights(s, c, -st.m_used * c, p);
  if (wave_any(!(sum <= kPfSumBound))) sum = pf_reref(st, s, c, p);
  st.l += sum;
  if (full)
    pf_pv<D, H>(st, lay, stage, p);
  else
    mt_pv_partial<D, H>(st, lay, stage, p, seen);
}

// The rows of one wave against the tiles [t0, t1) of the spans.  Rows gives
// the lane's query row (q) and what it sees; KV the key rows (nk of them: rows
// behind are read from the last).
template <int D, int W, class Rows, class KV>
__device__ __forceinline__ void masked_tile(const Rows& rows, const KV& kv, const KeySpans& sp,
                                            int t0, int t1, int nk, float scale,
                                            bf16_t* __restrict__ stage, PfState<D>& st) {
  constexpr int kCh = D / 8;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const ChunkLayout<D> lay;
  const float c = scale * kLog2e;
  const bf16_t* q = rows.q() + 8 * half;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) st.qf[ks] = as_bf16x8(load16(q + 16 * ks));
  pf_reset(st);
  for (int t = t0; t < t1; ++t) {
    const int k0 = sp.key0(t);
    __syncthreads();
    for (int p = tid; p < kPfBN * kCh; p += 64 * W) {
      int r, ch;
      ChunkLayout<D>::k_src(p, r, ch);
      *reinterpret_cast<u32x4*>(stage + 8 * p) = load16(kv.krow(min(k0 + r, nk - 1)) + 8 * ch);
      ChunkLayout<D>::v_src(p, r, ch);
      *reinterpret_cast<u32x4*>(stage + kPfBN * D + 8 * p) =
          load16(kv.vrow(min(k0 + r, nk - 1)) + 8 * ch);
    }
    __syncthreads();
    mt_block<D, 0>(st, lay, stage, rows, k0, c);
    mt_block<D, 1>(st, lay, stage, rows, k0 + 32, c);
  }
}

// A row's normalised output, element j of d tile dt at
// d = 32 dt + 8 (j / 4) + 4 half + j % 4, and its log-sum-exp.
template <int D>
__device__ __forceinline__ float mt_finish(PfState<D>& st, float scale) {
  const float l = st.l + wave_xor(st.l, 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 16; ++j) st.oacc[dt][j] *= inv;
  return l == 0.f ? -INFINITY : st.m_used * scale + logf(l);
}

}  // namespace rag
