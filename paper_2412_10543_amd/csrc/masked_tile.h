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

#include <type_traits>

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

// V^T fragment of 16 keys (rows rw.. of the stage's V) and d tile dt.
template <int D>
__device__ __forceinline__ u32x4 mt_v(const ChunkLayout<D>& lay, const bf16_t* vst, int rw, int dt) {
  return as_u32x4(join_bf16x8(lds_read_tr4(vst + lay.v_off(rw, dt)),
                              lds_read_tr4(vst + lay.v_off(rw + 8, dt))));
}

// Bit 15 of each half: its bf16 value is infinite or NaN.
__device__ __forceinline__ uint32_t mt_odd(uint32_t x) {
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// O^T += V^T P^T over the 32 keys 32*H of a stage, where some rows do not see
// some keys.  With finite values this is the product of a full block.  Otherwise
// infinite and NaN values count as 0 in the product, and the rows that see them
// get theirs by two products of their own whose terms are 2^254, an infinity in
// fp32, where the row sees the key, and 0 elsewhere: +inf and NaN values give
// +inf, -inf and NaN values -inf (the two together NaN).
template <int D, int H>
__device__ __forceinline__ void mt_pv_partial(PfState<D>& st, const ChunkLayout<D>& lay,
                                              const bf16_t* __restrict__ stage,
                                              const bf16x8 (&p)[2], uint32_t seen) {
  const bf16_t* vst = stage + kPfBN * D;
  uint32_t odd = 0;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const u32x4 v = mt_v<D>(lay, vst, 32 * H + 16 * s2, dt);
      odd |= mt_odd(v[0]) | mt_odd(v[1]) | mt_odd(v[2]) | mt_odd(v[3]);
    }
  if (__builtin_expect(!wave_any(odd != 0), 1)) {
    pf_pv<D, H>(st, lay, stage, p);
    return;
  }
  asm volatile("");
  const uint32_t mine = seen >> (4 * ((threadIdx.x & 63) >> 5));
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {         // finite; +inf or NaN; -inf or NaN
    const uint32_t flip = kind == 1 ? 0xffffffffu : 0u, huge = kind == 1 ? 0x7f00u : 0xff00u;
    bf16x8 w[2];
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      u32x4 u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {              // weight i of s2: key 16 s2 + 8 (i / 4) + i % 4
        const uint32_t bits = mine >> (16 * s2 + 8 * (e >> 1) + 2 * (e & 1));
        u[e] = ((bits & 1u) | (bits & 2u) << 15) * 0x7f00u;
      }
      w[s2] = kind == 0 ? p[s2] : as_bf16x8(u);
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        u32x4 v = mt_v<D>(lay, vst, 32 * H + 16 * s2, dt);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = v[e], o = mt_odd(x), nan = ((x & 0x007f007fu) + 0x007f007fu) << 8;
          const uint32_t is = (o & ((x ^ flip) | nan)) >> 15;
          v[e] = kind == 0 ? x & ~((o >> 15) * 0xffffu) : is * huge;
        }
        st.oacc[dt] = mfma32(as_bf16x8(v), w[s2], st.oacc[dt]);
      }
  }
}

// The K/V tiles of a list of spans, copied into LDS stages (ChunkLayout) by
// all W waves: a full tile with a scalar base and per-lane 32-bit offsets, one
// that reaches past the last key row by row, from the last (finite data or not:
// those keys are masked).  For a paged cache the ids of a tile's four pages are
// read while the tile before it is issued.
template <int D, int W, class KV>
struct TileCopy {
  using Lay = ChunkLayout<D>;
  static constexpr int kCh = D / 8;
  static constexpr int kInstr = kPfBN * kCh / (64 * W);   // K (and V) instructions per wave
  static_assert(kInstr == 1 || kInstr == 2 || kInstr == 4, "tile staging layout");
  static constexpr int kLoads = 2 * kInstr;
  static_assert(4 * kInstr <= kCh && 16 * kInstr <= kPfBN, "an instruction's place in the tile");
  const KV& kv;
  const KeySpans& sp;
  int nk, wave;
  int k_page, v_page;           // page of the tile that the wave's first instruction copies
  uint32_t k_off, v_off;
  int pid[4];
  __device__ __forceinline__ TileCopy(const KV& kv_, const KeySpans& sp_, int nk_)
      : kv(kv_), sp(sp_), nk(nk_), wave(wave_id()) {
    int kr, kc, vr, vc;
    Lay::k_src(64 * wave * kInstr, kr, kc);
    Lay::v_src(64 * wave * kInstr, vr, vc);
    k_page = kr >> 4;
    v_page = vr >> 4;
    Lay::k_src(64 * wave * kInstr + (threadIdx.x & 63), kr, kc);
    Lay::v_src(64 * wave * kInstr + (threadIdx.x & 63), vr, vc);
    if constexpr (KV::kPaged) {
      k_off = (uint32_t)(((kr & 15) * D + kc * 8) * sizeof(bf16_t));
      v_off = (uint32_t)(((vr & 15) * D + vc * 8) * sizeof(bf16_t));
    } else {
      k_off = (uint32_t)((kr * kv.stride + kc * 8) * sizeof(bf16_t));
      v_off = (uint32_t)((vr * kv.stride + vc * 8) * sizeof(bf16_t));
    }
    pid[0] = pid[1] = pid[2] = pid[3] = 0;
  }
  // Page ids of the tile that is issued next.
  __device__ __forceinline__ void ids(int t, int t1) {
    if constexpr (KV::kPaged) {
      if (t >= t1) return;
      const int p0 = sp.key0(t) >> 4, last = (nk - 1) >> 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) pid[i] = kv.page(min(p0 + i, last));
    }
  }
  __device__ __forceinline__ int pick(int i) const {
    const int lo = (i & 1) ? pid[1] : pid[0], hi = (i & 1) ? pid[3] : pid[2];
    return (i & 2) ? hi : lo;
  }
  // Instruction `part` of the wave's 2 kInstr for tile t (K, V, K, V, ...); part 0
  // of a tile that reaches past the last key issues all of them.  K chunks of
  // instruction i are those of instruction 0 moved by four chunks of the same
  // rows, V's by 16 rows.
  __device__ __forceinline__ void part(bf16_t* stage, int t, int t1, int part) {
    const int k0 = sp.key0(t), i = part >> 1;
    bf16_t* dst = stage + ((part & 1) ? kPfBN * D : 0) + 64 * (wave * kInstr + i) * 8;
    if (k0 + kPfBN > nk) {
      if (part == 0) tail(stage, k0);
    } else if constexpr (KV::kPaged) {
      if (part & 1)
        dma16_s(kv.v + kv.at(pick(v_page + i), 0), v_off, dst);
      else
        dma16_s(kv.k + kv.at(pick(k_page), 0) + 32 * i, k_off, dst);
    } else {
      if (part & 1)
        dma16_s(kv.vrow(k0 + 16 * i), v_off, dst);
      else
        dma16_s(kv.krow(k0) + 32 * i, k_off, dst);
    }
    if (part == kLoads - 1) ids(t + 1, t1);
  }
  __device__ __forceinline__ void tail(bf16_t* stage, int k0) const {
    const int lane = opaque_lane();
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int g = wave * kInstr + i;
      int kr, kc, vr, vc;
      Lay::k_src(64 * g + lane, kr, kc);
      Lay::v_src(64 * g + lane, vr, vc);
      const int kj = min(k0 + kr, nk - 1), vj = min(k0 + vr, nk - 1);
      if constexpr (KV::kPaged) {
        int kr0, vr0, unused;
        Lay::k_src(64 * g, kr0, unused);
        Lay::v_src(64 * g, vr0, unused);
        // (pages past the last are the last: see ids)
        dma16(kv.k + kv.at(pick(kr0 >> 4), kj & 15) + 8 * kc, stage + 64 * g * 8);
        dma16(kv.v + kv.at(pick(vr0 >> 4), vj & 15) + 8 * vc, stage + kPfBN * D + 64 * g * 8);
      } else {
        dma16(kv.krow(kj) + 8 * kc, stage + 64 * g * 8);
        dma16(kv.vrow(vj) + 8 * vc, stage + kPfBN * D + 64 * g * 8);
      }
    }
  }
  __device__ __forceinline__ void issue(bf16_t* stage, int t, int t1) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) part(stage, t, t1, i);
  }
  // Waits until at most n tiles of this wave are in flight.
  __device__ __forceinline__ static void wait(int n) {
    constexpr int k1 = kLoads, k2 = 2 * kLoads;
    if (n >= 2)
      __builtin_amdgcn_s_waitcnt(0x0F70 | (k2 & 15) | ((k2 >> 4) << 14));
    else if (n == 1)
      __builtin_amdgcn_s_waitcnt(0x0F70 | (k1 & 15) | ((k1 >> 4) << 14));
    else
      __builtin_amdgcn_s_waitcnt(0x0F70);
  }
};

// Whether the wave's part of 32 staged V rows (32*H on) holds an infinite or NaN
// value.
template <int D, int H>
__device__ __forceinline__ uint32_t mt_look(const ChunkLayout<D>& lay, const bf16_t* stage) {
  uint32_t odd = 0;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const u32x4 v = mt_v<D>(lay, stage + kPfBN * D, 32 * H + 16 * s2, dt);
      odd |= mt_odd(v[0]) | mt_odd(v[1]) | mt_odd(v[2]) | mt_odd(v[3]);
    }
  return odd;
}

// One 32-key block of a staged tile, for masked_tile_odd.
template <int D, int H, class Rows>
__device__ __forceinline__ void mt_block(PfState<D>& st, const ChunkLayout<D>& lay,
                                         const bf16_t* __restrict__ stage, const Rows& rows,
                                         int k0, float c) {
  const uint32_t seen = rows.full(k0) ? 0xffffffffu : rows.seen(k0);
  if (!wave_any(seen != 0)) return;
  f32x16 s = pf_qk<D, H>(st, lay, stage);
  mt_mask(s, seen);
  bf16x8 p[2];
  float sum = pf_weights(s, c, -st.m_used * c, p);
  if (wave_any(!(sum <= kPfSumBound))) sum = pf_reref(st, s, c, p);
  st.l += sum;
  mt_pv_partial<D, H>(st, lay, stage, p, seen);
}

template <int D, class Rows>
__device__ __forceinline__ void mt_load_q(PfState<D>& st, const Rows& rows) {
  const bf16_t* q = rows.q() + 8 * (opaque_lane() >> 5);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) st.qf[ks] = as_bf16x8(load16(q + 16 * ks));
}

// The rows of one wave against the tiles [t0, t1) of the spans, where keys that
// some row does not see have infinite or NaN values: one tile at a time.
template <int D, int W, class Rows, class KV>
__device__ __forceinline__ void masked_tile_odd(const Rows& rows, const KV& kv, const KeySpans& sp,
                                                int t0, int t1, int nk, float scale,
                                                bf16_t* __restrict__ stage, PfState<D>& st) {
  const ChunkLayout<D> lay;
  const float c = scale * kLog2e;
  TileCopy<D, W, KV> copy(kv, sp, nk);
  mt_load_q(st, rows);
  pf_reset(st);
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    copy.ids(t, t1);
    copy.issue(stage, t, t1);
    copy.wait(0);
    pf_barrier();
    mt_block<D, 0>(st, lay, stage, rows, sp.key0(t), c);
    mt_block<D, 1>(st, lay, stage, rows, sp.key0(t) + 32, c);
    pf_barrier();
  }
}

// The rows of one wave against the tiles [t0, t1) of the spans.  Rows gives
// the lane's query row (q) and what it sees (full, seen); KV the key rows (nk of
// them).  The tile loop is prefill_items': slot b forms QK(b + 1) and PV(b - 1)
// on the matrix cores beside the weights of block b, tiles are copied three
// ahead into four stages, one barrier a tile.  Every slot is the same code, the
// first with weights and values of 0 for the block before it, the last with a
// product that nobody reads: with slots of several kinds the accumulators had
// other registers in each, and the spills made every slot wait for the copies.
// Returns whether a key that some row of the wave does not see has an infinite
// or NaN value: its weight of 0 has then made NaN of rows that it should not
// reach.
template <int D, int W, class Rows, class KV>
__device__ __forceinline__ bool masked_tile_fast(const Rows& rows, const KV& kv, const KeySpans& sp,
                                                 int t0, int t1, int nk, float scale,
                                                 bf16_t* __restrict__ s0, bf16_t* __restrict__ s1,
                                                 bf16_t* __restrict__ s2, bf16_t* __restrict__ s3,
                                                 PfState<D>& st) {
  const ChunkLayout<D> lay;
  const float c = scale * kLog2e;
  TileCopy<D, W, KV> copy(kv, sp, nk);
  bf16_t *prev = s3, *cur = s0, *next = s1, *after = s2;
  copy.ids(t0, t1);
  if (t0 < t1) copy.issue(cur, t0, t1);
  if (t0 + 1 < t1) copy.issue(next, t0 + 1, t1);
  mt_load_q(st, rows);
  pf_reset(st);
  if (t0 >= t1) return false;
  for (int i = threadIdx.x; i < kPfBN * D / 8; i += 64 * W)
    *reinterpret_cast<u32x4*>(prev + kPfBN * D + 8 * i) = u32x4{0, 0, 0, 0};
  // (the first product waits for Q, and with it for the copies before it)
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(st.qf[ks]));
  if (t0 + 2 < t1) copy.issue(after, t0 + 2, t1);
  __builtin_amdgcn_s_waitcnt(0xc07f);            // lgkmcnt(0): the zeros
  pf_barrier();

  f32x16 sE = pf_qk<D, 0>(st, lay, cur), sO = {};
  bf16x8 pE[2] = {}, pO[2] = {};
  uint32_t odd = 0;
  bool partial = false;                          // the block before was not full
  if (!rows.full(sp.key0(t0))) mt_mask(sE, rows.seen(sp.key0(t0)));
  float tmax = sE[0];
#pragma unroll
  for (int j = 1; j < 16; ++j) tmax = fmaxf(tmax, sE[j]);
  st.m_used = max_halves(tmax);
  // Block with first key k0, scores s_cur; hook as in pf_full_slot.
  auto slot = [&](auto hk, auto hv, int k0, f32x16& s_cur, f32x16& s_next, bf16x8 (&p_cur)[2],
                  const bf16x8 (&p_prev)[2], const bf16_t* kst, const bf16_t* vst,
                  const auto& hook) {
    constexpr int HK = decltype(hk)::value, HV = decltype(hv)::value;
    if (partial) odd |= mt_look<D, HV>(lay, vst);
    partial = !rows.full(k0);
    if (partial) mt_mask(s_cur, rows.seen(k0));
    float sum = pf_full_slot<D, HK, HV>(st, lay, kst, vst, s_cur, s_next, p_cur, p_prev, c,
                                        -st.m_used * c, hook);
    if (__builtin_expect(wave_any(!(sum <= kPfSumBound)), 0)) sum = pf_reref(st, s_cur, c, p_cur);
    st.l += sum;
  };
  for (int t = t0; t < t1; ++t) {
    const int k0 = sp.key0(t);
    slot(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, k0, sE, sO, pE, pO, cur,
         prev, PfNoHook{});
    if (t + 1 < t1) {
      copy.wait(t + 2 < t1 ? 1 : 0);
      pf_barrier();
    }
    bf16_t* const dst = prev;
    slot(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, k0 + 32, sO, sE, pO, pE,
         next, cur, [&](int i) {
           constexpr int kStep = D / 16 / TileCopy<D, W, KV>::kLoads;
           if (i % kStep == 0 && t + 3 < t1) copy.part(dst, t + 3, t1, i / kStep);
         });
    prev = cur;
    cur = next;
    next = after;
    after = dst;
  }
  if (partial) odd |= mt_look<D, 1>(lay, prev);
  pf_pv<D, 1>(st, lay, prev, pO);
  return wave_any(odd != 0);
}

// masked_tile_fast, and masked_tile_odd for the workgroup where a wave needs it.
template <int D, int W, class Rows, class KV>
__device__ __forceinline__ void masked_tile(const Rows& rows, const KV& kv, const KeySpans& sp,
                                            int t0, int t1, int nk, float scale,
                                            bf16_t* __restrict__ s0, bf16_t* __restrict__ s1,
                                            bf16_t* __restrict__ s2, bf16_t* __restrict__ s3,
                                            PfState<D>& st) {
  const bool odd = masked_tile_fast<D, W>(rows, kv, sp, t0, t1, nk, scale, s0, s1, s2, s3, st);
  if (__builtin_expect(__syncthreads_or(odd), 0))
    masked_tile_odd<D, W>(rows, kv, sp, t0, t1, nk, scale, s0, st);
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
