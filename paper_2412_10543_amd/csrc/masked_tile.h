// Attention of one tile of query rows to a list of key spans, with a mask per
// row, for gfx950: four waves of 32 rows each over shared blocks of 32 keys.
//
// Method: exact tiled attention with an online softmax, on the pieces of
// prefill_tile.h (S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16,
// one query row per lane).  What differs from the causal prefill:
//   * the key blocks are those of two spans (KeySpans), so that keys between
//     them cost nothing;
//   * a block is full (no mask) or partial (a 32-bit word per lane says which
//     of its keys the lane's row sees);
//   * a row may see no key at all: output 0, log-sum-exp -inf;
//   * values of keys that a row does not see never reach it, whatever they
//     are (a NaN or an infinity times a weight of 0 would);
//   * two workgroups share a CU, so that the start and the end of one, which a
//     short list of keys does not hide, run beside the products of the other.
#pragma once

#include <type_traits>

#include "common.h"
#include "prefill_tile.h"

namespace rag {

constexpr int kMtWaves = 4;
constexpr int kMtKeys = 32;      // keys of a block
constexpr int kMtRing = 4;       // blocks of K, and of V, in LDS

// Keys [0, a1) and [b0, b1) in blocks; b0 is a multiple of 32 with b0 >= a1, or
// the second span is empty.
struct KeySpans {
  int na, nb;                   // blocks of each
  int b0;
  __device__ __forceinline__ int blocks() const { return na + nb; }
  __device__ __forceinline__ int key0(int b) const {
    return b < na ? b * kMtKeys : b0 + (b - na) * kMtKeys;
  }
};

__device__ __forceinline__ KeySpans key_spans(int a1, int b0, int b1) {
  KeySpans k;
  k.b0 = 0;
  k.nb = 0;
  const int b0t = b0 & ~(kMtKeys - 1);
  if (b1 > b0 && b0t <= a1) {                    // one span
    a1 = max(a1, b1);
  } else if (b1 > b0) {
    k.b0 = b0t;
    k.nb = (b1 - b0t + kMtKeys - 1) / kMtKeys;
  }
  k.na = a1 > 0 ? (a1 + kMtKeys - 1) / kMtKeys : 0;
  return k;
}

// Element i of an array that nothing in the launch writes, i the same for the
// wave: a scalar load.
__device__ __forceinline__ int uniform_load(const int32_t* p, int i) {
  typedef __attribute__((address_space(4))) const int32_t const_i32;
  return ((const_i32*)p)[i];
}

// Bits of a word for the keys below n of a block (n counts from its first).
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
}

// LDS layout of a staged block of 32 keys, K and V in places of their own: the
// permuted chunks of ChunkLayout (which see) for half as many keys.
template <int D>
struct BlockLayout {
  static constexpr int kCh = D / 8;              // 16-byte chunks per row
  static constexpr int kElems = kMtKeys * D;     // of K, or of V
  static constexpr int kVBase = 0;
  int k_lane, v_lane;
  __device__ __forceinline__ BlockLayout() {
    const int lane = threadIdx.x & 63;
    const int l32 = lane & 31, half = lane >> 5, g16 = lane >> 4, r16 = lane & 15;
    k_lane = (l32 >> 4) * 128 * kCh + 128 * half + 8 * (l32 & 15);
    v_lane = 32 * (4 * half + (r16 >> 2)) + 16 * (g16 & 1) + 4 * (r16 & 3);
  }
  __device__ __forceinline__ int k_off(int, int ks) const { return k_lane + 256 * ks; }
  __device__ __forceinline__ int v_off(int r, int dt) const { return v_lane + 1024 * dt + 32 * r; }
  __device__ __forceinline__ static void k_src(int p, int& r, int& c) {
    r = (p / (16 * kCh)) * 16 + (p & 15);
    c = (p >> 4) % kCh;
  }
  __device__ __forceinline__ static void v_src(int p, int& r, int& c) {
    r = (p & 127) >> 2;
    c = 4 * (p >> 7) + (p & 3);
  }
};

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

// V^T fragment of 16 keys (rows rw.. of the staged V) and d tile dt.
template <int D>
__device__ __forceinline__ u32x4 mt_v(const BlockLayout<D>& lay, const bf16_t* v, int rw, int dt) {
  return as_u32x4(join_bf16x8(lds_read_tr4(v + lay.v_off(rw, dt)),
                              lds_read_tr4(v + lay.v_off(rw + 8, dt))));
}

// Bit 15 of each half: its bf16 value is infinite or NaN.
__device__ __forceinline__ uint32_t mt_odd(uint32_t x) {
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// Whether the wave's part of a staged V block holds an infinite or NaN value.
template <int D>
__device__ __forceinline__ uint32_t mt_look(const BlockLayout<D>& lay, const bf16_t* v) {
  uint32_t odd = 0;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const u32x4 x = mt_v<D>(lay, v, 16 * s2, dt);
      odd |= mt_odd(x[0]) | mt_odd(x[1]) | mt_odd(x[2]) | mt_odd(x[3]);
    }
  return odd;
}

// O^T += V^T P^T over a block where some rows do not see some keys and values
// may be infinite or NaN: those count as 0 in the product, and the rows that see
// them get theirs by two products of their own whose terms are 2^254, an infinity
// in fp32, where the row sees the key, and 0 elsewhere: +inf and NaN values give
// +inf, -inf and NaN values -inf (the two together NaN).
template <int D>
__device__ __forceinline__ void mt_pv_odd(PfState<D>& st, const BlockLayout<D>& lay,
                                          const bf16_t* __restrict__ vst, const bf16x8 (&p)[2],
                                          uint32_t seen) {
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
        u32x4 v = mt_v<D>(lay, vst, 16 * s2, dt);
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

// Copies of K and V blocks from HBM to LDS by all four waves, each kInstr
// instructions of K and as many of V: a block inside the sequence with a scalar
// base and per-lane 32-bit offsets, one that reaches past the last key row by
// row, from the last (those keys are masked).  A wave's K instructions copy rows
// of one page; the page ids that the next copies need are read beforehand (ids).
template <int D, class KV>
struct BlockCopy {
  using Lay = BlockLayout<D>;
  static constexpr int kInstr = kMtKeys * Lay::kCh / (64 * kMtWaves);
  static_assert(kInstr == 1 || kInstr == 2, "block staging layout");
  const KV& kv;
  const KeySpans& sp;
  int nk, end, wave;            // keys of the sequence; blocks end here
  int k_page, v_page;           // page in the block of the wave's first K, V instruction
  uint32_t k_off, v_off;
  int kid, vid[kInstr];
  __device__ __forceinline__ BlockCopy(const KV& kv_, const KeySpans& sp_, int nk_, int end_)
      : kv(kv_), sp(sp_), nk(nk_), end(end_), wave(wave_id()) {
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
    kid = 0;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) vid[i] = 0;
  }
  // Page ids for the copies of K block bk and V block bv.
  __device__ __forceinline__ void ids(int bk, int bv) {
    if constexpr (KV::kPaged) {
      const int last = (nk - 1) >> 4;
      if (bk < end) kid = kv.page(min((sp.key0(bk) >> 4) + k_page, last));
      if (bv < end) {
#pragma unroll
        for (int i = 0; i < kInstr; ++i)
          vid[i] = kv.page(min((sp.key0(bv) >> 4) + v_page + i, last));
      }
    }
  }
  // Have the ids in scalar registers here, and not where the copies are.
  __device__ __forceinline__ void settle() {
    if constexpr (KV::kPaged) {
      asm volatile("" : "+s"(kid));
#pragma unroll
      for (int i = 0; i < kInstr; ++i) asm volatile("" : "+s"(vid[i]));
    }
  }
  __device__ __forceinline__ void k(bf16_t* place, int b, int i) const {
    if (b >= end) return;
    const int k0 = sp.key0(b), g = wave * kInstr + i;
    bf16_t* dst = place + 512 * g;
    if (k0 + kMtKeys <= nk) {
      if constexpr (KV::kPaged)
        dma16_s(kv.k + kv.at(kid, 0) + 32 * i, k_off, dst);
      else
        dma16_s(kv.krow(k0) + 32 * i, k_off, dst);
    } else {
      int r, c;
      Lay::k_src(64 * g + opaque_lane(), r, c);
      const int j = min(k0 + r, nk - 1);         // (its page: see ids)
      if constexpr (KV::kPaged)
        dma16(kv.k + kv.at(kid, j & 15) + 8 * c, dst);
      else
        dma16(kv.krow(j) + 8 * c, dst);
    }
  }
  __device__ __forceinline__ void v(bf16_t* place, int b, int i) const {
    if (b >= end) return;
    const int k0 = sp.key0(b), g = wave * kInstr + i;
    bf16_t* dst = place + 512 * g;
    if (k0 + kMtKeys <= nk) {
      if constexpr (KV::kPaged)
        dma16_s(kv.v + kv.at(vid[i], 0), v_off, dst);
      else
        dma16_s(kv.vrow(k0 + 16 * i), v_off, dst);
    } else {
      int r, c;
      Lay::v_src(64 * g + opaque_lane(), r, c);
      const int j = min(k0 + r, nk - 1);
      if constexpr (KV::kPaged)
        dma16(kv.v + kv.at(vid[i], j & 15) + 8 * c, dst);
      else
        dma16(kv.vrow(j) + 8 * c, dst);
    }
  }
  __device__ __forceinline__ void both(bf16_t* kp, int bk, bf16_t* vp, int bv) {
    ids(bk, bv);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) v(vp, bv, i);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) k(kp, bk, i);
  }
};

// The lane's query row.
template <int D>
__device__ __forceinline__ void mt_load_q(PfState<D>& st, const bf16_t* row) {
  const bf16_t* q = row + 8 * (opaque_lane() >> 5);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) st.qf[ks] = as_bf16x8(load16(q + 16 * ks));
}

// The rows of one wave against the blocks [b0, b1) of the spans, where keys that
// some row does not see have infinite or NaN values: one block at a time.
template <int D, class Rows, class KV>
__device__ __forceinline__ void masked_tile_odd(const Rows& rows, const KV& kv, const KeySpans& sp,
                                                int b0, int b1, int nk, float scale,
                                                bf16_t* __restrict__ kst, bf16_t* __restrict__ vst,
                                                PfState<D>& st) {
  const BlockLayout<D> lay;
  const float c = scale * kLog2e;
  BlockCopy<D, KV> copy(kv, sp, nk, b1);
  pf_reset(st);
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    copy.both(kst, b, vst, b);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    pf_barrier();
    const int k0 = sp.key0(b);
    const uint32_t seen = rows.full(k0) ? 0xffffffffu : rows.seen(k0);
    if (wave_any(seen != 0)) {
      f32x16 s = pf_qk<D, 0>(st, lay, kst);
      mt_mask(s, seen);
      bf16x8 p[2];
      float sum = pf_weights(s, c, -st.m_used * c, p);
      if (wave_any(!(sum <= kPfSumBound))) sum = pf_reref(st, s, c, p);
      st.l += sum;
      mt_pv_odd<D>(st, lay, vst, p, seen);
    }
    pf_barrier();
  }
}

// The rows of one wave against the blocks [b0, b1) of the spans.  Rows gives
// what the lane's row sees (full, seen), st.qf its query; KV the key rows (nk of
// them).  As in prefill_items, slot b forms QK(b + 1) and PV(b - 1) on the matrix
// cores beside the weights of block b.  K(b + 4) and V(b + 2) are requested in
// slot b, into the places of K(b) and V(b - 2), which slot b - 1 was the last to
// read; a barrier before every slot.  Every slot is the same code, the first with
// weights and values of 0 for the block before it, the last with a product that
// nobody reads, and an odd number of blocks with an empty one behind: with slots
// of several kinds the accumulators had other registers in each, and the spills
// made every slot wait for the copies (docs of 512 keys in a 5800-token prompt,
// 16 of them: 2273 us against 1441).
// Returns whether a key that some row of the wave does not see has an infinite
// or NaN value: its weight of 0 has then made NaN of rows that it should not
// reach.
template <int D, class Rows, class KV>
__device__ __forceinline__ bool masked_tile_fast(const Rows& rows, const KV& kv, const KeySpans& sp,
                                                 int b0, int b1, int nk, float scale,
                                                 bf16_t* __restrict__ kring,
                                                 bf16_t* __restrict__ vring, PfState<D>& st) {
  using Lay = BlockLayout<D>;
  const Lay lay;
  const float c = scale * kLog2e;
  const int n = b1 - b0;
  BlockCopy<D, KV> copy(kv, sp, nk, b1);
  constexpr int kInstr = BlockCopy<D, KV>::kInstr;
  auto kat = [&](int i) { return kring + (i & (kMtRing - 1)) * Lay::kElems; };
  auto vat = [&](int i) { return vring + (i & (kMtRing - 1)) * Lay::kElems; };
  copy.both(kat(0), b0, vat(0), b0);
  copy.both(kat(1), b0 + 1, vat(1), b0 + 1);
  copy.both(kat(2), b0 + 2, vat(2), b1);
  copy.both(kat(3), b0 + 3, vat(3), b1);
  pf_reset(st);
  if (n <= 0) return false;
  copy.ids(b0 + 4, b0 + 2);
  for (int i = threadIdx.x; i < Lay::kElems / 8; i += 64 * kMtWaves)
    *reinterpret_cast<u32x4*>(vat(3) + 8 * i) = u32x4{0, 0, 0, 0};
  // (the first product waits for Q, and with it for the copies before it)
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(st.qf[ks]));
  __builtin_amdgcn_s_waitcnt(0x0070);            // the copies and the zeros
  pf_barrier();
  copy.settle();

  f32x16 sE = pf_qk<D, 0>(st, lay, kat(0)), sO = {};
  bf16x8 pE[2] = {}, pO[2] = {};
  uint32_t odd = 0;
  bool partial = false;                          // the block before was not full
  if (!rows.full(sp.key0(b0))) mt_mask(sE, rows.seen(sp.key0(b0)));
  float tmax = sE[0];
#pragma unroll
  for (int j = 1; j < 16; ++j) tmax = fmaxf(tmax, sE[j]);
  st.m_used = max_halves(tmax);
  // Block b0 + i with scores s_cur.
  auto slot = [&](int i, f32x16& s_cur, f32x16& s_next, bf16x8 (&p_cur)[2],
                  const bf16x8 (&p_prev)[2]) {
    if (partial) odd |= mt_look<D>(lay, vat(i - 1));
    const int k0 = sp.key0(b0 + i);
    partial = !rows.full(k0) || i >= n;
    if (partial) mt_mask(s_cur, i < n ? rows.seen(k0) : 0u);
    float sum = pf_full_slot<D, 0, 0>(
        st, lay, kat(i + 1), vat(i - 1), s_cur, s_next, p_cur, p_prev, c, -st.m_used * c,
        [&](int step) {                          // V and K of later blocks, spread over the slot
          constexpr int kStep = D / 16 / (2 * kInstr);
          if (step % kStep == 0) {
            const int x = step / kStep;
            if (x < kInstr)
              copy.v(vat(i + 2), b0 + i + 2, x);
            else
              copy.k(kat(i), b0 + i + 4, x - kInstr);
          }
        });
    if (__builtin_expect(wave_any(!(sum <= kPfSumBound)), 0)) sum = pf_reref(st, s_cur, c, p_cur);
    st.l += sum;
  };
  // Slot i + 1 needs K(i + 2) and V(i), requested in slot i - 2 at the latest.
  auto turn = [&](int i) {
    __builtin_amdgcn_sched_barrier(0);
    copy.ids(b0 + i + 5, b0 + i + 3);
    constexpr int k2 = 4 * kInstr;               // the copies of two slots
    if (i + 4 < n)
      __builtin_amdgcn_s_waitcnt(0x0F70 | k2);
    else
      __builtin_amdgcn_s_waitcnt(0x0F70);
    pf_barrier();
    copy.settle();
  };
  int i = 0;
  for (; i < n; i += 2) {
    slot(i, sE, sO, pE, pO);
    turn(i);
    slot(i + 1, sO, sE, pO, pE);
    turn(i + 1);
  }
  if (i == n) {                                  // (else the empty block was the last)
    if (partial) odd |= mt_look<D>(lay, vat(n - 1));
    pf_pv<D, 0>(st, lay, vat(n - 1), pO);
  }
  return wave_any(odd != 0);
}

// masked_tile_fast, and masked_tile_odd for the workgroup where a wave needs it.
template <int D, class Rows, class KV>
__device__ __forceinline__ void masked_tile(const Rows& rows, const KV& kv, const KeySpans& sp,
                                            int b0, int b1, int nk, float scale,
                                            bf16_t* __restrict__ kring, bf16_t* __restrict__ vring,
                                            PfState<D>& st) {
  const bool odd = masked_tile_fast<D>(rows, kv, sp, b0, b1, nk, scale, kring, vring, st);
  if (__builtin_expect(__syncthreads_or(odd), 0))
    masked_tile_odd<D>(rows, kv, sp, b0, b1, nk, scale, kring, vring, st);
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

// Stores the lane's row (of the two lanes that hold a row, each the half of every
// 16 values): the halves trade four values for four, and each then stores 16
// bytes at a time.
template <int D>
__device__ __forceinline__ void mt_store(const PfState<D>& st, bf16_t* row, bool valid) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      const f32x16& o = st.oacc[dt];
      const bf16x4 a = to_bf16x4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
      const bf16x4 b = to_bf16x4(o[4 * g + 4], o[4 * g + 5], o[4 * g + 6], o[4 * g + 7]);
      const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
      // lane 0..31: a's first half from itself, its second from lane + 32; the
      // other lanes the same of b
      const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
      const u32x4 w = {s0[0], s1[0], s0[1], s1[1]};
      if (valid) *reinterpret_cast<u32x4*>(row + 32 * dt + 8 * (g + half)) = w;
    }
}

}  // namespace rag
