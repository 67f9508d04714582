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

#include "common.h"
#include "prefill_tile.h"

namespace rag {

constexpr int kMtWaves = 4;
constexpr int kMtKeys = 32;      // keys of a block
constexpr int kMtRing = 4;       // blocks of K, and of V, in LDS
#ifndef RAG_MT_AHEAD
#define RAG_MT_AHEAD 3
#endif
constexpr int kMtAhead = RAG_MT_AHEAD;   // steps of a slot that LDS reads run ahead

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

// The full blocks of a wave: [0, a) and [lo, lo + n) of the list.
struct FullBlocks {
  int a, lo;
  uint32_t n;
  __device__ __forceinline__ bool at(int b) const { return b < a || (uint32_t)(b - lo) < n; }
};

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
  // (row, chunk) of the block held by staged chunk p
  __device__ __forceinline__ static void k_src(uint32_t p, int& r, int& c) {
    r = (int)(p / (16 * kCh) * 16 + (p & 15));
    c = (int)((p >> 4) % kCh);
  }
  __device__ __forceinline__ static void v_src(uint32_t p, int& r, int& c) {
    r = (int)((p & 127) >> 2);
    c = (int)(4 * (p >> 7) + (p & 3));
  }
};

// Keys of the block that the lane's row does not see (seen: one bit per key).
__device__ __forceinline__ void mt_mask(f32x16& s, uint32_t seen) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint32_t mine = seen >> (4 * half);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const int key = 8 * (j >> 2) + (j & 3);      // + 4 * half
    const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)mine, key, 1);   // all ones or 0
    const uint32_t x = __float_as_uint(s[j]);
    s[j] = __uint_as_float((x & keep) | (0xff800000u & ~keep));
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

// dma16_s with the LDS address as a byte offset.
__device__ __forceinline__ void dma16_at(const void* sbase, uint32_t voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(voff), "s"(sbase), "s"(lds)
      : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_offset(const bf16_t* p) {
  typedef __attribute__((address_space(3))) char lds_char;
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char*)p);
}

// One side (K or V) of the copies of blocks from HBM to LDS by all four waves,
// kInstr instructions a wave and block, each with a scalar base and per-lane 32-bit
// offsets.  Blocks are requested in the order of the spans.  What a slot copies
// is prepared before the slot (ids, then next), as scalar instructions between the
// products of a wave cost as much as vector ones.  Only the last block can reach
// past the sequence's last key: its offsets then repeat that key's row (those keys
// are masked).  Behind the last block copies go on, of one 16-byte piece of it for
// all lanes, into places that nobody reads: the slots stay one code, and the number
// of copies in flight one number.
template <int D, class KV, bool kIsK>
struct BlockCopy {
  using Lay = BlockLayout<D>;
  static constexpr int kInstr = kMtKeys * Lay::kCh / (64 * kMtWaves);
  static_assert(kInstr == 1 || kInstr == 2, "block staging layout");
  static constexpr uint32_t kPlace = Lay::kElems * sizeof(bf16_t);
  const KV& kv;
  int nk, last;                 // keys of the sequence; last block
  int page;                     // page in the block of the wave's first instruction
  int b, na, k0, k0b;           // next block and its first key; the spans' border
  int id[kInstr];               // its page ids (K: all of a wave's rows are in one page)
  uint32_t off[kInstr], ring;
  const bf16_t* base[kInstr];
  __device__ __forceinline__ BlockCopy(const KV& kv_, const KeySpans& sp, int nk_, int b0, int b1,
                                       const bf16_t* ring_)
      : kv(kv_), nk(nk_), last(b1 - 1), b(b0), na(sp.na), k0(sp.key0(b0)), k0b(sp.b0) {
    const int wave = wave_id();
    ring = lds_offset(ring_) + 1024 * wave * kInstr;
    int r, c;
    src(64 * wave * kInstr, r, c);
    page = r >> 4;
    offsets(0, 1 << 30);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) id[i] = 0;
  }
  __device__ __forceinline__ static void src(int p, int& r, int& c) {
    if constexpr (kIsK) Lay::k_src(p, r, c); else Lay::v_src(p, r, c);
  }
  // Offsets of the lane's chunks for a block that starts at key k0 of n.
  __device__ __forceinline__ void offsets(int first, int n) {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      int r, c;
      src(64 * (wave_id() * kInstr + i) + opaque_lane(), r, c);
      r = min(r, n - 1 - first);
      if constexpr (KV::kPaged)
        off[i] = (uint32_t)((((first + r) & 15) * D + c * 8) * sizeof(bf16_t));
      else
        off[i] = (uint32_t)((r * kv.stride + c * 8) * sizeof(bf16_t));
    }
  }
  // Page ids of the next block (pages past the last are the last: see offsets).
  __device__ __forceinline__ void ids() {
    if constexpr (KV::kPaged) {
      const int p = (k0 >> 4) + page, lp = (nk - 1) >> 4;
      id[0] = kv.page(min(p, lp));
      if constexpr (kInstr == 2) id[1] = kIsK ? id[0] : kv.page(min(p + 1, lp));
    }
  }
  // The next block's copies from here on.
  __device__ __forceinline__ void next() {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      if constexpr (KV::kPaged) {
        asm volatile("" : "+s"(id[i]));
        base[i] = (kIsK ? kv.k : kv.v) + kv.at(id[i], 0);
      } else {
        base[i] = (kIsK ? kv.k : kv.v) + (size_t)((uint64_t)(uint32_t)k0 * (uint32_t)kv.stride);
      }
    }
    if (b >= last) end_of_list();
    const bool more = b < last;                  // (stays at the last block)
    const int after = b + 1 == na ? k0b : k0 + kMtKeys;
    k0 = more ? after : k0;
    b = more ? b + 1 : last + 1;
  }
  __device__ __forceinline__ void end_of_list() {
    asm volatile("");
    if (b > last) {
#pragma unroll
      for (int i = 0; i < kInstr; ++i) off[i] = 0;
    } else if (k0 + kMtKeys > nk) {
      offsets(k0, nk);
    }
  }
  __device__ __forceinline__ void copy(int place, int i) const {
    dma16_at(base[i], off[i], ring + place * kPlace + 1024 * i);
  }
  __device__ __forceinline__ void all(int place) {
    ids();
    next();
#pragma unroll
    for (int i = 0; i < kInstr; ++i) copy(place, i);
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
  BlockCopy<D, KV, true> kc(kv, sp, nk, b0, b1, kst);
  BlockCopy<D, KV, false> vc(kv, sp, nk, b0, b1, vst);
  pf_reset(st);
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    kc.all(0);
    vc.all(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    pf_barrier();
    const int k0 = sp.key0(b);
    const uint32_t seen = rows.seen(k0);
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
// what the lane's row sees (full_blocks, seen), st.qf its query; KV the key rows
// (nk of them).  As in prefill_items, slot b forms QK(b + 1) and PV(b - 1) on the matrix
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
  pf_reset(st);
  if (n <= 0) return false;
  BlockCopy<D, KV, true> kc(kv, sp, nk, b0, b1, kring);
  BlockCopy<D, KV, false> vc(kv, sp, nk, b0, b1, vring);
  constexpr int kInstr = BlockCopy<D, KV, true>::kInstr;
  auto kat = [&](int i) { return kring + (i & (kMtRing - 1)) * Lay::kElems; };
  auto vat = [&](int i) { return vring + (i & (kMtRing - 1)) * Lay::kElems; };
  kc.all(0);
  vc.all(0);
  kc.all(1);
  vc.all(1);
  kc.all(2);
  kc.all(3);
  kc.ids();
  vc.ids();
  for (int i = threadIdx.x; i < Lay::kElems / 8; i += 64 * kMtWaves)
    *reinterpret_cast<u32x4*>(vat(3) + 8 * i) = u32x4{0, 0, 0, 0};
  // (the first product waits for Q, and with it for the copies before it)
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(st.qf[ks]));
  __builtin_amdgcn_s_waitcnt(0x0070);            // the copies and the zeros
  pf_barrier();
  kc.next();
  vc.next();

  f32x16 sE = pf_qk<D, 0>(st, lay, kat(0)), sO = {};
  bf16x8 pE[2] = {}, pO[2] = {};
  uint32_t odd = 0;
  bool partial = false;                          // the block before was not full
  const FullBlocks fb = rows.full_blocks(sp);
  if (!fb.at(b0)) mt_mask(sE, rows.seen(sp.key0(b0)));
  float tmax = sE[0];
#pragma unroll
  for (int j = 1; j < 16; ++j) tmax = fmaxf(tmax, sE[j]);
  st.m_used = max_halves(tmax);
  // Block b0 + i with scores s_cur.
  auto slot = [&](int i, f32x16& s_cur, f32x16& s_next, bf16x8 (&p_cur)[2],
                  const bf16x8 (&p_prev)[2]) {
    if (partial) odd |= mt_look<D>(lay, vat(i - 1));
    partial = !fb.at(b0 + i) || i >= n;
    if (partial) mt_mask(s_cur, i < n ? rows.seen(sp.key0(b0 + i)) : 0u);
    float sum = pf_full_slot<D, 0, 0, Lay, kMtAhead>(
        st, lay, kat(i + 1), vat(i - 1), s_cur, s_next, p_cur, p_prev, c, -st.m_used * c,
        [&](int step) {                          // V and K of later blocks, spread over the slot
          constexpr int kStep = D / 16 / (2 * kInstr);
          if (step % kStep == 0) {
            const int x = step / kStep;
            if (x < kInstr)
              vc.copy((i + 2) & (kMtRing - 1), x);
            else
              kc.copy(i & (kMtRing - 1), x - kInstr);
          }
        });
    if (__builtin_expect(wave_any(!(sum <= kPfSumBound)), 0)) sum = pf_reref(st, s_cur, c, p_cur);
    st.l += sum;
  };
  // Slot i + 1 needs K(i + 2) and V(i), requested in slot i - 2 at the latest.
  auto turn = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    kc.ids();
    vc.ids();
    __builtin_amdgcn_s_waitcnt(0x0F70 | 4 * kInstr);   // the copies of two slots
    pf_barrier();
    kc.next();
    vc.next();
  };
  int i = 0;
  for (; i < n; i += 2) {
    slot(i, sE, sO, pE, pO);
    turn();
    slot(i + 1, sO, sE, pO, pE);
    turn();
  }
  if (i == n) {                                  // (else the empty block was the last)
    if (partial) odd |= mt_look<D>(lay, vat(n - 1));
    pf_pv<D, 0>(st, lay, vat(n - 1), pO);
  }
  // (no copy into LDS outlives the workgroup, or meets its next use of the rings)
  __builtin_amdgcn_s_waitcnt(0x0F70);
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
