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

template <int kN>
struct MtInt {
  static constexpr int value = kN;
};

constexpr int kMtWaves = 4;
constexpr int kMtKeys = 32;      // keys of a block
constexpr int kMtRing = 4;       // blocks of K, and of V, in LDS

// The blocks of an item: na from key a0 on, then nb from key b0 on (both multiples
// of 32).
struct KeySpans {
  int a0, na, b0, nb;
  __device__ __forceinline__ int blocks() const { return na + nb; }
  __device__ __forceinline__ int key0(int b) const {
    return b < na ? a0 + b * kMtKeys : b0 + (b - na) * kMtKeys;
  }
};

// Keys [0, a1) and [b0, b1).
__device__ __forceinline__ KeySpans key_spans(int a1, int b0, int b1) {
  KeySpans k{0, 0, 0, 0};
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

// The blocks of an item that all its rows see whole: [0, a) and [lo, hi) of its
// list.
struct FullBlocks {
  int a, lo, hi;
  // How many from block b on.
  __device__ __forceinline__ int run(int b) const {
    return b < a ? a - b : b >= lo && b < hi ? hi - b : 0;
  }
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

// Whether the wave's quarter of a staged V block holds an infinite or NaN value
// (a block is partial for all four waves or for none).
template <int D>
__device__ __forceinline__ uint32_t mt_look(const bf16_t* v) {
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(
        v + ((wave_id() * (D / 64) + i) * kWave + opaque_lane()) * 8);
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

// dma16_s with the LDS address as a byte offset, kPlus bytes behind lds.
template <int kPlus>
__device__ __forceinline__ void dma16_at(const void* sbase, uint32_t voff, uint32_t lds) {
  asm volatile(
      "s_add_u32 m0, %2, %3\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(voff), "s"(sbase), "s"(lds), "n"(kPlus)
      : "memory", "m0", "scc");
}

__device__ __forceinline__ uint32_t lds_offset(const bf16_t* p) {
  typedef __attribute__((address_space(3))) char lds_char;
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char*)p);
}

// Slots of an item of n blocks: an even number, and at least a ring's where another
// item follows, whose first K blocks are requested in those last slots.
__device__ __forceinline__ int mt_slots(int n, bool more) {
  const int even = (n + 1) & ~1;
  return more ? max(even, kMtRing) : even;
}

// One side (K or V) of the copies of blocks from HBM to LDS by all four waves,
// kInstr instructions a wave and block, each with a scalar base and per-lane 32-bit
// offsets.  The blocks of an item are requested in the order of its spans, those
// of the next item behind them.  What a slot copies is prepared before the slot
// (ready, then next), and counted in runs of blocks, as scalar instructions between
// the products of a wave cost as much as vector ones.  A block that reaches past
// the sequence's last key repeats that key's row (those keys are masked).  Slots
// without a block copy one 16-byte piece for all lanes, into places that nobody
// reads: the slots stay one code, and the number of copies in flight one number.
template <int D, class KV, bool kIsK>
struct BlockCopy {
  using Lay = BlockLayout<D>;
  static constexpr int kInstr = kMtKeys * Lay::kCh / (64 * kMtWaves);
  static_assert(kInstr == 1 || kInstr == 2, "block staging layout");
  KV kv;
  int nk;                       // keys of the sequence, at least one
  int page;                     // page in the block of the wave's first instruction
  int run;                      // blocks left of the run at hand
  int b, n, slots, na, a0, b0;  // the item: slots begun or in the run; blocks; spans
  int p, dp;                    // paged: the next block's first page, pages per block
  int id[kInstr];               //   and its page ids (K: all of a wave's rows in one page)
  const bf16_t* at;             // dense: the next block's first row,
  uint32_t step;                //   and elements to the one behind it
  const bf16_t* base[kInstr];   // the copies of the slot
  uint32_t off[kInstr], usual[kInstr], ring;
  __device__ __forceinline__ BlockCopy(const KV& kv_, int nk_, const bf16_t* ring_)
      : kv(kv_), nk(nk_) {
    const int wave = wave_id();
    ring = lds_offset(ring_) + 1024 * wave * kInstr;
    int r, c;
    src(64 * wave * kInstr, r, c);
    page = r >> 4;
    offsets(usual, 0, 1 << 30);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      off[i] = usual[i];
      id[i] = 0;
    }
    run = 0;
    p = dp = 0;
    at = kIsK ? kv.k : kv.v;
    step = 0;
  }
  __device__ __forceinline__ void item(const KeySpans& sp, int slots_) {
    b = 0;
    n = sp.blocks();
    slots = slots_;
    na = sp.na;
    a0 = sp.a0;
    b0 = sp.b0;
  }
  __device__ __forceinline__ static void src(int q, int& r, int& c) {
    if constexpr (kIsK) Lay::k_src(q, r, c); else Lay::v_src(q, r, c);
  }
  // Offsets of the lane's chunks for a block that starts at key `first` of n.
  __device__ __forceinline__ void offsets(uint32_t (&o)[kInstr], int first, int n) {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      int r, c;
      src(64 * (wave_id() * kInstr + i) + opaque_lane(), r, c);
      r = min(r, n - 1 - first);
      if constexpr (KV::kPaged)
        o[i] = (uint32_t)((((first + r) & 15) * D + c * 8) * sizeof(bf16_t));
      else
        o[i] = (uint32_t)((r * kv.stride + c * 8) * sizeof(bf16_t));
    }
  }
  // The run from slot b of the item on; behind its last slot the next item's
  // (after_slots 0: there is none).
  __device__ __forceinline__ void refill(const KeySpans& after, int after_slots) {
    asm volatile("");
    if (b >= slots && after_slots > 0) item(after, after_slots);
    if (b >= n) {                                // no block
      run = max(slots - b, 1);
      dp = 0;
      at = kIsK ? kv.k : kv.v;                   // (at is behind the last block by now)
      step = 0;
#pragma unroll
      for (int i = 0; i < kInstr; ++i) off[i] = 0;
    } else {
      const bool first = b < na;
      const int k0 = first ? a0 + b * kMtKeys : b0 + (b - na) * kMtKeys;
      const int inside = (nk - k0) / kMtKeys;    // whole blocks
      run = min((first ? na : n) - b, max(inside, 1));
      p = k0 >> 4;
      dp = kMtKeys / 16;
      if constexpr (!KV::kPaged) {
        at = (kIsK ? kv.k : kv.v) + (size_t)k0 * kv.stride;
        step = (uint32_t)(kMtKeys * kv.stride);
      }
#pragma unroll
      for (int i = 0; i < kInstr; ++i) off[i] = usual[i];
      if (inside < 1) offsets(off, k0, nk);
    }
    b += run;
  }
  // Before the slot's barrier: the next block's page ids (pages past the last are
  // the last: see offsets).
  __device__ __forceinline__ void ready(const KeySpans& after, int after_slots) {
    if (run == 0) refill(after, after_slots);
    if constexpr (KV::kPaged) {
      const int lp = (nk - 1) >> 4;
      id[0] = kv.page(min(p + page, lp));
      if constexpr (kInstr == 2) id[1] = kIsK ? id[0] : kv.page(min(p + page + 1, lp));
    }
  }
  // And behind it: the slot's copies are the next block's.
  __device__ __forceinline__ void next() {
    --run;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      if constexpr (KV::kPaged) {
        asm volatile("" : "+s"(id[i]));
        base[i] = (kIsK ? kv.k : kv.v) + kv.at(id[i], 0);
      } else {
        base[i] = at;
      }
    }
    if constexpr (KV::kPaged) p += dp; else at += step;
  }
  // Instruction i into the place at byte `place` + kPlus of the ring.
  template <int kPlus>
  __device__ __forceinline__ void copy(uint32_t place, int i) const {
    if (i == 0)
      dma16_at<kPlus>(base[0], off[0], ring + place);
    else
      dma16_at<kPlus + 1024>(base[kInstr - 1], off[kInstr - 1], ring + place);
  }
  __device__ __forceinline__ void all(int place) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) copy<0>(place * Lay::kElems * sizeof(bf16_t), i);
  }
};

// Rows of a wave go to and from memory as 64-byte pieces, 16 rows an instruction,
// through 2 KiB of LDS of the wave's own (io: 32 rows of 64 bytes, 16-byte chunk c
// of row r at c ^ (r / 4) % 4), where a lane has its own row.  (A lane's row in
// 16-byte pieces straight from memory, 8-byte ones back, is 64 pieces an instruction:
// 16 prompts of 5 to 20 documents of 400 to 512 tokens 958 us for 880, with windows 1242
// for 1154; trees, of fewer rows, the same.)
__device__ __forceinline__ int io_at(int r, int c) { return 32 * r + 8 * (c ^ ((r >> 2) & 3)); }

// The lane's query row: rows(r) is row r of the wave's 32.
template <int D, class RowPtr>
__device__ __forceinline__ void mt_request_q(PfState<D>& st, const RowPtr& rows) {
  const int lane = opaque_lane(), c = lane & 3;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bf16_t* q = rows((lane >> 2) + 16 * i) + 8 * c;
#pragma unroll
    for (int p = 0; p < D / 32; ++p) st.qf[2 * p + i] = as_bf16x8(load16(q + 32 * p));
  }
}
template <int D>
__device__ __forceinline__ void mt_place_q(PfState<D>& st, bf16_t* io) {
  const int lane = opaque_lane(), c = lane & 3, r = lane & 31, half = lane >> 5;
#pragma unroll
  for (int p = 0; p < D / 32; ++p) {             // columns 32 p on
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<bf16x8*>(io + io_at((lane >> 2) + 16 * i, c)) = st.qf[2 * p + i];
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < 2; ++i)
      st.qf[2 * p + i] = *reinterpret_cast<const bf16x8*>(io + io_at(r, 2 * i + half));
    wave_lds_sync();
  }
}

// A row's normalised output, element j of d tile dt at
// d = 32 dt + 8 (j / 4) + 4 half + j % 4; returns its sum of weights.
template <int D>
__device__ __forceinline__ float mt_finish(PfState<D>& st) {
  const float l = st.l + wave_xor(st.l, 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 16; ++j) st.oacc[dt][j] *= inv;
  return l;
}
// And its log-sum-exp.
template <int D>
__device__ __forceinline__ float mt_lse(const PfState<D>& st, float l, float scale) {
  return l == 0.f ? -INFINITY : st.m_used * scale + logf(l);
}

// Stores the wave's rows: rows(r) is where row r goes, or null.
template <int D, class RowPtr>
__device__ __forceinline__ void mt_store(const PfState<D>& st, bf16_t* io, const RowPtr& rows) {
  const int lane = opaque_lane(), c = lane & 3, r = lane & 31, half = lane >> 5;
  bf16_t* const to[2] = {rows(lane >> 2), rows((lane >> 2) + 16)};
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    const f32x16& o = st.oacc[dt];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<bf16x4*>(io + io_at(r, g) + 4 * half) =
          to_bf16x4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(io + io_at((lane >> 2) + 16 * i, c));
      if (to[i] != nullptr) *reinterpret_cast<u32x4*>(to[i] + 32 * dt + 8 * c) = x;
    }
    wave_lds_sync();
  }
}

// The same in fp32.
template <int D, class RowPtr>
__device__ __forceinline__ void mt_store_f32(const PfState<D>& st, bf16_t* io_, const RowPtr& rows) {
  const int lane = opaque_lane(), c = lane & 3, r = lane & 31, half = lane >> 5;
  float* const to[2] = {rows(lane >> 2), rows((lane >> 2) + 16)};
  float* io = reinterpret_cast<float*>(io_);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {                // columns 32 dt + 16 h on
      const f32x16& o = st.oacc[dt];
#pragma unroll
      for (int g = 2 * h; g < 2 * h + 2; ++g)
        *reinterpret_cast<f32x4*>(io + io_at(r, 2 * (g & 1) + half) / 2) =
            f32x4{o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]};
      wave_lds_sync();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(io + io_at((lane >> 2) + 16 * i, c) / 2);
        if (to[i] != nullptr) *reinterpret_cast<f32x4*>(to[i] + 32 * dt + 16 * h + 4 * c) = x;
      }
      wave_lds_sync();
    }
}

// The rows of one wave against the blocks of an item, where keys that some row
// does not see have infinite or NaN values: one block at a time.  st.qf is set.
template <int D, class Rows, class KV>
__device__ __forceinline__ void masked_item_odd(const Rows& rows, const KV& kv, const KeySpans& sp,
                                                int nk, float scale, bf16_t* __restrict__ kst,
                                                bf16_t* __restrict__ vst, PfState<D>& st) {
  const BlockLayout<D> lay;
  const float c = scale * kLog2e;
  const int n = sp.blocks();
  BlockCopy<D, KV, true> kc(kv, nk, kst);
  BlockCopy<D, KV, false> vc(kv, nk, vst);
  kc.item(sp, n);
  vc.item(sp, n);
  pf_reset(st);
#pragma unroll 1
  for (int b = 0; b < n; ++b) {
    kc.ready(sp, 0);
    vc.ready(sp, 0);
    kc.next();
    vc.next();
    kc.all(0);
    vc.all(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    pf_barrier();
    const uint32_t seen = rows.seen(sp.key0(b));
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

// LDS of a workgroup: rings of K and V blocks, a block of zeros, and the waves'
// 2 KiB for rows to and from memory (80 KiB at D = 128: two workgroups a CU; rings
// of eight blocks where a launch leaves one to a CU cost 0.7 to 2.3 us a call, of
// 10 to 20, for the longer start, and gained nothing).
template <int D>
struct MtLds {
  bf16_t k[kMtRing * BlockLayout<D>::kElems];
  bf16_t v[kMtRing * BlockLayout<D>::kElems];
  bf16_t zero[BlockLayout<D>::kElems];
  bf16_t io[kMtWaves][1024];
};

// The items of a workgroup, one after another: 128 (row, head) pairs each, 32 of
// them a wave's, against the blocks of the item's spans.  All items are of one
// sequence and kv head (kv, of nk >= 1 keys).  Src:
//   count               items
//   Rows rows           of the item settled last: what the lane's row sees
//   fetch(m)            requests what item m's rows and spans follow from
//   settle(m)           the spans of item m, from what was fetched last, and rows
//   q(m, r)             row r of the wave's 32 query rows
//   store(m, st, l, scale, io)   writes the wave's rows; l: the lane's row's sum of weights
// As in prefill_items, slot i of an item forms QK(i + 1) and PV(i - 1) on the
// matrix cores beside the weights of block i.  K(i + 4) and V(i + 2) are requested
// in slot i, into the places of K(i) and V(i - 2), which slot i - 1 was the last to
// read; a barrier before every slot.  The last slots of an item request the first
// blocks of the next, so that between items only its queries are waited for
// (beside the other workgroup's products).  Every slot is the same code, the
// first with zeros as the values of the block before it, and slots without a
// block (their number is even) with weights of 0: with slots of several kinds the
// accumulators had other registers in each, and the spills made every slot wait
// for the copies (in a first form, with eight waves and tiles of 64 keys, 16 prompts
// of 5 to 20 documents: 2273 us against 1441).
// Returns the items (a bit each) where a key that some row of the wave does not
// see has an infinite or NaN value: its weight of 0 has then made NaN of rows that
// it should not reach.
template <int D, class Src, class KV>
__device__ __forceinline__ uint32_t masked_items_fast(Src& src, const KV& kv, int nk, float scale,
                                                      MtLds<D>& lds) {
  using Lay = BlockLayout<D>;
  const Lay lay;
  const float c = scale * kLog2e;
  PfState<D> st;
  bf16_t* const io = lds.io[wave_id()];
  src.fetch(0);
  mt_request_q<D>(st, [&](int r) { return src.q(0, r); });
  KeySpans sp = src.settle(0), sp_next{0, 0, 0, 0};
  auto rows = src.rows;
  auto rows_next = rows;
  int slots = mt_slots(sp.blocks(), src.count > 1), slots_next = 0;
  BlockCopy<D, KV, true> kc(kv, nk, lds.k);
  BlockCopy<D, KV, false> vc(kv, nk, lds.v);
  kc.item(sp, slots);
  vc.item(sp, slots);
  constexpr int kInstr = BlockCopy<D, KV, true>::kInstr;
  if (src.count > 1) src.fetch(1);
#pragma unroll
  for (int i = 0; i < kMtRing; ++i) {
    kc.ready(sp, 0);
    kc.next();
    kc.all(i);
    if (i < kMtRing - 2) {
      vc.ready(sp, 0);
      vc.next();
      vc.all(i);
    }
  }
  for (int i = threadIdx.x; i < Lay::kElems / 8; i += 64 * kMtWaves)
    *reinterpret_cast<u32x4*>(lds.zero + 8 * i) = u32x4{0, 0, 0, 0};
  // (the first product waits for Q, and with it for the copies before it)
  mt_place_q<D>(st, io);
  if (src.count > 1) {
    sp_next = src.settle(1);
    rows_next = src.rows;
    slots_next = mt_slots(sp_next.blocks(), src.count > 2);
    if (src.count > 2) src.fetch(2);
  }
  kc.ready(sp_next, slots_next);
  vc.ready(sp_next, slots_next);
  __builtin_amdgcn_s_waitcnt(0x0070);            // the copies and the zeros
  pf_barrier();
  kc.next();
  vc.next();

  uint32_t odd_items = 0;
  // Places r, r + 1 and r + 2, r + 3 (mod 4) of the rings, in elements: slot i of
  // an even i has K(i) and V(i) in the first.
  constexpr int kE = Lay::kElems;
  int ra = 0, rb = 2 * kE;
  f32x16 sE, sO = {};
  bf16x8 pE[2] = {}, pO[2];
#pragma unroll 1
  for (int m = 0;; ++m) {
    const int n = sp.blocks();
    const FullBlocks fb = rows.full_blocks(sp);
    int run = min(fb.run(0), n);                 // blocks from the slot's on that are full
    uint32_t odd = 0;
    bool partial = false;                        // the block before was not full, and was there
    pf_reset(st);
    pO[0] = pO[1] = bf16x8{};                    // (the last item's may be NaN, and times 0 stay so)
    sE = pf_qk<D, 0>(st, lay, lds.k + ra);
    if (run == 0) mt_mask(sE, n == 0 ? 0u : rows.seen(sp.key0(0)));
    float tmax = sE[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) tmax = fmaxf(tmax, sE[j]);
    st.m_used = max_halves(tmax);
    // (K(0) is read by all waves before the first slot requests K(4) into its place)
    __builtin_amdgcn_s_waitcnt(0xC07F);
    pf_barrier();
    const bool more = m + 1 < src.count;
    // Block i with scores s_cur; the next block's K, the last one's V.
    auto slot = [&](int i, f32x16& s_cur, f32x16& s_next, bf16x8 (&p_cur)[2],
                    const bf16x8 (&p_prev)[2], const bf16_t* kst, const bf16_t* vst,
                    const auto& hook) {
      if (partial) odd |= mt_look<D>(vst);
      partial = false;
      if (run > 0) {
        --run;
      } else {
        asm volatile("");
        partial = i < n;
        mt_mask(s_cur, partial ? rows.seen(sp.key0(i)) : 0u);
        run = max(min(fb.run(i + 1), n - i - 1), 0);
      }
      float sum = pf_full_slot<D, 0, 0>(st, lay, kst, vst, s_cur, s_next, p_cur, p_prev, c,
                                        -st.m_used * c, hook);
      if (__builtin_expect(wave_any(!(sum <= kPfSumBound)), 0)) sum = pf_reref(st, s_cur, c, p_cur);
      st.l += sum;
    };
    // V(i + 2) and K(i + 4), spread over slot i.
    auto copies = [&](auto plus, uint32_t kplace, uint32_t vplace) {
      return [&kc, &vc, kplace, vplace](int step) {
        constexpr int kPlus = decltype(plus)::value, kStep = D / 16 / (2 * kInstr);
        if (step % kStep == 0) {
          const int x = step / kStep;
          if (x < kInstr)
            vc.template copy<kPlus>(vplace, x);
          else
            kc.template copy<kPlus>(kplace, x - kInstr);
        }
      };
    };
    // Slot i + 1 needs K(i + 2) and V(i), requested in slot i - 2 at the latest.
    auto turn = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      kc.ready(sp_next, slots_next);
      vc.ready(sp_next, slots_next);
      __builtin_amdgcn_s_waitcnt(0x0F70 | 4 * kInstr);   // the copies of two slots
      pf_barrier();
      kc.next();
      vc.next();
    };
    constexpr int kBytes = kE * sizeof(bf16_t);
#pragma unroll 1
    for (int i = 0; i < slots; i += 2) {
      if (i > 0) turn();
      slot(i, sE, sO, pE, pO, lds.k + ra + kE, i == 0 || i > n ? lds.zero : lds.v + rb + kE,
           copies(MtInt<0>{}, ra * sizeof(bf16_t), rb * sizeof(bf16_t)));
      turn();
      slot(i + 1, sO, sE, pO, pE, lds.k + rb, i + 1 > n ? lds.zero : lds.v + ra,
           copies(MtInt<kBytes>{}, ra * sizeof(bf16_t), rb * sizeof(bf16_t)));
      const int x = ra;
      ra = rb;
      rb = x;
    }
    // The copies are in the next item by now (an item has four slots), and may go on
    // to the one behind it.
    const KeySpans sp1 = sp_next;
    const auto rows1 = rows_next;
    const int slots1 = slots_next;
    slots_next = 0;
    if (m + 2 < src.count) {
      sp_next = src.settle(m + 2);
      rows_next = src.rows;
      slots_next = mt_slots(sp_next.blocks(), m + 3 < src.count);
      if (m + 3 < src.count) src.fetch(m + 3);
    }
    turn();
    if (n == slots && n > 0) {                   // (else the last block's was in a slot)
      if (partial) odd |= mt_look<D>(lds.v + rb + kE);
      pf_pv<D, 0>(st, lay, lds.v + rb + kE, pO);
    }
    if (wave_any(odd != 0)) odd_items |= 1u << m;
    if (more) mt_request_q<D>(st, [&](int r) { return src.q(m + 1, r); });
    src.store(m, st, mt_finish<D>(st), scale, io);
    if (!more) break;
    mt_place_q<D>(st, io);
    sp = sp1;
    rows = rows1;
    slots = slots1;
  }
  // (no copy into LDS outlives the workgroup, or meets its next use of the rings)
  __builtin_amdgcn_s_waitcnt(0x0F70);
  return odd_items;
}

// masked_items_fast, and the items again that need it (of any wave).
template <int D, class Src, class KV>
__device__ __forceinline__ void masked_items(Src& src, const KV& kv, int nk, float scale,
                                             MtLds<D>& lds) {
  uint32_t odd = masked_items_fast<D>(src, kv, nk, scale, lds);
  uint32_t* const all = reinterpret_cast<uint32_t*>(lds.zero);   // (nobody reads zeros any more)
  __syncthreads();
  if (threadIdx.x < kMtWaves) all[threadIdx.x] = 0;
  __syncthreads();
  if (odd != 0) all[wave_id()] = odd;
  __syncthreads();
  odd = 0;
#pragma unroll
  for (int w = 0; w < kMtWaves; ++w) odd |= all[w];
  odd = __builtin_amdgcn_readfirstlane(odd);
  if (__builtin_expect(odd == 0, 1)) return;
  asm volatile("");
  bf16_t* const io = lds.io[wave_id()];
#pragma unroll 1
  for (int m = 0; m < src.count; ++m) {
    if (!(odd >> m & 1)) continue;
    PfState<D> st;
    src.fetch(m);
    mt_request_q<D>(st, [&](int r) { return src.q(m, r); });
    const KeySpans sp = src.settle(m);
    mt_place_q<D>(st, io);
    masked_item_odd<D>(src.rows, kv, sp, nk, scale, lds.k, lds.v, st);
    src.store(m, st, mt_finish<D>(st), scale, io);
  }
}

}  // namespace rag
