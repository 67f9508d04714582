// Host-side launch descriptors of the new tokens' norm, rotation and cache
// writes, the 4-bit paged cache and the verification of drafted tokens
// (internal; the public ABI is include/rag_attn.h).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <stddef.h>
#include <stdint.h>

namespace rag {

struct RopeArgs {
  const void* q;                // [num_tokens, hq, d], q_stride elements a token; null: none
  const void* k;                // [num_tokens, hkv, d]
  const void* v;
  int64_t q_stride, k_stride, v_stride;
  void* q_out;                  // [num_tokens, hq, d]
  void* k_out;                  // [num_tokens, hkv, d] or null
  void* v_out;
  void* k_cache;                // bf16 [num_blocks, hkv, 16, d], or 4-bit pages; null: none
  void* v_cache;
  const int32_t* slots;         // null: no cache
  const int32_t* positions;     // null: no rotation
  const float* cos_sin;         // [max_position, rot]
  const void* q_weight;         // [d] or null
  const void* k_weight;
  float eps;
  int num_tokens, hq, hkv, d, max_position, rot, interleaved;
};

struct Kv4ReadArgs {
  const void* k_cache;
  const void* v_cache;
  const int32_t* tables;
  const int32_t* cu_k;
  void* k;                      // [num_rows, hkv, d]
  void* v;
  int num_rows, num_seqs, max_blocks, hkv, d;
};

struct Kv4Args {
  const void* q;                // [Tq, hq, d]
  const void* k_cache;
  const void* v_cache;
  void* o;
  const int32_t* tables;
  const int32_t* kv_lens;
  const int32_t* cu_q;          // null: one row a sequence
  int num_seqs, max_rows, max_blocks, hq, hkv, d;
  float scale;
  int cols = 0, tiles = 1;      // pairs of a tile, row tiles of a sequence and kv head, at most
  int units = 0;                // workgroups of a kv head that share all keys; 0: nothing is cut
  float* part_o = nullptr;      // [2 units][hkv][cols][d]
  float* part_lse = nullptr;    // [2 units][hkv][cols]
  int* arrivals = nullptr;      // [units][hkv]
};

struct VerifyArgs {
  const void* logits;           // [num_rows, vocab], bf16 or fp32
  const float* draft;           // [num_rows, vocab] or null
  int64_t logits_stride, draft_stride;
  const int32_t* tokens;        // [num_rows]
  const int32_t* parents;       // [num_rows] or null
  const int32_t* cu;            // [num_seqs + 1]
  const float* temperature;     // [num_seqs]
  const float* uniforms;        // [num_rows]
  int32_t* kept;                // [num_seqs, max_kept]
  int32_t* num_kept;
  int32_t* next_token;
  int num_rows, num_seqs, vocab, max_kept, wide;
  char* ws = nullptr;
};

// Row tiles of an attention launch over the 4-bit cache, and how it is cut.
struct Kv4Shape {
  int cols, tiles, units;       // (row, q head) pairs of a tile; tiles; units (see Kv4Args)
};

constexpr int kKv4PlanSeqs = 1024;         // sequences that are cut from their lengths
constexpr int kKv4Counters = 4096;         // arrival counters of a call, at most
constexpr int kVerifyMaxRows = 1 << 20;
constexpr int kVerifyMaxSeqs = 16384;      // (two counters each)
constexpr int kVerifyMaxVocab = 1 << 28;

int64_t rope_grid(const RopeArgs& a);
hipError_t launch_rope(const RopeArgs& a, bool kv4, hipStream_t stream);
int64_t kv4_read_grid(const Kv4ReadArgs& a);
hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream);
Kv4Shape kv4_shape(int num_seqs, int max_rows, int hq, int hkv, int max_blocks);
int64_t kv4_grid(const Kv4Shape& t, int num_seqs, int hkv);
hipError_t launch_kv4(const Kv4Args& a, const Kv4Shape& t, hipStream_t stream);
size_t verify_workspace(int num_rows, int num_seqs, int vocab);
int64_t verify_grid(const VerifyArgs& a);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream);

}  // namespace rag
