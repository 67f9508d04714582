// Host-side launch descriptors of the page tables, the drafted-token and the
// key-range kernels (internal; the public ABI is include/rag_attn.h).
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

namespace rag {

struct PagesArgs {
  int32_t* tables;              // [num_seqs, max_blocks]
  int32_t* stack;               // [num_blocks], num_free of them used
  const int32_t* num_free;
  const int32_t* old_lens;      // [num_seqs]
  const int32_t* new_lens;
  int32_t* num_free_out;
  int32_t* lens_out;
  int32_t* cu_new;              // [num_seqs + 1]
  int32_t* slots;               // [max_new_tokens]
  int32_t* num_granted;
  int num_seqs, max_blocks, num_blocks, max_new_tokens;
};

struct KeepArgs {
  void* k_cache;                // [num_blocks, hkv, 16, d]
  void* v_cache;
  const int32_t* tables;
  const int32_t* base_lens;     // [num_seqs]
  const int32_t* kept;          // [num_seqs, max_kept]
  const int32_t* num_kept;      // [num_seqs]
  int num_seqs, max_blocks, max_kept, hkv, d;
};

struct TreeArgs {
  const void* q;                // [Tq, hq, d]
  const void* k_cache;
  const void* v_cache;
  void* o;
  const uint64_t* mask;         // [Tq, mask_words]
  const int32_t* tables;
  const int32_t* kv_lens;
  const int32_t* cu_q;
  int num_seqs, max_nodes, mask_words, max_blocks, hq, hkv, d;
  float scale;
  int row_blocks = 1;           // blocks of 128 (node, q head of a group) rows, at most
  int splits = 1;               // pieces of every sequence (0: cut from the lengths)
  int units = 0;                // for one kv head and row block
  int part_rows = 0;            // rows of a row block in the partials
  // a launch that may cut: partial outputs [place][kv head][row block][part_rows][d], their
  // log-sum-exps, and what places a sequence's pieces have and their number (else null)
  float* part_o = nullptr;
  float* part_lse = nullptr;
  int32_t* part_of = nullptr;
};

// How a tree launch is cut (requested splits 0: chosen).
struct TreeShape {
  int row_blocks, splits, part_rows;
  int64_t units, places;
};

struct RangesArgs {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  const int32_t* cu_q;
  const int32_t* cu_k;
  const int32_t* ranges;        // [Tq, 2]
  int num_seqs, max_seqlen_q, hq, hkv, d;
  float scale;
};

constexpr int kPagesMaxSeqs = 4096;        // rows of one rag_kv_pages_update call (LDS)
constexpr int kTreeMaxSplits = 64;
constexpr int kTreePlanSeqs = 256;         // sequences whose pieces are cut from their lengths

int64_t pages_grid(const PagesArgs& a);
hipError_t launch_pages(const PagesArgs& a, hipStream_t stream);
int64_t keep_grid(const KeepArgs& a);
hipError_t launch_keep(const KeepArgs& a, hipStream_t stream);
TreeShape tree_shape(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks,
                     int requested);
size_t tree_partial_rows(const TreeShape& t, int hkv);
size_t tree_partial_rows_upto(int num_seqs, int max_nodes, int hq, int hkv, int d, int max_blocks,
                              int requested);
int64_t tree_grid(const TreeShape& t, const TreeArgs& a);
hipError_t launch_tree(const TreeArgs& a, hipStream_t stream);
int64_t ranges_grid(const RangesArgs& a);       // workgroups, at most
hipError_t launch_ranges(const RangesArgs& a, hipStream_t stream);

}  // namespace rag
