// C ABI of the page tables, the drafted-token operators and the prefill with
// key ranges (declared in include/rag_attn.h): argument validation, workspace
// sizing, optional device-array checks.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <vector>

#include "checks.h"
#include "draft.h"
#include "errors.h"
#include "rag_attn.h"

namespace {

using rag::aligned16;
using rag::check_mode;
using rag::fail;
using rag::fetch;
using rag::kBlock;
using rag::ok;

// Page ids fit in int32 slots (page * 16 + offset), table widths in int32 keys.
constexpr int32_t kMaxPages = 1 << 27;

rag_status check_heads(const char* who, int32_t hq, int32_t hkv, int32_t d, float scale) {
  if (hq <= 0 || hkv <= 0 || hq % hkv != 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: num_q_heads %d must be a positive multiple of "
                                     "num_kv_heads %d", who, hq, hkv);
  if (!(scale > 0.f) || scale > 1e30f)
    return fail(RAG_ERR_INVALID_ARG, "%s: softmax_scale must be positive and finite", who);
  if (d != 64 && d != 128)
    return fail(RAG_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", who, d);
  return RAG_OK;
}

rag_status check_paging(const char* who, int32_t block_size, int32_t max_blocks,
                        int32_t num_blocks) {
  if (max_blocks < 0 || num_blocks < 0) return fail(RAG_ERR_INVALID_ARG, "%s: negative size", who);
  if (block_size != kBlock)
    return fail(RAG_ERR_UNSUPPORTED, "%s: block_size %d (supported: 16)", who, block_size);
  if (max_blocks >= kMaxPages || num_blocks > kMaxPages)
    return fail(RAG_ERR_UNSUPPORTED, "%s: more than %d pages", who, kMaxPages);
  return RAG_OK;
}

// An int32 array of a call.
struct Array {
  const char* name;
  const int32_t* at;
  size_t count;
};

// None of the first `written` arrays overlaps another one.
rag_status check_apart(const char* who, const Array* arrays, int count, int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < count; ++j) {
      const Array &a = arrays[i], &b = arrays[j];
      const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
      if (a.count > 0 && b.count > 0 &&
          (x >= y ? x - y < b.count * sizeof(int32_t) : y - x < a.count * sizeof(int32_t)))
        return fail(RAG_ERR_INVALID_ARG, "%s: %s and %s overlap", who, a.name, b.name);
    }
  return RAG_OK;
}

// Debug mode: the first `pages` entries of table row s are pages of the pool.
rag_status check_table(const char* who, const std::vector<int32_t>& bt, int32_t s,
                       int32_t max_blocks, int32_t first, int32_t pages, int32_t num_blocks) {
  for (int32_t b = first; b < pages; ++b) {
    const int32_t id = bt[(size_t)s * max_blocks + b];
    if (id < 0 || id >= num_blocks)
      return fail(RAG_ERR_INVALID_ARG, "%s: block_tables[%d][%d] = %d outside [0, %d)", who, s, b,
                  id, num_blocks);
  }
  return RAG_OK;
}

int32_t pages_of(int32_t keys) { return (int32_t)(((int64_t)keys + kBlock - 1) / kBlock); }

rag_status check_pages(const rag::PagesArgs& a, hipStream_t stream) {
  std::vector<int32_t> bt, st, nf, ol, nl;
  if (!fetch(nf, a.num_free, 1, stream) || !fetch(ol, a.old_lens, a.num_seqs, stream) ||
      !fetch(nl, a.new_lens, a.num_seqs, stream) || !fetch(st, (const int32_t*)a.stack, a.num_blocks, stream) ||
      !fetch(bt, (const int32_t*)a.tables, (size_t)a.num_seqs * a.max_blocks, stream))
    return fail(RAG_ERR_HIP, "kv pages: debug copy of device arrays failed");
  if (nf[0] < 0 || nf[0] > a.num_blocks)
    return fail(RAG_ERR_INVALID_ARG, "kv pages: num_free %d outside [0, %d]", nf[0], a.num_blocks);
  std::vector<char> seen;
  if (!rag::room(seen, (size_t)a.num_blocks))
    return fail(RAG_ERR_HIP, "kv pages: no host memory for the debug check");
  auto once = [&](int32_t id) { return id >= 0 && id < a.num_blocks && !seen[(size_t)id]++; };
  for (int32_t i = 0; i < nf[0]; ++i)
    if (!once(st[(size_t)i]))
      return fail(RAG_ERR_INVALID_ARG, "kv pages: free_pages[%d] = %d is no page of the pool, or "
                                       "held twice", i, st[(size_t)i]);
  for (int32_t s = 0; s < a.num_seqs; ++s) {
    const int32_t o = ol[(size_t)s];
    if (o < 0 || (int64_t)o > (int64_t)a.max_blocks * kBlock || nl[(size_t)s] < 0)
      return fail(RAG_ERR_INVALID_ARG, "kv pages: row %d holds %d tokens and is to hold %d (table "
                                       "of %d pages)", s, o, nl[(size_t)s], a.max_blocks);
    for (int32_t b = 0; b < pages_of(o); ++b) {
      const int32_t id = bt[(size_t)s * a.max_blocks + b];
      if (!once(id))
        return fail(RAG_ERR_INVALID_ARG, "kv pages: block_tables[%d][%d] = %d is no page of the "
                                         "pool, or held twice", s, b, id);
    }
  }
  return RAG_OK;
}

rag_status check_keep(const rag::KeepArgs& a, int32_t num_blocks, hipStream_t stream) {
  std::vector<int32_t> bt, bl, ke, nk;
  if (!fetch(bl, a.base_lens, a.num_seqs, stream) || !fetch(nk, a.num_kept, a.num_seqs, stream) ||
      !fetch(ke, a.kept, (size_t)a.num_seqs * a.max_kept, stream) ||
      !fetch(bt, a.tables, (size_t)a.num_seqs * a.max_blocks, stream))
    return fail(RAG_ERR_HIP, "kv keep: debug copy of device arrays failed");
  for (int32_t s = 0; s < a.num_seqs; ++s) {
    const int32_t n = nk[(size_t)s], base = bl[(size_t)s];
    if (n < 0 || n > a.max_kept || base < 0)
      return fail(RAG_ERR_INVALID_ARG, "kv keep: row %d keeps %d of at most %d nodes behind %d keys",
                  s, n, a.max_kept, base);
    int32_t last = -1;
    for (int32_t i = 0; i < n; ++i) {
      const int32_t node = ke[(size_t)s * a.max_kept + i];
      if (node <= last || (int64_t)base + node >= (int64_t)a.max_blocks * kBlock)
        return fail(RAG_ERR_INVALID_ARG, "kv keep: kept[%d][%d] = %d (increasing nodes inside the "
                                         "table needed)", s, i, node);
      last = node;
    }
    if (n > 0) {
      const rag_status st = check_table("kv keep", bt, s, a.max_blocks, base / kBlock,
                                        pages_of(base + last + 1), num_blocks);
      if (st != RAG_OK) return st;
    }
  }
  return RAG_OK;
}

rag_status check_tree(const rag::TreeArgs& a, int32_t num_blocks, hipStream_t stream) {
  std::vector<int32_t> bt, kl, cq;
  if (!fetch(kl, a.kv_lens, a.num_seqs, stream) || !fetch(cq, a.cu_q, a.num_seqs + 1, stream) ||
      !fetch(bt, a.tables, (size_t)a.num_seqs * a.max_blocks, stream))
    return fail(RAG_ERR_HIP, "decode tree: debug copy of device arrays failed");
  rag_status st = rag::check_cu(cq, "cu_seqlens_q", a.max_nodes);
  if (st != RAG_OK) return st;
  for (int32_t s = 0; s < a.num_seqs; ++s) {
    const int32_t n = kl[(size_t)s], nodes = cq[(size_t)s + 1] - cq[(size_t)s];
    if (nodes == 0) continue;
    if (n < nodes || (int64_t)n > (int64_t)a.max_blocks * kBlock)
      return fail(RAG_ERR_INVALID_ARG, "decode tree: kv_lens[%d] = %d with %d nodes and a table of "
                                       "%d pages", s, n, nodes, a.max_blocks);
    st = check_table("decode tree", bt, s, a.max_blocks, 0, pages_of(n), num_blocks);
    if (st != RAG_OK) return st;
  }
  return RAG_OK;
}

// (Rows of a sequence are counted in 32 bits, with room for their blocks.)
bool too_many_rows(int32_t nodes, int32_t hq) { return (int64_t)nodes * hq >= 1 << 24; }

// Workspace of a tree launch that may cut: fp32 partial outputs, fp32
// log-sum-exps, int32 pairs per sequence.
struct TreeWs {
  size_t lse_off, of_off, bytes;
};

TreeWs tree_workspace(size_t rows, int32_t num_seqs, int32_t d) {
  if (rows == 0) return {0, 0, 0};
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  TreeWs w;
  w.lse_off = up(rows * d * sizeof(float));
  w.of_off = w.lse_off + up(rows * sizeof(float));
  w.bytes = w.of_off + up((size_t)num_seqs * 2 * sizeof(int32_t));
  return w;
}

}  // namespace

extern "C" {

rag_status rag_kv_pages_update(int32_t* block_tables, int32_t* free_pages, const int32_t* num_free,
                               const int32_t* old_lens, const int32_t* new_lens, int32_t num_seqs,
                               int32_t max_blocks_per_seq, int32_t num_blocks, int32_t block_size,
                               int32_t max_new_tokens, int32_t* num_free_out, int32_t* lens_out,
                               int32_t* cu_new, int32_t* slot_mapping, int32_t* num_granted,
                               hipStream_t stream) {
  if (num_seqs < 0 || max_new_tokens < 0) return fail(RAG_ERR_INVALID_ARG, "kv pages: negative size");
  rag_status st = check_paging("kv pages", block_size, max_blocks_per_seq, num_blocks);
  if (st != RAG_OK) return st;
  if (num_seqs > rag::kPagesMaxSeqs)
    return fail(RAG_ERR_UNSUPPORTED, "kv pages: %d rows (at most %d)", num_seqs, rag::kPagesMaxSeqs);
  if (max_new_tokens >= 1 << 30)
    return fail(RAG_ERR_UNSUPPORTED, "kv pages: max_new_tokens %d (below 2^30)", max_new_tokens);
  if (!num_free || !num_free_out || !cu_new || !num_granted ||
      (num_seqs > 0 && (!old_lens || !new_lens || !lens_out)) ||
      (num_seqs > 0 && max_blocks_per_seq > 0 && !block_tables) || (num_blocks > 0 && !free_pages) ||
      (max_new_tokens > 0 && !slot_mapping))
    return fail(RAG_ERR_INVALID_ARG, "kv pages: null pointer argument");
  // (every workgroup reads the inputs, and no workgroup waits for another)
  const size_t rows = (size_t)num_seqs;
  const Array arrays[] = {{"block_tables", block_tables, rows * (size_t)max_blocks_per_seq},
                          {"free_pages", free_pages, (size_t)num_blocks},
                          {"num_free_out", num_free_out, 1},
                          {"lens_out", lens_out, rows},
                          {"cu_new", cu_new, rows + 1},
                          {"slot_mapping", slot_mapping, (size_t)max_new_tokens},
                          {"num_granted", num_granted, 1},
                          {"num_free", num_free, 1},
                          {"old_lens", old_lens, rows},
                          {"new_lens", new_lens, rows}};
  st = check_apart("kv pages", arrays, 10, 7);
  if (st != RAG_OK) return st;
  const rag::PagesArgs a{block_tables, free_pages, num_free,     old_lens,           new_lens,
                         num_free_out, lens_out,   cu_new,       slot_mapping,       num_granted,
                         num_seqs,     max_blocks_per_seq,       num_blocks,         max_new_tokens};
  if (check_mode()) {
    st = check_pages(a, stream);
    if (st != RAG_OK) return st;
  }
  const hipError_t e = rag::launch_pages(a, stream);
  if (e != hipSuccess) return fail(RAG_ERR_HIP, "kv pages launch: %s", hipGetErrorString(e));
  return ok();
}

rag_status rag_kv_cache_keep(void* k_cache, void* v_cache, const int32_t* block_tables,
                             const int32_t* base_lens, const int32_t* kept, const int32_t* num_kept,
                             int32_t num_seqs, int32_t max_blocks_per_seq, int32_t max_kept,
                             int32_t num_blocks, int32_t num_kv_heads, int32_t head_dim,
                             int32_t block_size, hipStream_t stream) {
  if (num_seqs < 0 || max_kept < 0) return fail(RAG_ERR_INVALID_ARG, "kv keep: negative size");
  if (num_kv_heads <= 0) return fail(RAG_ERR_INVALID_ARG, "kv keep: num_kv_heads must be > 0");
  if (head_dim != 64 && head_dim != 128)
    return fail(RAG_ERR_UNSUPPORTED, "kv keep: head_dim %d (supported: 64, 128)", head_dim);
  rag_status st = check_paging("kv keep", block_size, max_blocks_per_seq, num_blocks);
  if (st != RAG_OK) return st;
  if (num_seqs == 0 || max_kept == 0 || max_blocks_per_seq == 0) return ok();
  if (!k_cache || !v_cache || !block_tables || !base_lens || !kept || !num_kept)
    return fail(RAG_ERR_INVALID_ARG, "kv keep: null pointer argument");
  if (!aligned16(k_cache) || !aligned16(v_cache))
    return fail(RAG_ERR_INVALID_ARG, "kv keep: k_cache/v_cache must be 16-byte aligned");
  const rag::KeepArgs a{k_cache,  v_cache,  block_tables,       base_lens, kept,         num_kept,
                        num_seqs, max_blocks_per_seq, max_kept, num_kv_heads, head_dim};
  if (rag::keep_grid(a) > INT_MAX)
    return fail(RAG_ERR_UNSUPPORTED, "kv keep: batch too large for one grid");
  if (check_mode()) {
    st = check_keep(a, num_blocks, stream);
    if (st != RAG_OK) return st;
  }
  const hipError_t e = rag::launch_keep(a, stream);
  if (e != hipSuccess) return fail(RAG_ERR_HIP, "kv keep launch: %s", hipGetErrorString(e));
  return ok();
}

size_t rag_attn_decode_tree_workspace_size(int32_t num_seqs, int32_t max_nodes, int32_t num_q_heads,
                                           int32_t num_kv_heads, int32_t head_dim,
                                           int32_t max_blocks_per_seq, int32_t block_size,
                                           int32_t num_splits) {
  (void)block_size;
  if (num_seqs <= 0 || max_nodes <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 ||
      num_q_heads % num_kv_heads != 0 || head_dim <= 0 || max_blocks_per_seq <= 0 || num_splits < 0 ||
      too_many_rows(max_nodes, num_q_heads) || max_blocks_per_seq >= kMaxPages)
    return 0;
  const size_t rows = rag::tree_partial_rows_upto(num_seqs, max_nodes, num_q_heads, num_kv_heads,
                                                  head_dim, max_blocks_per_seq, num_splits);
  return tree_workspace(rows, num_splits > 0 ? num_seqs : std::min(num_seqs, rag::kTreePlanSeqs),
                        head_dim).bytes;
}

rag_status rag_attn_decode_paged_tree(const void* q, const void* k_cache, const void* v_cache,
                                      void* o, const uint64_t* tree_mask,
                                      const int32_t* block_tables, const int32_t* kv_lens,
                                      const int32_t* cu_seqlens_q, int32_t num_seqs,
                                      int32_t max_nodes, int32_t mask_words,
                                      int32_t max_blocks_per_seq, int32_t num_blocks,
                                      int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                      int32_t block_size, float softmax_scale, int32_t num_splits,
                                      void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const char* who = "decode tree";
  if (!q || !k_cache || !v_cache || !o || !tree_mask || !block_tables || !kv_lens || !cu_seqlens_q)
    return fail(RAG_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (num_seqs < 0 || max_nodes < 0 || mask_words < 0 || num_splits < 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: negative size", who);
  rag_status st = check_heads(who, num_q_heads, num_kv_heads, head_dim, softmax_scale);
  if (st != RAG_OK) return st;
  st = check_paging(who, block_size, max_blocks_per_seq, num_blocks);
  if (st != RAG_OK) return st;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o))
    return fail(RAG_ERR_INVALID_ARG, "%s: q/k_cache/v_cache/o must be 16-byte aligned", who);
  if ((reinterpret_cast<uintptr_t>(tree_mask) & 7u) != 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: tree_mask must be 8-byte aligned", who);
  if ((int64_t)mask_words * 64 < max_nodes)
    return fail(RAG_ERR_INVALID_ARG, "%s: %d mask words for %d nodes", who, mask_words, max_nodes);
  if (num_seqs == 0 || max_nodes == 0) return ok();
  if (max_blocks_per_seq == 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: max_blocks_per_seq is 0", who);
  if (too_many_rows(max_nodes, num_q_heads))
    return fail(RAG_ERR_UNSUPPORTED, "%s: %d nodes of %d heads", who, max_nodes, num_q_heads);
  rag::TreeArgs a{q, k_cache, v_cache, o, tree_mask, block_tables, kv_lens, cu_seqlens_q, num_seqs,
                  max_nodes, mask_words, max_blocks_per_seq, num_q_heads, num_kv_heads, head_dim,
                  softmax_scale};
  const rag::TreeShape t = rag::tree_shape(num_seqs, max_nodes, num_q_heads, num_kv_heads,
                                           head_dim, max_blocks_per_seq, num_splits);
  if (rag::tree_grid(t, a) > INT_MAX)
    return fail(RAG_ERR_UNSUPPORTED, "%s: batch too large for one grid", who);
  a.row_blocks = t.row_blocks;
  a.splits = t.splits;
  a.units = (int)t.units;
  a.part_rows = t.part_rows;
  // (what this launch uses; the size asked for before may be that of a larger one)
  const TreeWs ws = tree_workspace(rag::tree_partial_rows(t, num_kv_heads), num_seqs, head_dim);
  if (ws.bytes > 0) {
    if (workspace == nullptr || workspace_bytes < ws.bytes)
      return fail(RAG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, ws.bytes,
                  workspace == nullptr ? (size_t)0 : workspace_bytes);
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
      return fail(RAG_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
    a.part_o = static_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.lse_off);
    a.part_of = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + ws.of_off);
  }
  if (check_mode()) {
    st = check_tree(a, num_blocks, stream);
    if (st != RAG_OK) return st;
  }
  const hipError_t e = rag::launch_tree(a, stream);
  if (e != hipSuccess) return fail(RAG_ERR_HIP, "%s launch: %s", who, hipGetErrorString(e));
  return ok();
}

rag_status rag_attn_prefill_varlen_ranges(const void* q, const void* k, const void* v, void* o,
                                          float* lse, const int32_t* cu_seqlens_q,
                                          const int32_t* cu_seqlens_k, const int32_t* key_ranges,
                                          int32_t num_seqs, int32_t max_seqlen_q,
                                          int32_t max_seqlen_k, int32_t num_q_heads,
                                          int32_t num_kv_heads, int32_t head_dim,
                                          float softmax_scale, hipStream_t stream) {
  const char* who = "prefill ranges";
  if (!q || !k || !v || !o || !cu_seqlens_q || !cu_seqlens_k || !key_ranges)
    return fail(RAG_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (num_seqs < 0 || max_seqlen_q < 0 || max_seqlen_k < 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: negative size", who);
  rag_status st = check_heads(who, num_q_heads, num_kv_heads, head_dim, softmax_scale);
  if (st != RAG_OK) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o))
    return fail(RAG_ERR_INVALID_ARG, "%s: q/k/v/o must be 16-byte aligned", who);
  if ((reinterpret_cast<uintptr_t>(key_ranges) & 7u) != 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: key_ranges must be 8-byte aligned", who);
  if (num_seqs == 0 || max_seqlen_q == 0) return ok();
  const rag::RangesArgs a{q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, key_ranges, num_seqs,
                          max_seqlen_q, num_q_heads, num_kv_heads, head_dim, softmax_scale};
  if (rag::ranges_grid(a) > INT_MAX || (int64_t)num_seqs * num_kv_heads > INT_MAX)
    return fail(RAG_ERR_UNSUPPORTED, "%s: batch too large for one grid", who);
  if (check_mode()) {
    std::vector<int32_t> cq, ck;
    if (!fetch(cq, cu_seqlens_q, num_seqs + 1, stream) ||
        !fetch(ck, cu_seqlens_k, num_seqs + 1, stream))
      return fail(RAG_ERR_HIP, "%s: debug copy of cu_seqlens failed", who);
    st = rag::check_cu(cq, "cu_seqlens_q", max_seqlen_q);
    if (st != RAG_OK) return st;
    st = rag::check_cu(ck, "cu_seqlens_k", max_seqlen_k);
    if (st != RAG_OK) return st;
  }
  const hipError_t e = rag::launch_ranges(a, stream);
  if (e != hipSuccess) return fail(RAG_ERR_HIP, "%s launch: %s", who, hipGetErrorString(e));
  return ok();
}

}  // extern "C"
