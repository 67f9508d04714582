// C ABI of the new tokens' norm, rotation and cache writes, the 4-bit paged cache
// and the verification of drafted tokens (declared in include/rag_attn.h): argument
// validation, workspace sizing, optional device-array checks.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <vector>

#include "checks.h"
#include "errors.h"
#include "rag_attn.h"
#include "serve.h"

namespace {

using rag::aligned16;
using rag::check_mode;
using rag::fail;
using rag::fetch;
using rag::kBlock;
using rag::ok;

// Page ids fit in int32 slots (page * 16 + offset), table widths in int32 keys.
constexpr int32_t kMaxPages = 1 << 27;
// Pages of a sequence that is attended: keys behind its last block, and the places where all
// sequences' shares start (512 of up to 1/62 of the longest, four a block), fit in int32 too.
constexpr int32_t kMaxAttended = 1 << 26;
// Workgroups of a launch, of 256 threads at most: it takes less than 2^32 threads.
constexpr int64_t kMaxGroups = (1 << 24) - 1;

rag_status check_shape(const char* who, int32_t hq, int32_t hkv, int32_t d) {
  if (hkv <= 0 || hq < 0)
    return fail(RAG_ERR_INVALID_ARG, "%s: %d q heads, %d kv heads", who, hq, hkv);
  if (d != 64 && d != 128)
    return fail(RAG_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", who, d);
  if (hq > 1 << 16 || hkv > 1 << 16)
    return fail(RAG_ERR_UNSUPPORTED, "%s: more than 65536 heads", who);
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

int32_t pages_of(int32_t keys) { return (int32_t)(((int64_t)keys + kBlock - 1) / kBlock); }

// Debug mode: the first `pages` entries of table row s are pages of the pool.
rag_status check_table(const char* who, const std::vector<int32_t>& bt, int32_t s,
                       int32_t max_blocks, int32_t pages, int32_t num_blocks) {
  for (int32_t b = 0; b < pages; ++b) {
    const int32_t id = bt[(size_t)s * max_blocks + b];
    if (id < 0 || id >= num_blocks)
      return fail(RAG_ERR_INVALID_ARG, "%s: block_tables[%d][%d] = %d outside [0, %d)", who, s, b,
                  id, num_blocks);
  }
  return RAG_OK;
}

// Memory that a call reads or writes.
struct Span {
  const char* name;
  const void* at;
  size_t bytes;
};

rag_status check_apart(const char* who, const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  if (a.at != nullptr && b.at != nullptr && a.bytes > 0 && b.bytes > 0 &&
      (x >= y ? x - y < b.bytes : y - x < a.bytes))
    return fail(RAG_ERR_INVALID_ARG, "%s: %s and %s overlap", who, a.name, b.name);
  return RAG_OK;
}

rag_status check_tokens(const char* who, const rag::RopeArgs& a, int32_t num_blocks,
                        hipStream_t stream) {
  std::vector<int32_t> sl, po;
  if ((a.slots && !fetch(sl, a.slots, (size_t)a.num_tokens, stream)) ||
      (a.positions && !fetch(po, a.positions, (size_t)a.num_tokens, stream)))
    return fail(RAG_ERR_HIP, "%s: debug copy of device arrays failed", who);
  std::vector<char> seen;
  if (a.slots && !rag::room(seen, (size_t)num_blocks * kBlock))
    return fail(RAG_ERR_HIP, "%s: no host memory for the debug check", who);
  for (int32_t t = 0; t < a.num_tokens; ++t) {
    if (a.slots) {
      const int32_t s = sl[(size_t)t];
      if (s < 0) continue;
      if ((int64_t)s >= (int64_t)num_blocks * kBlock || seen[(size_t)s]++)
        return fail(RAG_ERR_INVALID_ARG, "%s: slot_mapping[%d] = %d is outside the pool, or twice "
                                         "there", who, t, s);
    }
    if (a.positions && (po[(size_t)t] < 0 || po[(size_t)t] >= a.max_position))
      return fail(RAG_ERR_INVALID_ARG, "%s: positions[%d] = %d outside [0, %d)", who, t,
                  po[(size_t)t], a.max_position);
  }
  return RAG_OK;
}

rag_status rope(const char* who, rag::RopeArgs a, bool kv4, int32_t block_size, int32_t num_blocks,
                hipStream_t stream) {
  if (a.num_tokens < 0) return fail(RAG_ERR_INVALID_ARG, "%s: negative size", who);
  rag_status st = check_shape(who, a.hq, a.hkv, a.d);
  if (st != RAG_OK) return st;
  const bool cached = a.slots != nullptr;
  if (cached || kv4) {
    st = check_paging(who, block_size, 0, num_blocks);
    if (st != RAG_OK) return st;
  }
  if (a.num_tokens == 0) return ok();
  if ((a.q == nullptr) != (a.q_out == nullptr) || (a.q != nullptr && a.hq == 0))
    return fail(RAG_ERR_INVALID_ARG, "%s: q, q_out and num_q_heads go together", who);
  if (a.q == nullptr && a.q_weight != nullptr)
    return fail(RAG_ERR_INVALID_ARG, "%s: q_weight without q", who);
  if (cached != (a.k_cache != nullptr) || cached != (a.v_cache != nullptr))
    return fail(RAG_ERR_INVALID_ARG, "%s: slot_mapping, k_cache and v_cache go together", who);
  if ((a.k_out == nullptr) != (a.v_out == nullptr))
    return fail(RAG_ERR_INVALID_ARG, "%s: k_out and v_out go together", who);
  if ((a.positions == nullptr) != (a.cos_sin == nullptr))
    return fail(RAG_ERR_INVALID_ARG, "%s: positions and cos_sin go together", who);
  if (a.positions != nullptr) {
    if (a.max_position <= 0 || a.rot <= 0 || a.rot > a.d)
      return fail(RAG_ERR_INVALID_ARG, "%s: cos_sin [%d, %d] for heads of %d", who, a.max_position,
                  a.rot, a.d);
    if (a.rot % 16 != 0)
      return fail(RAG_ERR_UNSUPPORTED, "%s: rotary_dim %d (a multiple of 16)", who, a.rot);
    if (a.interleaved != 0 && a.interleaved != 1)
      return fail(RAG_ERR_INVALID_ARG, "%s: interleaved %d (0 or 1)", who, a.interleaved);
  }
  if ((a.q_weight != nullptr || a.k_weight != nullptr) && !(a.eps >= 0.f && a.eps < INFINITY))
    return fail(RAG_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
  if (!a.k || !a.v) return fail(RAG_ERR_INVALID_ARG, "%s: null k or v", who);
  if (!cached && a.k_out == nullptr)
    return fail(RAG_ERR_INVALID_ARG, "%s: neither a cache nor k_out and v_out", who);
  for (const void* p : {a.q, a.k, a.v, (const void*)a.q_out, (const void*)a.k_out,
                        (const void*)a.v_out, (const void*)a.k_cache, (const void*)a.v_cache,
                        (const void*)a.cos_sin, a.q_weight, a.k_weight})
    if (!aligned16(p)) return fail(RAG_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  const int64_t wq = (int64_t)a.hq * a.d, wk = (int64_t)a.hkv * a.d;
  if (a.num_tokens == 1) {                 // (there is no second token)
    a.q_stride = wq;
    a.k_stride = a.v_stride = wk;
  }
  auto bad = [](int64_t stride, int64_t width) {
    return stride < width || stride % 8 != 0 || stride > (int64_t)1 << 40;
  };
  if ((a.q && bad(a.q_stride, wq)) || bad(a.k_stride, wk) || bad(a.v_stride, wk))
    return fail(RAG_ERR_INVALID_ARG, "%s: token strides %lld, %lld, %lld (multiples of 8, at least "
                                     "the heads)", who, (long long)a.q_stride,
                (long long)a.k_stride, (long long)a.v_stride);
  // (a row is written by the lanes that have read it, so that an output may be its own input)
  const size_t last = (size_t)a.num_tokens - 1;
  const size_t pool = (size_t)num_blocks * a.hkv * (kv4 ? 9 * a.d : kBlock * a.d * 2);
  const size_t weight = (size_t)a.d * 2;
  const Span in[] = {{"q", a.q, 2 * (last * a.q_stride + wq)},
                     {"k", a.k, 2 * (last * a.k_stride + wk)},
                     {"v", a.v, 2 * (last * a.v_stride + wk)},
                     {"slot_mapping", a.slots, (last + 1) * 4},
                     {"positions", a.positions, (last + 1) * 4},
                     {"cos_sin", a.cos_sin, a.cos_sin ? (size_t)a.max_position * a.rot * 4 : 0},
                     {"q_weight", a.q_weight, weight},
                     {"k_weight", a.k_weight, weight}};
  const Span out[] = {{"q_out", a.q_out, 2 * (last + 1) * wq},
                      {"k_out", a.k_out, 2 * (last + 1) * wk},
                      {"v_out", a.v_out, 2 * (last + 1) * wk},
                      {"k_cache", a.k_cache, pool},
                      {"v_cache", a.v_cache, pool}};
  for (int i = 0; i < 5; ++i) {
    for (int j = i + 1; j < 5; ++j)
      if ((st = check_apart(who, out[i], out[j])) != RAG_OK) return st;
    for (int j = 0; j < 8; ++j)
      if (!(i == j && out[i].at == in[j].at && out[i].bytes == in[j].bytes) &&
          (st = check_apart(who, out[i], in[j])) != RAG_OK)
        return st;
  }
  if (check_mode() && (st = check_tokens(who, a, num_blocks, stream)) != RAG_OK) return st;
  if (rag::rope_grid(a) > kMaxGroups) return fail(RAG_ERR_UNSUPPORTED, "%s: too many tokens", who);
  if (rag::launch_rope(a, kv4, stream) != hipSuccess)
    return fail(RAG_ERR_HIP, "%s: kernel launch failed", who);
  return ok();
}

// Workspace of an attention launch over the 4-bit cache: arrival counters (as many for
// every call), fp32 log-sum-exps, fp32 partial outputs.
struct Kv4Ws {
  size_t lse_off, o_off, bytes;
};

Kv4Ws kv4_workspace(const rag::Kv4Shape& t, int32_t hkv, int32_t d) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t rows = (size_t)2 * t.units * hkv * t.cols;
  Kv4Ws w;
  w.lse_off = rag::kKv4Counters * sizeof(int);
  w.o_off = w.lse_off + up(rows * sizeof(float));
  w.bytes = rows == 0 ? 0 : w.o_off + up(rows * d * sizeof(float));
  return w;
}

rag_status check_kv4(const rag::Kv4Args& a, int32_t num_blocks, hipStream_t stream) {
  std::vector<int32_t> bt, kl, cq;
  if (!fetch(kl, a.kv_lens, (size_t)a.num_seqs, stream) ||
      (a.cu_q && !fetch(cq, a.cu_q, (size_t)a.num_seqs + 1, stream)) ||
      !fetch(bt, a.tables, (size_t)a.num_seqs * a.max_blocks, stream))
    return fail(RAG_ERR_HIP, "decode kv4: debug copy of device arrays failed");
  if (a.cu_q) {
    const rag_status st = rag::check_cu(cq, "cu_seqlens_q", a.max_rows);
    if (st != RAG_OK) return st;
  }
  for (int32_t s = 0; s < a.num_seqs; ++s) {
    const int32_t n = kl[(size_t)s], rows = a.cu_q ? cq[(size_t)s + 1] - cq[(size_t)s] : 1;
    if (rows == 0) continue;
    if (n < (a.cu_q ? rows : 0) || (int64_t)n > (int64_t)a.max_blocks * kBlock)
      return fail(RAG_ERR_INVALID_ARG, "decode kv4: kv_lens[%d] = %d with %d query rows and a table "
                                       "of %d pages", s, n, rows, a.max_blocks);
    const rag_status st = check_table("decode kv4", bt, s, a.max_blocks, pages_of(n), num_blocks);
    if (st != RAG_OK) return st;
  }
  return RAG_OK;
}

rag_status check_read(const rag::Kv4ReadArgs& a, int32_t num_blocks, hipStream_t stream) {
  std::vector<int32_t> bt, cu;
  if (!fetch(cu, a.cu_k, (size_t)a.num_seqs + 1, stream) ||
      !fetch(bt, a.tables, (size_t)a.num_seqs * a.max_blocks, stream))
    return fail(RAG_ERR_HIP, "kv4 read: debug copy of device arrays failed");
  rag_status st = rag::check_cu(cu, "cu_seqlens_k",
                                (int32_t)std::min<int64_t>((int64_t)a.max_blocks * kBlock, INT_MAX));
  if (st != RAG_OK) return st;
  if (cu[(size_t)a.num_seqs] > a.num_rows)
    return fail(RAG_ERR_INVALID_ARG, "kv4 read: cu_seqlens_k ends at %d of %d rows",
                cu[(size_t)a.num_seqs], a.num_rows);
  for (int32_t s = 0; s < a.num_seqs; ++s) {
    st = check_table("kv4 read", bt, s, a.max_blocks, pages_of(cu[(size_t)s + 1] - cu[(size_t)s]),
                     num_blocks);
    if (st != RAG_OK) return st;
  }
  return RAG_OK;
}

rag_status check_verify(const rag::VerifyArgs& a, hipStream_t stream) {
  std::vector<int32_t> cu, to, pa;
  if (!fetch(cu, a.cu, (size_t)a.num_seqs + 1, stream) ||
      !fetch(to, a.tokens, (size_t)a.num_rows, stream) ||
      (a.parents && !fetch(pa, a.parents, (size_t)a.num_rows, stream)))
    return fail(RAG_ERR_HIP, "draft verify: debug copy of device arrays failed");
  const rag_status st = rag::check_cu(cu, "cu_seqlens_q", a.num_rows);
  if (st != RAG_OK) return st;
  if (cu[(size_t)a.num_seqs] > a.num_rows)
    return fail(RAG_ERR_INVALID_ARG, "draft verify: cu_seqlens_q ends at %d of %d rows",
                cu[(size_t)a.num_seqs], a.num_rows);
  for (int32_t s = 0; s < a.num_seqs; ++s)
    for (int32_t i = 1; i < cu[(size_t)s + 1] - cu[(size_t)s]; ++i) {
      const size_t row = (size_t)cu[(size_t)s] + i;
      if (to[row] < 0 || to[row] >= a.vocab)
        return fail(RAG_ERR_INVALID_ARG, "draft verify: tokens[%zu] = %d outside [0, %d)", row,
                    to[row], a.vocab);
      if (a.parents && (pa[row] < 0 || pa[row] >= i))
        return fail(RAG_ERR_INVALID_ARG, "draft verify: parents[%zu] = %d of node %d", row, pa[row],
                    i);
    }
  return RAG_OK;
}

}  // namespace

extern "C" {

rag_status rag_qkv_rope_write(const void* q, const void* k, const void* v, int64_t q_stride,
                              int64_t k_stride, int64_t v_stride, void* q_out, void* k_out,
                              void* v_out, void* k_cache, void* v_cache,
                              const int32_t* slot_mapping, const int32_t* positions,
                              const float* cos_sin, int32_t max_position, int32_t rotary_dim,
                              int32_t interleaved, const void* q_weight, const void* k_weight,
                              float eps, int32_t num_tokens, int32_t num_q_heads,
                              int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                              int32_t num_blocks, hipStream_t stream) {
  return rope("qkv rope write",
              {q, k, v, q_stride, k_stride, v_stride, q_out, k_out, v_out, k_cache, v_cache,
               slot_mapping, positions, cos_sin, q_weight, k_weight, eps, num_tokens, num_q_heads,
               num_kv_heads, head_dim, max_position, rotary_dim, interleaved},
              false, block_size, num_blocks, stream);
}

rag_status rag_qkv_rope_write_kv4(const void* q, const void* k, const void* v, int64_t q_stride,
                                  int64_t k_stride, int64_t v_stride, void* q_out, void* k_out,
                                  void* v_out, void* k_cache, void* v_cache,
                                  const int32_t* slot_mapping, const int32_t* positions,
                                  const float* cos_sin, int32_t max_position, int32_t rotary_dim,
                                  int32_t interleaved, const void* q_weight, const void* k_weight,
                                  float eps, int32_t num_tokens, int32_t num_q_heads,
                                  int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                                  int32_t num_blocks, hipStream_t stream) {
  if (num_tokens > 0 && slot_mapping == nullptr)
    return fail(RAG_ERR_INVALID_ARG, "qkv rope write kv4: null slot_mapping");
  return rope("qkv rope write kv4",
              {q, k, v, q_stride, k_stride, v_stride, q_out, k_out, v_out, k_cache, v_cache,
               slot_mapping, positions, cos_sin, q_weight, k_weight, eps, num_tokens, num_q_heads,
               num_kv_heads, head_dim, max_position, rotary_dim, interleaved},
              true, block_size, num_blocks, stream);
}

rag_status rag_kv4_read(const void* k_cache, const void* v_cache, const int32_t* block_tables,
                        const int32_t* cu_seqlens_k, void* k, void* v, int32_t num_rows,
                        int32_t num_seqs, int32_t max_blocks_per_seq, int32_t num_blocks,
                        int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                        hipStream_t stream) {
  if (num_rows < 0 || num_seqs < 0) return fail(RAG_ERR_INVALID_ARG, "kv4 read: negative size");
  rag_status st = check_shape("kv4 read", 0, num_kv_heads, head_dim);
  if (st == RAG_OK) st = check_paging("kv4 read", block_size, max_blocks_per_seq, num_blocks);
  if (st != RAG_OK) return st;
  if (num_rows == 0 || num_seqs == 0 || max_blocks_per_seq == 0) return ok();
  if (!k_cache || !v_cache || !block_tables || !cu_seqlens_k || !k || !v)
    return fail(RAG_ERR_INVALID_ARG, "kv4 read: null pointer argument");
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k) || !aligned16(v))
    return fail(RAG_ERR_INVALID_ARG, "kv4 read: pointer not 16-byte aligned");
  const rag::Kv4ReadArgs a{k_cache,  v_cache,  block_tables,       cu_seqlens_k, k,       v,
                           num_rows, num_seqs, max_blocks_per_seq, num_kv_heads, head_dim};
  if (rag::kv4_read_grid(a) > kMaxGroups) return fail(RAG_ERR_UNSUPPORTED, "kv4 read: too many rows");
  const size_t rows = (size_t)num_rows * num_kv_heads * head_dim * 2;
  const size_t pool = (size_t)num_blocks * num_kv_heads * 9 * head_dim;
  const Span spans[] = {{"k", k, rows},
                        {"v", v, rows},
                        {"k_cache", k_cache, pool},
                        {"v_cache", v_cache, pool},
                        {"block_tables", block_tables, (size_t)num_seqs * max_blocks_per_seq * 4},
                        {"cu_seqlens_k", cu_seqlens_k, ((size_t)num_seqs + 1) * 4}};
  for (int i = 0; i < 2; ++i)
    for (int j = i + 1; j < 6; ++j)
      if ((st = check_apart("kv4 read", spans[i], spans[j])) != RAG_OK) return st;
  if (check_mode() && (st = check_read(a, num_blocks, stream)) != RAG_OK) return st;
  if (rag::launch_kv4_read(a, stream) != hipSuccess)
    return fail(RAG_ERR_HIP, "kv4 read: kernel launch failed");
  return ok();
}

size_t rag_attn_decode_kv4_workspace_size(int32_t num_seqs, int32_t max_seqlen_q,
                                          int32_t num_q_heads, int32_t num_kv_heads,
                                          int32_t head_dim, int32_t max_blocks_per_seq,
                                          int32_t block_size) {
  if (num_seqs <= 0 || max_seqlen_q <= 0 || num_kv_heads <= 0 || num_q_heads <= 0 ||
      num_q_heads % num_kv_heads != 0 || (head_dim != 64 && head_dim != 128) ||
      max_blocks_per_seq <= 0 || max_blocks_per_seq > kMaxAttended || block_size != kBlock)
    return 0;
  // (of one sequence: the same for all numbers of them, and for all table widths)
  return kv4_workspace(rag::kv4_shape(1, max_seqlen_q, num_q_heads, num_kv_heads, 1), num_kv_heads,
                       head_dim)
      .bytes;
}

rag_status rag_attn_decode_paged_kv4(const void* q, const void* k_cache, const void* v_cache,
                                     void* o, const int32_t* block_tables, const int32_t* kv_lens,
                                     const int32_t* cu_seqlens_q, int32_t num_seqs,
                                     int32_t max_seqlen_q, int32_t max_blocks_per_seq,
                                     int32_t num_blocks, int32_t num_q_heads, int32_t num_kv_heads,
                                     int32_t head_dim, int32_t block_size, float softmax_scale,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (num_seqs < 0 || max_seqlen_q < 0) return fail(RAG_ERR_INVALID_ARG, "decode kv4: negative size");
  if (num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads != 0)
    return fail(RAG_ERR_INVALID_ARG, "decode kv4: num_q_heads %d must be a positive multiple of "
                                     "num_kv_heads %d", num_q_heads, num_kv_heads);
  if (!(softmax_scale > 0.f) || softmax_scale > 1e30f)
    return fail(RAG_ERR_INVALID_ARG, "decode kv4: softmax_scale must be positive and finite");
  rag_status st = check_shape("decode kv4", num_q_heads, num_kv_heads, head_dim);
  if (st == RAG_OK) st = check_paging("decode kv4", block_size, max_blocks_per_seq, num_blocks);
  if (st != RAG_OK) return st;
  if (max_blocks_per_seq > kMaxAttended)
    return fail(RAG_ERR_UNSUPPORTED, "decode kv4: tables of more than %d pages", kMaxAttended);
  if (cu_seqlens_q == nullptr) max_seqlen_q = 1;
  if ((int64_t)max_seqlen_q * num_q_heads >= 1 << 24)
    return fail(RAG_ERR_UNSUPPORTED, "decode kv4: %d rows of %d heads (2^24 of them)", max_seqlen_q,
                num_q_heads);
  if (num_seqs == 0 || max_seqlen_q == 0) return ok();
  if (!q || !o || !kv_lens || (max_blocks_per_seq > 0 && (!k_cache || !v_cache || !block_tables)))
    return fail(RAG_ERR_INVALID_ARG, "decode kv4: null pointer argument");
  if (!aligned16(q) || !aligned16(o) || !aligned16(k_cache) || !aligned16(v_cache))
    return fail(RAG_ERR_INVALID_ARG, "decode kv4: pointer not 16-byte aligned");
  const rag::Kv4Shape t =
      rag::kv4_shape(num_seqs, max_seqlen_q, num_q_heads, num_kv_heads, max_blocks_per_seq);
  rag::Kv4Args a{q,        k_cache,      v_cache,            o,           block_tables,
                 kv_lens,  cu_seqlens_q, num_seqs,           max_seqlen_q, max_blocks_per_seq,
                 num_q_heads, num_kv_heads, head_dim,        softmax_scale};
  a.cols = t.cols;
  a.tiles = t.tiles;
  a.units = t.units;
  if (rag::kv4_grid(t, num_seqs, num_kv_heads) > kMaxGroups)
    return fail(RAG_ERR_UNSUPPORTED, "decode kv4: too many sequences");
  const Kv4Ws ws = kv4_workspace(t, num_kv_heads, head_dim);
  if (ws.bytes > 0) {
    if (!workspace || workspace_bytes < ws.bytes)
      return fail(RAG_ERR_WORKSPACE, "decode kv4: workspace of %zu bytes, %zu needed",
                  workspace ? workspace_bytes : 0, ws.bytes);
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
      return fail(RAG_ERR_INVALID_ARG, "decode kv4: workspace not 256-byte aligned");
    a.arrivals = reinterpret_cast<int*>(workspace);
    a.part_lse = reinterpret_cast<float*>((char*)workspace + ws.lse_off);
    a.part_o = reinterpret_cast<float*>((char*)workspace + ws.o_off);
  }
  // (o may be q: a tile's rows are written when all its pieces have read them.  How many rows there are
  // with cu_seqlens_q the host does not know: one at least.)
  const size_t width = (size_t)num_q_heads * head_dim * 2, seqs = (size_t)num_seqs;
  const size_t rows = (cu_seqlens_q ? 1 : seqs) * width;
  const size_t pool = (size_t)num_blocks * num_kv_heads * 9 * head_dim;
  const Span spans[] = {{"o", o, rows},
                        {"workspace", ws.bytes > 0 ? workspace : nullptr, ws.bytes},
                        {"q", q, rows},
                        {"k_cache", k_cache, pool},
                        {"v_cache", v_cache, pool},
                        {"block_tables", block_tables, seqs * max_blocks_per_seq * 4},
                        {"kv_lens", kv_lens, seqs * 4},
                        {"cu_seqlens_q", cu_seqlens_q, (seqs + 1) * 4}};
  for (int i = 0; i < 2; ++i)
    for (int j = i + 1; j < 8; ++j)
      if (!(i == 0 && j == 2 && o == q) &&
          (st = check_apart("decode kv4", spans[i], spans[j])) != RAG_OK)
        return st;
  if (check_mode() && (st = check_kv4(a, num_blocks, stream)) != RAG_OK) return st;
  if (rag::launch_kv4(a, t, stream) != hipSuccess)
    return fail(RAG_ERR_HIP, "decode kv4: kernel launch failed");
  return ok();
}

size_t rag_draft_verify_workspace_size(int32_t num_rows, int32_t num_seqs, int32_t vocab) {
  if (num_rows < 0 || num_seqs < 0 || vocab <= 0 || num_rows > rag::kVerifyMaxRows ||
      num_seqs > rag::kVerifyMaxSeqs || vocab > rag::kVerifyMaxVocab)
    return 0;
  return rag::verify_workspace(num_rows, num_seqs, vocab);
}

rag_status rag_draft_verify(const void* logits, int32_t logits_fp32, int64_t logits_stride,
                            const float* draft_probs, int64_t draft_stride, const int32_t* tokens,
                            const int32_t* parents, const int32_t* cu_seqlens_q,
                            const float* temperature, const float* uniforms, int32_t* kept,
                            int32_t* num_kept, int32_t* next_token, int32_t num_rows,
                            int32_t num_seqs, int32_t vocab, int32_t max_kept, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) {
  if (num_rows < 0 || num_seqs < 0 || max_kept < 0)
    return fail(RAG_ERR_INVALID_ARG, "draft verify: negative size");
  if (vocab <= 0) return fail(RAG_ERR_INVALID_ARG, "draft verify: vocab %d", vocab);
  if (logits_fp32 != 0 && logits_fp32 != 1)
    return fail(RAG_ERR_INVALID_ARG, "draft verify: logits_fp32 %d (0 or 1)", logits_fp32);
  if (num_rows > rag::kVerifyMaxRows || num_seqs > rag::kVerifyMaxSeqs ||
      vocab > rag::kVerifyMaxVocab)
    return fail(RAG_ERR_UNSUPPORTED, "draft verify: %d rows, %d sequences, %d tokens (at most %d, %d, "
                                     "%d)", num_rows, num_seqs, vocab, rag::kVerifyMaxRows,
                rag::kVerifyMaxSeqs, rag::kVerifyMaxVocab);
  if (draft_probs != nullptr && parents != nullptr)
    return fail(RAG_ERR_UNSUPPORTED, "draft verify: draft_probs with trees (chains only)");
  if (num_seqs == 0) return ok();
  if (!cu_seqlens_q || !num_kept || !next_token || !temperature || (max_kept > 0 && !kept) ||
      (num_rows > 0 && (!logits || !tokens || !uniforms)))
    return fail(RAG_ERR_INVALID_ARG, "draft verify: null pointer argument");
  if (num_rows > 0 && max_kept == 0)
    return fail(RAG_ERR_INVALID_ARG, "draft verify: max_kept 0 (node 0 is always kept)");
  if (!aligned16(logits) || !aligned16(draft_probs))
    return fail(RAG_ERR_INVALID_ARG, "draft verify: pointer not 16-byte aligned");
  if (num_rows == 1) {                     // (there is no second row)
    logits_stride = vocab;
    draft_stride = vocab;
  }
  const int64_t most = (int64_t)1 << 40;
  if (num_rows > 0 && (logits_stride < vocab || logits_stride > most ||
                       (draft_probs && (draft_stride < vocab || draft_stride > most))))
    return fail(RAG_ERR_INVALID_ARG, "draft verify: row strides %lld, %lld below vocab %d",
                (long long)logits_stride, (long long)draft_stride, vocab);
  const size_t need = rag::verify_workspace(num_rows, num_seqs, vocab);
  if (!workspace || workspace_bytes < need)
    return fail(RAG_ERR_WORKSPACE, "draft verify: workspace of %zu bytes, %zu needed",
                workspace ? workspace_bytes : 0, need);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return fail(RAG_ERR_INVALID_ARG, "draft verify: workspace not 256-byte aligned");
  rag::VerifyArgs a{logits, draft_probs, logits_stride, draft_stride, tokens,   parents,  cu_seqlens_q,
                    temperature, uniforms, kept, num_kept, next_token, num_rows, num_seqs, vocab,
                    max_kept, logits_fp32};
  a.ws = static_cast<char*>(workspace);
  const size_t e = logits_fp32 ? 4 : 2, last = num_rows > 0 ? (size_t)num_rows - 1 : 0;
  const size_t rows = (size_t)num_rows, seqs = (size_t)num_seqs;
  const Span spans[] = {{"kept", kept, seqs * max_kept * 4},
                        {"num_kept", num_kept, seqs * 4},
                        {"next_token", next_token, seqs * 4},
                        {"workspace", workspace, need},
                        {"logits", logits, rows ? (last * logits_stride + vocab) * e : 0},
                        {"draft_probs", draft_probs, rows ? (last * draft_stride + vocab) * 4 : 0},
                        {"tokens", tokens, rows * 4},
                        {"parents", parents, rows * 4},
                        {"cu_seqlens_q", cu_seqlens_q, (seqs + 1) * 4},
                        {"temperature", temperature, seqs * 4},
                        {"uniforms", uniforms, rows * 4}};
  rag_status st;
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 11; ++j)
      if ((st = check_apart("draft verify", spans[i], spans[j])) != RAG_OK) return st;
  if (check_mode() && (st = check_verify(a, stream)) != RAG_OK) return st;
  if (rag::verify_grid(a) > kMaxGroups)
    return fail(RAG_ERR_UNSUPPORTED, "draft verify: too many rows of %d tokens", vocab);
  if (rag::launch_verify(a, stream) != hipSuccess)
    return fail(RAG_ERR_HIP, "draft verify: kernel launch failed");
  return ok();
}

}  // extern "C"
