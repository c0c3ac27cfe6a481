// Attention over a cache of several sequences without a rule: its calls.
#include "spd_seqattn.h"

using namespace spd;

extern "C" spd_status spd_prompt_attention_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                     int32_t rows, int32_t max_len, size_t* bytes) {
  const char* call = "prompt attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (!bytes || rows < 0) return invalid(call, "NULL pointer or negative rows");
  const Request q = request(*c, n_q_heads, nseqs, rows, 0, max_len, false);
  if (q.items * c->n_kv_heads > kMaxWGs) return invalid(call, "more rows than one launch takes (2^24 tiles of 128 queries, with all KV heads)");
  *bytes = q.bytes;
  return SPD_OK;
}

extern "C" spd_status spd_prompt_attention(const spd_cache* c, int32_t layer, const void* q, int64_t q_stride, void* out,
                                           int64_t out_stride, int32_t n_q_heads, int32_t dtype, const int32_t* seqs,
                                           const int32_t* cu_rows, int32_t nseqs, int32_t rows, int32_t max_len,
                                           void* workspace, size_t ws_bytes, void* stream) {
  const char* call = "prompt attention";
  spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st == SPD_OK) st = check_call(call, c, layer, q, q_stride, out, out_stride, n_q_heads, dtype, seqs);
  if (st != SPD_OK) return st;
  if (!cu_rows || misaligned(cu_rows, 4)) return invalid(call, "NULL or misaligned pointer");
  if (rows < 0) return invalid(call, "rows must not be negative");
  size_t need = 0;
  if ((st = spd_prompt_attention_workspace(c, n_q_heads, dtype, nseqs, rows, max_len, &need)) != SPD_OK) return st;
  if ((st = check_workspace(call, workspace, ws_bytes, need)) != SPD_OK) return st;
  if (rows == 0) return SPD_OK;
  SeqArgs a = args_of(c, layer, q, q_stride, out, out_stride, n_q_heads, seqs, nseqs);
  a.cu = cu_rows;
  a.rows = rows;
  run_attention<0>(a, dtype, request(*c, n_q_heads, nseqs, rows, 0, max_len, false), false, workspace, (hipStream_t)stream);
  return check_launch(call);
}

extern "C" spd_status spd_prefix_attention_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                     int32_t ngroups, int32_t max_len, size_t* bytes) {
  const char* call = "prefix attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (nseqs > 4096) return invalid(call, "nseqs must be at most 4096");
  if (!bytes || ngroups < 0 || ngroups > nseqs) return invalid(call, "NULL pointer, or ngroups outside [0, nseqs]");
  *bytes = request(*c, n_q_heads, nseqs, nseqs, ngroups, max_len, true).bytes;
  return SPD_OK;
}

extern "C" spd_status spd_prefix_attention(const spd_cache* c, int32_t layer, const void* q, int64_t q_stride, void* out,
                                           int64_t out_stride, int32_t n_q_heads, int32_t dtype, const int32_t* seqs,
                                           int32_t nseqs, const int32_t* cu_groups, const int32_t* prefix_lens,
                                           int32_t ngroups, int32_t max_len, void* workspace, size_t ws_bytes, void* stream) {
  const char* call = "prefix attention";
  size_t need = 0;
  spd_status st = spd_prefix_attention_workspace(c, n_q_heads, dtype, nseqs, ngroups, max_len, &need);
  if (st == SPD_OK) st = check_call(call, c, layer, q, q_stride, out, out_stride, n_q_heads, dtype, seqs);
  if (st != SPD_OK) return st;
  if ((ngroups > 0) != (cu_groups != nullptr) || (ngroups > 0) != (prefix_lens != nullptr))
    return invalid(call, "cu_groups and prefix_lens come with ngroups > 0, or are NULL with 0");
  if (misaligned(cu_groups, 4) || misaligned(prefix_lens, 4)) return invalid(call, "misaligned pointer");
  if ((st = check_workspace(call, workspace, ws_bytes, need)) != SPD_OK) return st;
  SeqArgs a = args_of(c, layer, q, q_stride, out, out_stride, n_q_heads, seqs, nseqs);
  a.cu = cu_groups;
  a.prefix = prefix_lens;
  a.ngroups = ngroups;
  a.rows = nseqs;
  run_attention<0>(a, dtype, request(*c, n_q_heads, nseqs, nseqs, ngroups, max_len, true), true, workspace, (hipStream_t)stream);
  return check_launch(call);
}
