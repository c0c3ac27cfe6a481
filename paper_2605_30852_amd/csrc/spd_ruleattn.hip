// Attention over a cache of several sequences under a rule (spd_rule.h): its calls. The kernels are spd_seqattn.h's, one for each set of
// a rule's parts: keys alone, a cap, distances, both, and both with a cap too high for one offset.
#include "spd_seqattn.h"

namespace spd {
namespace {

template <int RL>
__device__ __forceinline__ float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }

// tanh to 2^-22 of itself: below kTanhPoly a polynomial of x^2, fitted to the least largest relative error, 1e-9; above it 1 - 2 / (1 +
// e^2x) loses at most a bit.
constexpr float kTanhPoly = 0.55f;
template <int RL>
__device__ __forceinline__ float tanh_of(float x) {
  const float y = x * x;
  float p = -0.00627423963f;
  p = fmaf(y, p, 0.0210716799f);
  p = fmaf(y, p, -0.0538523085f);
  p = fmaf(y, p, 0.13332586f);
  p = fmaf(y, p, -0.333333164f);
  const float small = fmaf(x * y, p, x), t = __builtin_amdgcn_exp2f(fabsf(x) * 2.88539008177792681f);
  const float big = fmaf(-2.0f, reciprocal<RL>(1.0f + t), 1.0f);
  return fabsf(x) < kTanhPoly ? small : copysignf(big, x);
}

// tanh(x) / x in powers of x^2, for x from 0 up to `to`, fitted to the least largest error of tanh(x) relative to itself. Three terms,
// 3.9e-5, and four, 4.0e-5, are enough for probabilities that are rounded to bf16, of caps up to 55: the largest score that they take, 0.72 of
// the cap, is off by 1.6e-3, as p of itself, its rounding by up to 3.9e-3. It does not cancel in the softmax, where tiles of other
// ranges have other formulas: at a cap of 512 equal scores would differ by 1.5e-2, so higher caps of bf16 queries take the exponential
// formula, which is off by 3.4e-4 there. Five terms, 3e-8, and seven, 5e-8, are what fp32 holds.
struct Tanh {
  double to;
  int terms;
  double c[7];
};
constexpr Tanh kTanh3{0.55, 3, {0.999961253, -0.330998277, 0.111880151}}, kTanh4{0.9, 4, {0.999960199, -0.331725224, 0.122781884, -0.0300411835}},
    kTanh5{0.55, 5, {0.999999968, -0.33332795, 0.133188769, -0.0525893176, 0.0163154405}},
    kTanh7{1.0, 7, {0.99999995, -0.333328392, 0.133252041, -0.0534570295, 0.0202899804, -0.00620337906, 0.00104102262}};

// Whether the exponents of scores under a cap lie in a range that one offset serves.
bool one_offset(float cap) { return cap * kLog2e <= kFixedTop; }

// The polynomials with the scale of the products S in their coefficients. Caps for which these would leave fp32's range have none (a
// limit of -1): their scores take the other formula.
void scaled_polys(RuleArgs& r, int dtype, float scale) {
  r.limit = r.near = -1.f;
  if (!(r.cap >= 0x1p-6f && r.cap <= 0x1p9f)) return;
  if (dtype == SPD_BF16 && !one_offset(r.cap)) {
    r.limit = 0.f;
    return;
  }
  const double top = (double)r.cap * kLog2e, k = dtype == SPD_BF16 ? (double)scale / r.cap : 1.0 / top;  // x = S k
  auto take = [&](const Tanh& t, float* c) {
    double power = k * top;
    for (int i = 0; i < t.terms; i++, power *= k * k) c[i] = (float)(t.c[i] * power);
    return (float)(t.to / k);
  };
  r.limit = take(dtype == SPD_BF16 ? kTanh4 : kTanh7, r.c);
  r.near = take(dtype == SPD_BF16 ? kTanh3 : kTanh5, r.n);
}

spd_status check_rule(const char* call, const spd_attention_rule* r) {
  if (!r) return invalid(call, "NULL rule");
  if (r->cap != 0.f && !(r->cap >= 0x1p-20f && r->cap <= 0x1p20f)) return invalid(call, "cap must be 0 or in [2^-20, 2^20]");
  if (r->window < 0) return invalid(call, "window must not be negative");
  if (misaligned(r->slopes, 4) || misaligned(r->first, 4) || misaligned(r->open_lens, 4)) return invalid(call, "misaligned pointer");
  return SPD_OK;
}

// The kernels of a rule's parts.
void run_ruled(const SeqArgs& plain, const spd_attention_rule& r, int dtype, const Request& q, bool prefix, void* workspace,
               hipStream_t s) {
  RuledSeqArgs a{plain, RuleArgs{r.cap, r.window, r.slopes, r.first, r.open_lens, 0.f, {}, 0.f, {}}};
  scaled_polys(a.rule, dtype, plain.scale);
  constexpr int CAP = RULE_KEYS | RULE_CAP;
  if (r.cap == 0.f)
    r.slopes ? run_attention<RULE_KEYS | RULE_SLOPES>(a, dtype, q, prefix, workspace, s)
             : run_attention<RULE_KEYS>(a, dtype, q, prefix, workspace, s);
  else if (!one_offset(r.cap))
    run_attention<CAP | RULE_SLOPES>(a, dtype, q, prefix, workspace, s);
  else
    r.slopes ? run_attention<CAP | RULE_SLOPES | RULE_FIXED>(a, dtype, q, prefix, workspace, s)
             : run_attention<CAP | RULE_FIXED>(a, dtype, q, prefix, workspace, s);
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" spd_status spd_prompt_attention_ruled_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                           int32_t rows, int32_t max_len, size_t* bytes) {
  const char* call = "ruled prompt attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (!bytes || rows < 0) return invalid(call, "NULL pointer or negative rows");
  const Request q = request(*c, n_q_heads, nseqs, rows, 0, max_len, false, true);
  if (q.items * c->n_kv_heads > kMaxWGs) return invalid(call, "more rows than one launch takes (2^24 tiles of 128 queries, with all KV heads)");
  *bytes = q.bytes;
  return SPD_OK;
}

extern "C" spd_status spd_prompt_attention_ruled(const spd_cache* c, int32_t layer, const void* q, int64_t q_stride, void* out,
                                                 int64_t out_stride, int32_t n_q_heads, int32_t dtype, const int32_t* seqs,
                                                 const int32_t* cu_rows, int32_t nseqs, int32_t rows, int32_t max_len,
                                                 const spd_attention_rule* rule, void* workspace, size_t ws_bytes, void* stream) {
  const char* call = "ruled prompt attention";
  spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st == SPD_OK) st = check_call(call, c, layer, q, q_stride, out, out_stride, n_q_heads, dtype, seqs);
  if (st == SPD_OK) st = check_rule(call, rule);
  if (st != SPD_OK) return st;
  if (!cu_rows || misaligned(cu_rows, 4)) return invalid(call, "NULL or misaligned pointer");
  if (rows < 0) return invalid(call, "rows must not be negative");
  size_t need = 0;
  if ((st = spd_prompt_attention_ruled_workspace(c, n_q_heads, dtype, nseqs, rows, max_len, &need)) != SPD_OK) return st;
  if ((st = check_workspace(call, workspace, ws_bytes, need)) != SPD_OK) return st;
  if (rows == 0) return SPD_OK;
  SeqArgs a = args_of(c, layer, q, q_stride, out, out_stride, n_q_heads, seqs, nseqs);
  a.cu = cu_rows;
  a.rows = rows;
  run_ruled(a, *rule, dtype, request(*c, n_q_heads, nseqs, rows, 0, max_len, false, true, rule->window, rule->open_lens != nullptr), false, workspace, (hipStream_t)stream);
  return check_launch(call);
}

extern "C" spd_status spd_prefix_attention_ruled_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                           int32_t ngroups, int32_t max_len, size_t* bytes) {
  const char* call = "ruled prefix attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (nseqs > 4096) return invalid(call, "nseqs must be at most 4096");
  if (!bytes || ngroups < 0 || ngroups > nseqs) return invalid(call, "NULL pointer, or ngroups outside [0, nseqs]");
  *bytes = request(*c, n_q_heads, nseqs, nseqs, ngroups, max_len, true, true).bytes;
  return SPD_OK;
}

extern "C" spd_status spd_prefix_attention_ruled(const spd_cache* c, int32_t layer, const void* q, int64_t q_stride, void* out,
                                                 int64_t out_stride, int32_t n_q_heads, int32_t dtype, const int32_t* seqs,
                                                 int32_t nseqs, const int32_t* cu_groups, const int32_t* prefix_lens,
                                                 int32_t ngroups, int32_t max_len, const spd_attention_rule* rule, void* workspace,
                                                 size_t ws_bytes, void* stream) {
  const char* call = "ruled prefix attention";
  size_t need = 0;
  spd_status st = spd_prefix_attention_ruled_workspace(c, n_q_heads, dtype, nseqs, ngroups, max_len, &need);
  if (st == SPD_OK) st = check_call(call, c, layer, q, q_stride, out, out_stride, n_q_heads, dtype, seqs);
  if (st == SPD_OK) st = check_rule(call, rule);
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
  run_ruled(a, *rule, dtype, request(*c, n_q_heads, nseqs, nseqs, ngroups, max_len, true, true, rule->window, rule->open_lens != nullptr), true, workspace, (hipStream_t)stream);
  return check_launch(call);
}
