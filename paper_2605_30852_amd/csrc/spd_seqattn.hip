// Attention over a cache of several sequences: packed causal rows (prompts), and decode rows of which groups share a
// prefix.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "spd_cachefn.h"

namespace spd {
namespace {

constexpr int kMaxG = 16;  // query heads of a KV head

// One layer of the cache, and the rows.
struct SeqArgs {
  spd_cache c;
  const void* kv;  // the layer's pool
  const void* q;
  void* out;
  int64_t qs, os;  // row strides, elements
  const int* seqs;
  const int* cu;      // prompts: cu_rows; decode rows: cu_groups
  const int* prefix;  // decode rows: prefix_lens
  int hq, G, nseqs, rows, ngroups;
  float scale;
};

// Where a row's keys are: those below `shared` through `first`, the others through `own` (rows of the page table).
struct Keys {
  const int *first, *own;
  int shared;
  __device__ __forceinline__ int page(const spd_cache& c, int key) const {
    return page_to_read(c, (key < shared ? first : own)[key / kPage]);
  }
};

// A query over the keys [0, n) in plain fp32, by the whole workgroup: scores in passes of 256 keys, computed twice
// rather than kept. M, L and a (dims 4 d4 .. + 3 of thread d4 = tid % (DH / 4)) are the maximum, the sum and the
// output; true in the threads that hold them. lds: kWG * 6 floats.
template <typename T, typename KVT, int DH>
__device__ bool plain_query(const spd_cache& c, const KVT* pool, const Keys keys, int g, const T* q, float scale, int k0, int k1,
                            float* lds, float& M, float& L, float (&a)[4]) {
  constexpr int TPQ = DH / 4, NG = kWG / TPQ;
  const int tid = threadIdx.x, d4 = tid % TPQ, grp = tid / TPQ;
  const size_t half = (size_t)c.n_kv_heads * kPage * DH;
  float* sp = lds;
  float* sr = lds + kWG;
  auto row = [&](int key) { return pool + keys.page(c, key) * 2 * half + (size_t)(g * kPage + key % kPage) * DH; };
  auto score = [&](int key) {
    const KVT* k = row(key);
    float s = 0.f;
#pragma unroll 4
    for (int d = 0; d < DH; d += 8) {
      float f[8], x[8];
      load8(k + d, f);
      load8(q + d, x);
#pragma unroll
      for (int e = 0; e < 8; e++) s = fmaf(x[e] * scale, f[e], s);
    }
    return s;
  };
  float m = -INFINITY;
  bool sound = true;
  for (int key = k0 + tid; key < k1; key += kWG) {
    const float s = score(key);
    m = fmaxf(m, s);
    sound = sound && s < INFINITY;
  }
  m = wave_max(m);
  const bool wave_sound = __all(sound);
  __syncthreads();  // the area's earlier readers are done
  if ((tid & 63) == 0) {
    sp[tid >> 6] = m;
    sp[4 + (tid >> 6)] = wave_sound ? 0.f : 1.f;
  }
  __syncthreads();
  M = fmaxf(fmaxf(sp[0], sp[1]), fmaxf(sp[2], sp[3]));
  const bool all_sound = sp[4] + sp[5] + sp[6] + sp[7] == 0.f;
  __syncthreads();
  if (!all_sound) {  // a score that is NaN or +inf makes every dim NaN
    L = a[0] = a[1] = a[2] = a[3] = NAN;
    return grp == 0;
  }
  L = a[0] = a[1] = a[2] = a[3] = 0.f;
  for (int base = k0; base < k1; base += kWG) {
    float p = 0.f;
    if (base + tid < k1) {
      const float s = score(base + tid);
      p = s == -INFINITY ? 0.f : expf(s - M);
    }
    sp[tid] = p;
    __syncthreads();
    const int n = min(kWG, k1 - base);
    for (int i = grp; i < n; i += NG) {
      const KVT* v = row(base + i) + half + 4 * d4;
      const float2 v0 = ld2<KVT>(v), v1 = ld2<KVT>(v + 2);
      const float pk = sp[i];
      L += pk;
      a[0] = fmaf(pk, v0.x, a[0]);
      a[1] = fmaf(pk, v0.y, a[1]);
      a[2] = fmaf(pk, v1.x, a[2]);
      a[3] = fmaf(pk, v1.y, a[3]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; i++) sr[tid * 5 + i] = a[i];
  sr[tid * 5 + 4] = L;
  __syncthreads();
  if (grp != 0) return false;
#pragma unroll 1
  for (int i = 1; i < NG; i++) {
    const float* o = sr + (i * TPQ + d4) * 5;
#pragma unroll
    for (int k = 0; k < 4; k++) a[k] += o[k];
    L += o[4];
  }
  return true;
}

__device__ __forceinline__ void store4(float* p, const float (&a)[4], float f) {
  *reinterpret_cast<float4*>(p) = make_float4(a[0] * f, a[1] * f, a[2] * f, a[3] * f);
}
__device__ __forceinline__ void store4(uint16_t* p, const float (&a)[4], float f) {
  *reinterpret_cast<uint2*>(p) = make_uint2(to_bf16(a[0] * f) | (uint32_t)to_bf16(a[1] * f) << 16,
                                            to_bf16(a[2] * f) | (uint32_t)to_bf16(a[3] * f) << 16);
}

// Row r's heads of KV head g over keys [0, n).
template <typename T, typename KVT, int DH>
__device__ void plain_row(const SeqArgs& A, const Keys keys, int r, int g, int n, float* lds) {
  for (int h = g * A.G; h < (g + 1) * A.G; h++) {
    float a[4], M, L;
    T* out = (T*)A.out + r * A.os + h * DH + 4 * (threadIdx.x % (DH / 4));
    if (n <= 0) {
      const float z[4] = {0.f, 0.f, 0.f, 0.f};
      if (threadIdx.x < DH / 4) store4(out, z, 0.f);
    } else if (plain_query<T, KVT, DH>(A.c, (const KVT*)A.kv, keys, g, (const T*)A.q + r * A.qs + h * DH, A.scale, 0, n, lds, M, L, a)) {
      store4(out, a, 1.0f / L);
    }
  }
}

template <typename T, typename KVT, int DH>
__global__ __launch_bounds__(kWG) void k_prompt_plain(SeqArgs A) {
  __shared__ float lds[kWG * 6];
  const RowAt at = row_at(A.c, A.seqs, A.cu, A.nseqs, blockIdx.x);
  if (at.seq < 0) return;
  const int* table = A.c.page_table + (size_t)at.seq * A.c.max_pages;
  plain_row<T, KVT, DH>(A, Keys{table, table, 0}, blockIdx.x, blockIdx.y, at.key + 1, lds);
}

template <typename T, typename KVT, int DH>
__global__ __launch_bounds__(kWG) void k_prefix_plain(SeqArgs A) {
  __shared__ float lds[kWG * 6];
  const int r = blockIdx.x, s = A.seqs[r];
  if ((unsigned)s >= (unsigned)A.c.max_seqs) return;
  const int* own = A.c.page_table + (size_t)s * A.c.max_pages;
  Keys keys{own, own, 0};
  if (A.ngroups > 0) {
    const int j = find_last(A.cu, A.ngroups, r), b = A.cu[j];
    const int f = (unsigned)b < (unsigned)A.nseqs ? A.seqs[b] : -1;
    if ((unsigned)f < (unsigned)A.c.max_seqs) {
      keys.first = A.c.page_table + (size_t)f * A.c.max_pages;
      keys.shared = min(A.prefix[j], seq_len(A.c, f));
    }
  }
  plain_row<T, KVT, DH>(A, keys, r, blockIdx.y, seq_len(A.c, s), lds);
}

template <typename T, typename KVT, int DH>
void launch_plain(const SeqArgs& a, bool prefix, hipStream_t s) {
  if (prefix)
    hipLaunchKernelGGL((k_prefix_plain<T, KVT, DH>), dim3(a.nseqs, a.c.n_kv_heads), dim3(kWG), 0, s, a);
  else
    hipLaunchKernelGGL((k_prompt_plain<T, KVT, DH>), dim3(a.rows, a.c.n_kv_heads), dim3(kWG), 0, s, a);
}

void launch_plain_typed(const SeqArgs& a, int dtype, bool prefix, hipStream_t s) {
  const bool wide = a.c.head_dim == 128;
  if (dtype == SPD_BF16)
    wide ? launch_plain<uint16_t, uint16_t, 128>(a, prefix, s) : launch_plain<uint16_t, uint16_t, 64>(a, prefix, s);
  else if (a.c.dtype == SPD_BF16)
    wide ? launch_plain<float, uint16_t, 128>(a, prefix, s) : launch_plain<float, uint16_t, 64>(a, prefix, s);
  else
    wide ? launch_plain<float, float, 128>(a, prefix, s) : launch_plain<float, float, 64>(a, prefix, s);
}

// What both attentions check of their sizes.
spd_status check_sizes(const char* call, const spd_cache* c, int n_q_heads, int dtype, int nseqs, int max_len) {
  const spd_status st = check_cache(call, c, false);
  if (st != SPD_OK) return st;
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads || n_q_heads / c->n_kv_heads > kMaxG)
    return invalid(call, "n_q_heads must be n_kv_heads times 1 .. 16");
  if (dtype != SPD_F32 && dtype != SPD_BF16) return invalid(call, "dtype must be SPD_F32 or SPD_BF16");
  if (dtype == SPD_BF16 && c->dtype != SPD_BF16) return invalid(call, "bf16 queries need a bf16 cache");
  if (nseqs < 1 || nseqs > kMaxSeqs) return invalid(call, "nseqs must be in [1, 65536]");
  if (max_len < 0) return invalid(call, "max_len must not be negative");
  return SPD_OK;
}

spd_status check_call(const char* call, const spd_cache* c, int layer, const void* q, int64_t q_stride, const void* out,
                      int64_t out_stride, int n_q_heads, int dtype, const int* seqs) {
  spd_status st = check_rows(call, q, q_stride, n_q_heads, c->head_dim, dtype);
  if (st == SPD_OK) st = check_rows(call, out, out_stride, n_q_heads, c->head_dim, dtype);
  if (st != SPD_OK) return st;
  if (layer < 0 || layer >= c->n_layers) return invalid(call, "no such layer");
  if (!seqs || misaligned(seqs, 4)) return invalid(call, "NULL or misaligned pointer");
  return SPD_OK;
}

SeqArgs args_of(const spd_cache* c, int layer, const void* q, int64_t q_stride, void* out, int64_t out_stride, int n_q_heads,
                const int* seqs, int nseqs) {
  SeqArgs a{};
  a.c = *c;
  a.kv = (const char*)c->kv + (size_t)layer * c->num_pages * 2 * c->n_kv_heads * kPage * c->head_dim * elem_bytes(c->dtype);
  a.q = q;
  a.out = out;
  a.qs = q_stride;
  a.os = out_stride;
  a.seqs = seqs;
  a.hq = n_q_heads;
  a.G = n_q_heads / c->n_kv_heads;
  a.nseqs = nseqs;
  a.scale = (float)(1.0 / std::sqrt((double)c->head_dim));
  return a;
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" spd_status spd_prompt_attention_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                     int32_t rows, int32_t max_len, size_t* bytes) {
  const char* call = "prompt attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (!bytes || rows < 0) return invalid(call, "NULL pointer or negative rows");
  *bytes = 0;
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
  launch_plain_typed(a, dtype, false, (hipStream_t)stream);
  return check_launch(call);
}

extern "C" spd_status spd_prefix_attention_workspace(const spd_cache* c, int32_t n_q_heads, int32_t dtype, int32_t nseqs,
                                                     int32_t ngroups, int32_t max_len, size_t* bytes) {
  const char* call = "prefix attention workspace";
  const spd_status st = check_sizes(call, c, n_q_heads, dtype, nseqs, max_len);
  if (st != SPD_OK) return st;
  if (nseqs > 4096) return invalid(call, "nseqs must be at most 4096");
  if (!bytes || ngroups < 0 || ngroups > nseqs) return invalid(call, "NULL pointer, or ngroups outside [0, nseqs]");
  *bytes = 0;
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
  launch_plain_typed(a, dtype, true, (hipStream_t)stream);
  return check_launch(call);
}
