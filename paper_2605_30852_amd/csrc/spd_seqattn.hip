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
  int G, nseqs, rows, ngroups, rpt;
  float scale;
};

constexpr float kLog2e = 1.44269504088896341f;

// 2^-down times n numbers sum to less than the largest of them.
__device__ __forceinline__ int down_of(int n) { return 33 - __clz(n); }

// A query over the keys [k0, k1) in plain fp32, by the whole workgroup, which a query, key or value that is not finite
// needs: there 0 times a value behind the query's own keys, or a plane's 0 * inf, is NaN on matrix cores. So do finite values
// whose sum is not, and here every probability, at most 1, is lowered by a power of two that keeps a sum below the largest value.
// Scores in passes of a key a thread, computed twice rather than kept. M, L and a (dims 4 d4 .. + 3 of thread d4 = tid % (DH / 4))
// are the offset of the exponents (in units of log2), the sum and the output; true in the threads that hold them. lds: 6 * kWG floats.
template <typename T, typename KVT, int DH>
__device__ bool plain_query(const spd_cache& c, const KVT* pool, const int* table, int g, const T* q, float scale, int k0,
                            int k1, float* lds, float& M, float& L, float (&a)[4]) {
  constexpr int TPQ = DH / 4, NG = kWG / TPQ, NW = kWG / 64;
  const int tid = threadIdx.x, d4 = tid % TPQ, grp = tid / TPQ;
  const size_t half = (size_t)c.n_kv_heads * kPage * DH;
  float* sp = lds;
  float* sr = lds + kWG;
  auto row = [&](int key) { return pool + page_to_read(c, table[key / kPage]) * 2 * half + (size_t)(g * kPage + key % kPage) * DH; };
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
    sp[NW + (tid >> 6)] = wave_sound ? 0.f : 1.f;
  }
  __syncthreads();
  float unsound = 0.f;
  M = sp[0];
#pragma unroll
  for (int i = 0; i < NW; i++) {
    M = fmaxf(M, sp[i]);
    unsound += sp[NW + i];
  }
  const bool all_sound = unsound == 0.f;
  __syncthreads();
  if (!all_sound) {  // a score that is NaN or +inf makes every dim NaN
    L = a[0] = a[1] = a[2] = a[3] = NAN;
    return grp == 0;
  }
  L = a[0] = a[1] = a[2] = a[3] = 0.f;
  const int down = down_of(k1 - k0);
  const float top = M, part = ldexpf(1.0f, -down);
  M = fmaf(top, kLog2e, (float)down);
  for (int base = k0; base < k1; base += kWG) {
    float p = 0.f;
    if (base + tid < k1) {
      const float s = score(base + tid);
      p = s == -INFINITY ? 0.f : expf(s - top) * part;
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
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a[0] * f, a[1] * f), pack_bf16(a[2] * f, a[3] * f));
}

// --------------------------------------------------------------------------------------- pieces of the work
// A call's work is cut on the device, by one workgroup, into pieces: some queries of a KV head (rows times its G
// heads) over a run of keys. A prompt's tile of rows is a job over the keys up to its last row; a group's rows are jobs
// over its prefix, and each row one over the keys behind it. Jobs longer than a `chunk` are split, so that a few rows
// behind long caches fill the GPU: chunk = all jobs' keys / pieces wanted of a KV head. The pieces are
// handed out longest first (a counting sort of their lengths), which is what keeps the last workgroups short.
// 512 pieces wanted, two a CU: with 256 a prefix of 8192 keys for 64 rows takes 47.5 us instead of 42.2, with 384, 768 or 1024
// no case gains. The plan itself is a chain of loads and barriers, 5 to 8 us by rocprofv3 up to 1024 jobs.
// A job of one piece writes its rows' outputs; the pieces of others leave records (o, m, l), which the merge joins in
// the order of the keys.
struct Item {
  int row0, nrows;  // rows of q
  int table;        // the sequence whose pages hold the keys
  int k0, k1;       // keys
  int rec;          // first record, -1: outputs
  int lim0;         // causal: row row0 + i attends keys below lim0 + i
  int mode;
};
enum { ITEM_FEW = 1, ITEM_PAIR = 2, ITEM_FLAT = 4 };  // at most 16 queries; at most 32 (of an fp32 cache); each row attends its sequence's keys

// Rows whose pieces' records are to be joined: those of up to two jobs.
struct Merge {
  int row0, nrows;
  int rec[2], pieces[2];
  int queries[2], first[2];  // queries of the job (a KV head's records of a piece), and the first one of these rows
  int lim0, mode;
};

constexpr int kPlanWG = 1024, kSmallPlanWG = 256;
constexpr int kMinChunk = 256;
constexpr int kWantedWGs = 512;
constexpr size_t kMaxWGs = (1 << 24) - 1;  // of 256 threads: a launch's threads are below 2^32
constexpr int kBuckets = 64;  // a wave's lanes

// The sums of some queries: `query` of merge `merge` and those behind it, as many as a workgroup of the merge takes.
struct Unit {
  int merge, query;
};

struct PlanArgs {
  spd_cache c;
  const int *seqs, *cu, *prefix;
  int nseqs, rows, ngroups, G, wanted;  // wanted: pieces of a KV head; 0: no job is split
  int rpt;                              // rows of a tile
  int tiles, jobs;
  int pair;                             // an fp32 cache: pieces of up to 32 queries
  int wide_cost;                        // of a key of a wide piece; 1: of one of few queries, 2: of a pair
  int qpu;                              // queries of a merge's workgroup
  int* count;                           // items, units
  Item* items;
  Merge* merges;
  Unit* units;
  int4* tile_rec;                       // decode rows: a tile's first record, pieces and queries
};

struct Job {
  int row0, nrows, table, a, b, lim0, mode;
};

// The batch's description, in LDS where it fits: the plan's searches wait for each of its loads.
constexpr int kPlanSeqs = 4096;
struct Batch {
  const int *cu, *seqs, *lens, *prefix;  // LDS: cu_rows or cu_groups, sequences, their lengths by row of the batch, prefix_lens
  const int* base;                       // LDS: the number of a sequence's or group's first tile
  const PlanArgs* P;
  bool in_lds;
  __device__ __forceinline__ int cu_at(int i) const { return in_lds ? cu[i] : P->cu[i]; }
  __device__ __forceinline__ int seq_at(int i) const { return in_lds ? seqs[i] : P->seqs[i]; }
  __device__ __forceinline__ int prefix_at(int i) const { return in_lds ? prefix[i] : P->prefix[i]; }
  // The tiles of entry i have the numbers cu[i] / rpt + i and up: enough of them, in order, without a sum over those before.
  __device__ __forceinline__ int base_at(int i) const { return in_lds ? base[i] : P->cu[i] / P->rpt + i; }
  __device__ __forceinline__ int len_at(int i) const {  // -1: no such sequence
    if (in_lds) return lens[i];
    const int s = P->seqs[i];
    return (unsigned)s < (unsigned)P->c.max_seqs ? seq_len(P->c, s) : -1;
  }
  // last i in [0, n) with at(i) <= t, for at that ascends from at(0) <= t
  template <typename F>
  static __device__ __forceinline__ int last(int n, int t, F at) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (at(mid) <= t)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  }
  __device__ __forceinline__ int of_tile(int n, int t) const {
    return last(n, t, [&](int i) { return base_at(i); });
  }
  __device__ __forceinline__ int of_row(int n, int r) const {
    return last(n, r, [&](int i) { return cu_at(i); });
  }
};

__device__ __forceinline__ int size_mode(const PlanArgs& P, int nq) {
  return nq <= 16 ? ITEM_FEW : P.pair && nq <= 32 ? ITEM_PAIR : 0;
}

// Job t of a prompt call: a tile of a sequence's rows.
__device__ bool prompt_job(const PlanArgs& P, const Batch& B, int t, Job& j) {
  const int i = B.of_tile(P.nseqs, t);
  const int begin = B.cu_at(i), stop = B.cu_at(i + 1), end = min(stop, P.rows), len = B.len_at(i);
  if (begin < 0 || begin >= end || len < 0) return false;
  const long long row0 = begin + (long long)(t - B.base_at(i)) * P.rpt;
  if (row0 < begin || row0 >= end) return false;
  j.row0 = (int)row0;
  j.nrows = min(P.rpt, end - j.row0);
  j.table = B.seq_at(i);
  j.a = 0;
  j.lim0 = (int)max((long long)len - stop + j.row0 + 1, -(1ll << 30));
  j.b = max(0, j.lim0 + j.nrows - 1);
  j.mode = size_mode(P, j.nrows * P.G);
  return true;
}

// The prefix that group j shares: its length (0: none), the first row and the number of rows.
__device__ int shared_prefix(const PlanArgs& P, const Batch& B, int j, int& first, int& rows) {
  first = B.cu_at(j);
  rows = min(B.cu_at(j + 1), P.nseqs) - first;
  if (first < 0 || rows < 2) return 0;
  return min(max(B.prefix_at(j), 0), max(B.len_at(first), 0));
}

// Job t of a decode call: below `tiles` a tile of a group's rows over the prefix, else a row over the keys behind it.
// shared: a row's own job is joined with its prefix's, of tile `tile` from query `query` on.
__device__ bool prefix_job(const PlanArgs& P, const Batch& B, int t, Job& j, bool& shared, int& tile, int& query) {
  shared = false;
  int first, rows;
  j.lim0 = 0;
  j.a = 0;
  if (t < P.tiles) {
    if (P.ngroups == 0) return false;
    const int g = B.of_tile(P.ngroups, t), n = shared_prefix(P, B, g, first, rows);
    if (n == 0) return false;
    const long long at = (long long)(t - B.base_at(g)) * P.rpt;
    if (at < 0 || at >= rows) return false;
    j.row0 = first + (int)at;
    j.nrows = min(P.rpt, rows - (int)at);
    j.table = B.seq_at(first);
    j.b = n;
    j.mode = ITEM_FLAT | size_mode(P, j.nrows * P.G);
    shared = true;
    return true;
  }
  const int r = t - P.tiles, len = B.len_at(r);
  if (len < 0) return false;
  j.row0 = r;
  j.nrows = 1;
  j.table = B.seq_at(r);
  j.b = len;
  j.mode = ITEM_FLAT | ITEM_FEW;
  if (P.ngroups > 0) {
    const int g = B.of_row(P.ngroups, r), n = shared_prefix(P, B, g, first, rows);
    if (n > 0 && r >= first && r < first + rows) {
      shared = true;
      j.a = min(n, len);
      const int in_group = (r - first) / P.rpt;
      tile = B.base_at(g) + in_group;
      query = (r - first - in_group * P.rpt) * P.G;
    }
  }
  return true;
}

// Tiles whose records are kept in LDS for the rows that join them.
constexpr int kPlanTiles = 1024;

template <bool PREFIX, int NTH>
__global__ __launch_bounds__(NTH) void k_plan_attention(PlanArgs P) {
  __shared__ int s_cu[kPlanSeqs + 1], s_seqs[kPlanSeqs], s_lens[kPlanSeqs], s_base[kPlanSeqs], s_prefix[PREFIX ? kPlanSeqs : 1];
  __shared__ int4 s_tile[PREFIX ? kPlanTiles : 1];
  __shared__ unsigned long long s_total, s_max, s_sums[NTH / 64];
  __shared__ int s_back[NTH / 64];
  __shared__ int s_count[kBuckets], s_items;
  const int tid = threadIdx.x;
  const Batch B{s_cu, s_seqs, s_lens, s_prefix, s_base, &P, P.nseqs <= kPlanSeqs};
  bool back = false;  // a group that ends before it begins
  if (B.in_lds) {
    const int n = PREFIX ? P.ngroups : P.nseqs;
    for (int i = tid; i < P.nseqs; i += NTH) {
      const int s = P.seqs[i], c = i < n ? P.cu[i] : 0, x = PREFIX && i < n ? P.prefix[i] : 0;
      if (PREFIX) back = back || (i < n && P.cu[i + 1] < c);
      s_seqs[i] = s;
      s_lens[i] = (unsigned)s < (unsigned)P.c.max_seqs ? seq_len(P.c, s) : -1;
      if (i < n) {
        s_cu[i] = c;
        s_base[i] = c / P.rpt + i;
        if (PREFIX) s_prefix[i] = x;
      }
    }
    if (tid == 0 && n > 0) s_cu[n] = P.cu[n];
  }
  if (tid < kBuckets) s_count[tid] = 0;
  if (tid == 0) {
    s_total = 0ull;
    s_max = 1ull;
  }
  if (PREFIX) {
    const bool any = __any(back);
    if ((tid & 63) == 0) s_back[tid >> 6] = any;
  }
  __syncthreads();
  // Groups that ascend have no row in common, which is what the room for records is made for. Others are none: every row goes
  // through its own pages.
  if (PREFIX) {
#pragma unroll
    for (int i = 0; i < NTH / 64; i++)
      if (s_back[i]) P.ngroups = 0;
  }
  // A thread's jobs are tid, tid + NTH, ..: the first is kept.
  struct Known {
    Job j;
    bool is, shared;
    int tile, query;
  };
  auto work_out = [&](int t, Known& k) {
    if constexpr (PREFIX) {
      k.is = prefix_job(P, B, t, k.j, k.shared, k.tile, k.query);
    } else {
      k.shared = false;
      k.is = prompt_job(P, B, t, k.j);
    }
  };
  Known mine;
  mine.is = false;
  if (tid < P.jobs) work_out(tid, mine);
  auto each = [&](auto f) {
    if (mine.is) f(tid, mine);
    for (int t = tid + NTH; t < P.jobs; t += NTH) {
      Known k;
      work_out(t, k);
      if (k.is) f(t, k);
    }
  };
  auto cost = [&](int keys, int mode) { return (unsigned long long)keys * (mode & ITEM_FEW ? 1 : mode & ITEM_PAIR ? 2 : P.wide_cost); };
  {
    unsigned long long sum = 0ull, longest = 1ull;
    each([&](int, const Known& k) {
      const unsigned long long c = cost(k.j.b - k.j.a, k.j.mode);
      sum += c;
      longest = max(longest, c);
    });
    sum = wave_scan(sum);
    longest = wave_top(longest);
    if ((tid & 63) == 63) {
      atomicAdd(&s_total, sum);
      atomicMax(&s_max, longest);
    }
  }
  __syncthreads();
  // Split where a job is longer than a CU's share, two workgroups being on one.
  const bool split = P.wanted > 0 && s_max * (unsigned)max(P.wanted / 2, 1) > s_total;
  const unsigned long long share = split ? min((s_total + P.wanted - 1) / P.wanted, s_max) : s_max;
  const int chunk_few = max(kMinChunk, (int)((min(share, 1ull << 30) + 63) / 64 * 64));
  const int chunk_pair = max(kMinChunk / 2, (int)((min(share / 2, 1ull << 30) + 64) / 64 * 64));
  const int chunk_wide = max(kMinChunk / 2, (int)((min(share / P.wide_cost, 1ull << 30) + 64) / 64 * 64));
  auto chunk_of = [&](const Known& k) { return k.j.mode & ITEM_FEW ? chunk_few : k.j.mode & ITEM_PAIR ? chunk_pair : chunk_wide; };
  const float per_cost = (float)(kBuckets - 1) / (float)max(max(cost(chunk_few, ITEM_FEW), cost(chunk_pair, ITEM_PAIR)), cost(chunk_wide, 0));
  auto bucket = [&](int keys, int mode) {  // the costliest first
    return kBuckets - 1 - min((int)((float)cost(keys, mode) * per_cost), kBuckets - 1);
  };
  // a job's pieces; 0: nothing to do (a row that ends with its prefix)
  auto pieces_of = [&](const Known& k) {
    const int chunk = chunk_of(k);
    return k.j.b > k.j.a ? (k.j.b - k.j.a + chunk - 1) / chunk : k.shared ? 0 : 1;
  };
  each([&](int, const Known& k) {
    const int n = pieces_of(k), chunk = chunk_of(k);  // all but the last are whole
    if (n > 1) atomicAdd(&s_count[bucket(chunk, k.j.mode)], n - 1);
    if (n > 0) atomicAdd(&s_count[bucket(k.j.b - k.j.a - (n - 1) * chunk, k.j.mode)], 1);
  });
  __syncthreads();
  if (tid < kBuckets) {  // bucket counts to their first places
    const int v = s_count[tid], x = (int)wave_scan((unsigned)v);
    s_count[tid] = x - v;
    if (tid == kBuckets - 1) P.count[0] = s_items = x;
  }
  __syncthreads();
  // Where all pieces are on the GPU at once, the second half comes in ascending order: a CU has a long one and a short one.
  const int all = s_items, half = max(P.wanted / 2, 1);
  auto place = [&](int at) { return at < half || all > 2 * half ? at : all - 1 - (at - half); };
  // Places of records, merges and units come from a prefix sum over the jobs (64 lanes that add to one LDS word take about a
  // microsecond), packed: records of a KV head above, then merges and units, which stay below 2^16.
  unsigned long long before = 0ull;
  for (int t0 = 0; t0 < P.jobs; t0 += NTH) {
    const int t = t0 + tid;
    Known k = mine;
    if (t0 > 0) {
      k.is = false;
      if (t < P.jobs) work_out(t, k);
    }
    const bool tile = PREFIX && t < P.tiles;
    const int n = k.is ? pieces_of(k) : 0, nq = k.is ? k.j.nrows * P.G : 0, units = (nq + P.qpu - 1) / P.qpu;
    const bool joins = k.is && (n > 1 || k.shared);
    const unsigned long long v = joins ? (unsigned long long)(unsigned)(n * nq) << 32 | (tile ? 0 : 1u << 16 | units) : 0ull;
    const unsigned long long x = wave_scan(v);
    if ((tid & 63) == 63) s_sums[tid >> 6] = x;
    __syncthreads();
    unsigned long long at = before + x - v;
#pragma unroll
    for (int i = 0; i < NTH / 64; i++) {
      if (i < tid >> 6) at += s_sums[i];
      before += s_sums[i];
    }
    const int rec = joins ? (int)((long long)(at >> 32) * P.c.n_kv_heads) : -1;
    if (tile) {
      const int4 r = joins ? make_int4(rec, n, nq, 0) : make_int4(0, 0, 0, 0);
      if (t < kPlanTiles)
        s_tile[t] = r;
      else
        P.tile_rec[t] = r;
    }
    __syncthreads();  // tiles come before the rows that join them; the sums are read
    if (joins && !tile) {
      int4 r = make_int4(0, 0, 0, 0);
      if (PREFIX && k.shared) r = k.tile < kPlanTiles ? s_tile[k.tile] : P.tile_rec[k.tile];
      Merge m;
      m.row0 = k.j.row0;
      m.nrows = k.j.nrows;
      m.rec[0] = r.x;
      m.pieces[0] = k.shared && k.query + nq <= r.z ? r.y : 0;
      m.queries[0] = r.z;
      m.first[0] = k.shared ? k.query : 0;
      m.rec[1] = rec;
      m.pieces[1] = n;
      m.queries[1] = nq;
      m.first[1] = 0;
      m.lim0 = k.j.lim0;
      m.mode = k.j.mode;
      const int at_merge = (int)(at >> 16 & 0xffff), at_unit = (int)(at & 0xffff);
      P.merges[at_merge] = m;
      for (int u = 0; u < units; u++) P.units[at_unit + u] = Unit{at_merge, u * P.qpu};
    }
    int chunk = 0, whole = 0, rest = 0;
    if (n > 0) {
      chunk = chunk_of(k);
      if (n > 1) whole = atomicAdd(&s_count[bucket(chunk, k.j.mode)], n - 1);
      rest = atomicAdd(&s_count[bucket(k.j.b - k.j.a - (n - 1) * chunk, k.j.mode)], 1);
    }
    const int step = P.c.n_kv_heads * nq;
    auto write = [&](const Job& j, int p, int n, int chunk, int whole, int rest, int rec, int step) {
      const int a = j.a + p * chunk;
      P.items[place(p < n - 1 ? whole + p : rest)] =
          Item{j.row0, j.nrows, j.table, a, max(a, min(j.b, a + chunk)), rec < 0 ? -1 : rec + p * step, j.lim0, j.mode};
    };
    // A few long jobs are written by their wave, a piece a lane: 0.5 us of 7.1 with 16 pieces in each of two, the call 1.1 of 42.4.
    unsigned long long many = __ballot(n > 8);
    if (__popcll(many) > 8) many = 0ull;
    if (!(many >> (tid & 63) & 1ull))
      for (int p = 0; p < n; p++) write(k.j, p, n, chunk, whole, rest, rec, step);
    for (; many != 0ull; many &= many - 1ull) {
      const int from = __builtin_ctzll(many);
      auto of = [&](int x) { return __builtin_amdgcn_readlane(x, from); };
      const Job j{of(k.j.row0), of(k.j.nrows), of(k.j.table), of(k.j.a), of(k.j.b), of(k.j.lim0), of(k.j.mode)};
      const int jn = of(n), jc = of(chunk), jw = of(whole), jr = of(rest), rec0 = of(rec), st = of(step);
      for (int p = tid & 63; p < jn; p += 64) write(j, p, jn, jc, jw, jr, rec0, st);
    }
  }
  if (tid == 0) P.count[1] = (int)(before & 0xffff);
}

// Records: o, then (m, l) with m in units of log2.
struct Records {
  float* o;
  float2* ml;
};

// ------------------------------------------------------------------------------------------ a piece on matrix cores
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const char gbytes;
typedef __attribute__((address_space(3))) char lbytes;
typedef __attribute__((address_space(3))) bf16x4 lbf16x4;

// x as three bf16 values by truncation, whose sum it is exactly (finite x).
__device__ __forceinline__ void planes3(float x, uint32_t& h, uint32_t& m, uint32_t& l) {
  const uint32_t a = __float_as_uint(x);
  const float r1 = x - __uint_as_float(a & 0xffff0000u);
  const uint32_t b = __float_as_uint(r1);
  h = a >> 16;
  m = b >> 16;
  l = __float_as_uint(r1 - __uint_as_float(b & 0xffff0000u)) >> 16;
}

// Two probabilities (finite, not negative) as planes of a product's operand: rounded to one bf16 each, or three that are exact.
__device__ __forceinline__ void planes_of(float p0, float p1, uint32_t (&u)[1]) { u[0] = pack_bf16(p0, p1); }
__device__ __forceinline__ void planes_of(float p0, float p1, uint32_t (&u)[3]) {
  const uint32_t h0 = __float_as_uint(p0), h1 = __float_as_uint(p1);
  const float r0 = p0 - __uint_as_float(h0 & 0xffff0000u), r1 = p1 - __uint_as_float(h1 & 0xffff0000u);
  const uint32_t m0 = __float_as_uint(r0), m1 = __float_as_uint(r1);
  const uint32_t l0 = __float_as_uint(r0 - __uint_as_float(m0 & 0xffff0000u));
  const uint32_t l1 = __float_as_uint(r1 - __uint_as_float(m1 & 0xffff0000u));
  u[0] = __builtin_amdgcn_perm(h1, h0, 0x07060302u);
  u[1] = __builtin_amdgcn_perm(m1, m0, 0x07060302u);
  u[2] = __builtin_amdgcn_perm(l1, l0, 0x07060302u);
}

// l plus what was made of the two: the rounded values in one instruction (1% of a long prompt's time), or the values.
__device__ __forceinline__ float add_planes(float l, float, float, const uint32_t (&u)[1]) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u[0]), __builtin_bit_cast(bf16x2, 0x3f803f80u), l, false);
}
__device__ __forceinline__ float add_planes(float l, float p0, float p1, const uint32_t (&)[3]) { return l + (p0 + p1); }

// A lane's part of a query: 8 dims from q on, every `step`. bf16 as they are; fp32 times f, as planes.
template <typename T, int KS, int STEP, int NP>
__device__ __forceinline__ void load_query(bf16x8 (&qf)[NP][KS], const T* q, float f) {
#pragma unroll
  for (int s = 0; s < KS; s++) {
    if constexpr (NP == 1) {
      qf[0][s] = *reinterpret_cast<const bf16x8*>(q + s * STEP);
    } else {
      float x[8];
      load8(q + s * STEP, x);
      union { uint16_t u[8]; bf16x8 v; } t[3];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        uint32_t a, b, c;
        planes3(x[e] * f, a, b, c);
        t[0].u[e] = (uint16_t)a;
        t[1].u[e] = (uint16_t)b;
        t[2].u[e] = (uint16_t)c;
      }
#pragma unroll
      for (int p = 0; p < 3; p++) qf[p][s] = t[p].v;
    }
  }
}

// Keys that a row of a piece attends (of the whole sequence).
__device__ __forceinline__ int row_limit(const SeqArgs& A, const Item& it, int row) {
  if (!(it.mode & ITEM_FLAT)) return it.lim0 + row - it.row0;
  const int s = A.seqs[row];
  return (unsigned)s < (unsigned)A.c.max_seqs ? seq_len(A.c, s) : 0;
}

// Query j of a piece again, in plain arithmetic, in the place of its result.
template <typename T, typename KVT, int DH>
__device__ void plain_piece(const SeqArgs& A, const Item& it, const Records& R, int g, int j, float* lds) {
  const int r = it.row0 + j / A.G, head = g * A.G + j % A.G, d = 4 * (threadIdx.x % (DH / 4));
  const int n = min(row_limit(A, it, r), it.k1);
  float a[4] = {0.f, 0.f, 0.f, 0.f}, M = -INFINITY, L = 0.f;
  bool holds = threadIdx.x < DH / 4;
  if (n > it.k0)
    holds = plain_query<T, KVT, DH>(A.c, (const KVT*)A.kv, A.c.page_table + (size_t)it.table * A.c.max_pages, g,
                                    (const T*)A.q + r * A.qs + head * DH, A.scale, it.k0, n, lds, M, L, a);
  if (!holds) return;
  if (it.rec < 0) {
    store4((T*)A.out + r * A.os + head * DH + d, a, n > 0 ? 1.0f / L : 0.f);
  } else {
    const size_t at = (size_t)it.rec + (size_t)g * it.nrows * A.G + j;
    store4(R.o + at * DH + d, a, 1.0f);
    if (d == 0) R.ml[at] = make_float2(M, L);
  }
}

// The end of a piece of 32 queries a wave: registers 4 v .. + 3 of tile t are dims 32 t + 8 v + 4 h .. + 3 of the lane's query, which
// attends keys below lim.
template <typename T, typename KVT, int DH>
__device__ void finish_wide(const SeqArgs& A, const Item& it, const Records R, int g, const f32x16 (&o)[DH / 32], float m_run,
                            float l_run, int lim, char* lds) {
  constexpr int NT = DH / 32;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int G = A.G, nq = it.nrows * G, jq = w * 32 + col, jj = min(jq, nq - 1), row = it.row0 + jj / G, head = g * G + jj % G;
  const bool active = w * 32 < nq, mine = jq < nq;
  l_run += __shfl_xor(l_run, 32, 64);

  __shared__ uint32_t s_bad[kWG / 64];  // queries whose result here is not finite
  if (tid < kWG / 64) s_bad[tid] = 0u;
  __syncthreads();
  if (active) {
    bool bad = !(l_run > 0.f) && lim > it.k0;  // NaN, or nothing but scores of -inf
#pragma unroll
    for (int tt = 0; tt < NT; tt++)
#pragma unroll
      for (int v = 0; v < 16; v++) bad = bad || !(fabsf(o[tt][v]) < INFINITY);
    const unsigned long long bads = __ballot(bad && mine);
    if (lane == 0) s_bad[w] = (uint32_t)bads | (uint32_t)(bads >> 32);
    if (mine) {
      const size_t at = (size_t)max(it.rec, 0) + (size_t)g * nq + jq;
      const float inv = lim > 0 ? 1.0f / l_run : 0.f;
#pragma unroll
      for (int tt = 0; tt < NT; tt++)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
          const float x[4] = {o[tt][v], o[tt][v + 1], o[tt][v + 2], o[tt][v + 3]};
          const int d = tt * 32 + 2 * v + 4 * h;
          if (it.rec < 0)
            store4((T*)A.out + row * A.os + head * DH + d, x, inv);
          else
            store4(R.o + at * DH + d, x, 1.0f);
        }
      if (it.rec >= 0 && h == 0) R.ml[at] = make_float2(m_run, l_run);
    }
  }
  __syncthreads();  // every result is stored, and the tiles are free
  for (int i = 0; i < kWG / 64; i++)
    for (uint32_t m = __builtin_amdgcn_readfirstlane(s_bad[i]); m != 0u; m &= m - 1u)
      plain_piece<T, KVT, DH>(A, it, R, g, i * 32 + __builtin_ctz(m), (float*)lds);
}

// A piece of bf16 keys for 32 queries a wave. Query j of the tile is row row0 + j / G, head g * G + j % G.
//   S^T = K Q^T (v_mfma_f32_32x32x16_bf16: lane l supplies 8 consecutive k of A row l % 32 and of B column l % 32, from
//     k = 8 (l / 32); accumulator register v of lane l is row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32): lane l
//     holds 16 of a 32-key block's scores of query l % 32, lane l ^ 32 the others.
//   The softmax is in powers of two. Its offset m is a maximum that is only renewed, and the sums rescaled, when a score of some
//     query of the wave exceeds it by more than 8: p stays below 2^8, its rounding is relative and the sums are
//     fp32, and the other steps need neither the other half's scores nor a rescaling.
//   O^T += V^T P^T: registers 8 s .. 8 s + 7 of half h are the probabilities of keys 16 s + 4 h + 0..3 and 16 s + 8 + 4 h
//     + 0..3, which two transposing LDS reads of V rows give as the A operand.
// bf16 queries: q as it is, the scale in the exponent's FMA, p rounded to bf16 (half a step, 2^-8 of each p: as much as the
// rounding of the output), l the sum of the rounded p. The outputs' error against 64 bits is 2.0e-3 to 2.3e-3 (relative norm, values of
// mean 0, where roundings show most); p as two planes, 16 bits, makes it the output's own rounding, 1.63e-3 to 1.66e-3, and takes 2932 us
// for 2144 at 16381 rows, 172 for 140 in ten packed prompts, 56 for 46 behind long caches, 44.5 for 42 behind a shared prefix. Who
// wants more than a bf16 output's accuracy has fp32 queries: q (scaled in fp32) and p as three exact planes, three products each.
// K and V go to LDS by direct loads, the 16-byte chunks of a row permuted by its key so that neither kind of read
// meets itself in a bank. A step reads its V fragments before it requests the next tile: the compiler lets every read of LDS
// wait for the direct loads before it, and so the request has the softmax and the products to land in.
// Two workgroups are on a CU, so that one's matrix work meets the other's vector work: a step of 64 keys takes a workgroup
// 1.17 us alone on its CU and 2.0 beside another. 64 queries a wave instead leave registers for one workgroup a CU and reached
// 664 TFLOP/s; eight waves of 256 queries that take turns were 2% faster at 16381 rows and slower on short prompts.
// Measured (32 heads of 128 over 8): 16381 causal rows 2.04 to 2.18 ms, 1010 to 1075 TFLOP/s of 1360 that a square product of 16384
// reaches, two thirds of its cycles in the matrix cores with the clock down to 1.5 GHz: power bounds it. Ten packed prompts of 8191
// rows 135 us, 720 TFLOP/s, 40% of the cycles in the matrix cores: a piece costs some 6 us beside its steps (item, pages, first
// keys, output), which workgroups that stay and take piece after piece did not shorten (149 us where the others took 143). fp32
// queries, 2048 rows: 110 us, 312 TFLOP/s of the scores and outputs, three times that in products, 57% of the cycles.
template <typename T, int DH>
__device__ void piece_wide(const SeqArgs& A, const Item& it, const Records R, int g, char* lds) {
  constexpr int NP = sizeof(T) == 4 ? 3 : 1;
  constexpr int KT = NP == 3 && DH == 128 ? 32 : 64;  // 32: three planes of q leave no registers for 64
  constexpr int NT = DH / 32, KS = DH / 16, NCH = DH / 8, SB = KT / 32;
  constexpr int KBUF = KT * DH * 2, LPT = KT * NCH / kWG;
  constexpr int KROT = DH == 128 ? 0 : 1;  // K: chunk c of key k sits at c ^ (k >> KROT) % NCH: 16 keys in 64 banks
  constexpr int VROT = DH == 128 ? 0 : 1;  // V: chunk c of key k sits at c ^ (k % 8 >> VROT) << 1
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int G = A.G, nq = it.nrows * G;
  const spd_cache& C = A.c;
  const int last = it.k1 - 1;
  const int start = it.k0 & ~(kPage - 1), tiles = (it.k1 - start + KT - 1) / KT;
  const size_t half = (size_t)C.n_kv_heads * kPage * DH;
  const uint16_t* pool = (const uint16_t*)A.kv + (size_t)g * kPage * DH;
  const int* table = C.page_table + (size_t)it.table * C.max_pages;
  // The pages of a tile, one a lane (mod their number), are read a tile ahead of their use, and looked at only there: a look
  // at them here would wait for them and for the keys requested before them.
  auto pages = [&](int t) { return table[min(start / kPage + t * (KT / kPage) + (lane & (KT / kPage - 1)), last / kPage)]; };
  const int pg0 = tiles > 0 ? pages(0) : 0;
  int pg = tiles > 0 ? pages(1) : 0;
  const float sc = NP == 1 ? A.scale * kLog2e : 1.0f;  // from scores to exponents
  const bool active = w * 32 < nq;
  const int jq = w * 32 + col, jj = min(jq, nq - 1), row = it.row0 + jj / G, head = g * G + jj % G;
  const int lim = min(row_limit(A, it, row), it.k1);

  bf16x8 qf[NP][KS];
  load_query<T, KS, 16>(qf, (const T*)A.q + row * A.qs + head * DH + h * 8, A.scale * kLog2e);
  // keys below wmin are attended by every query of the wave, none at wmax and above by any
  int wmin = it.lim0 + w * 32 / G, wmax = it.lim0 + min(w * 32 + 31, nq - 1) / G;
  if (it.mode & ITEM_FLAT) {
    wmin = wmax = lim;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      wmin = min(wmin, __shfl_xor(wmin, d, 64));
      wmax = max(wmax, __shfl_xor(wmax, d, 64));
    }
  }
  wmin = __builtin_amdgcn_readfirstlane(min(wmin, it.k1));
  wmax = __builtin_amdgcn_readfirstlane(active ? min(wmax, it.k1) : 0);

  // A thread's bytes of a page, load i: chunk lc of key lk, or of keys 16 apart.
  const int lk = tid / NCH, lc = tid % NCH;
  static_assert(kWG / NCH % kPage == 0 && LPT >= 1, "a pass of the workgroup is whole pages");
  const uint32_t koff = (lc ^ (lk >> KROT) % NCH) << 4;
  const uint32_t voff = (lc ^ (lk & 7) >> VROT << 1) << 4;
  const size_t page_bytes = 2 * half * sizeof(uint16_t);
  // Tile t. Keys outside [k0, k1) are read as the nearest one inside: their probability is 0, and 0 times a value must be 0. The
  // pages go to scalar registers first: looked at between loads, a lane's register would wait for those before it.
  auto request = [&](int t, int pg) {
    const int first = start + t * KT, to = (t & 1) * 2 * KBUF;
    int page[LPT];
#pragma unroll
    for (int i = 0; i < LPT; i++) page[i] = page_to_read(C, __builtin_amdgcn_readlane(pg, (i * kWG + w * 64) / (NCH * kPage)));
#pragma unroll
    for (int i = 0; i < LPT; i++) {
      const uint32_t at = (uint32_t)(min(max(first + i * (kWG / NCH) + lk, it.k0), last) & (kPage - 1)) * (DH * 2);
      gbytes* p = (gbytes*)pool + (size_t)page[i] * page_bytes;
      lbytes* l = (lbytes*)(lds + to + (i * kWG + w * 64) * 16);
      __builtin_amdgcn_global_load_lds(p + (at + koff), l, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(p + half * sizeof(uint16_t) + (at + voff), l + KBUF, 16, 0, 0);
    }
  };
  // A lane's bytes of a K or V tile.
  uint32_t ka[KS], va[NT];
#pragma unroll
  for (int k = 0; k < KS; k++) ka[k] = col * DH * 2 + (((2 * k + h) ^ (col >> KROT) % NCH) << 4);
#pragma unroll
  for (int tt = 0; tt < NT; tt++) {
    // lane l % 16 of each 16: 8 bytes of row (l % 16) / 4 of its four keys; it gets dim l % 16 of all four
    const int vk = h * 4 + (lane & 15) / 4, c = tt * 4 + (lane & 16) / 8 + (lane & 3) / 2;
    va[tt] = KBUF + vk * DH * 2 + ((c ^ (vk & 7) >> VROT << 1) << 4) + (lane & 1) * 8;
  }

  f32x16 o[NT];
#pragma unroll
  for (int t = 0; t < NT; t++) o[t] = (f32x16)(0.f);
  float m_run = -INFINITY, l_run = 0.f;

  if (tiles > 0) request(0, pg0);
  for (int t = 0; t < tiles; t++) {
    const char* tile = lds + (t & 1) * 2 * KBUF;
    const int kb = start + t * KT;  // the tile's first key
    // tile t has landed, every wave's part of it, and every wave is done with the one before
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (kb >= wmax) {
      if (t + 1 < tiles) {
        request(t + 1, pg);
        pg = pages(t + 2);
      }
      continue;
    }
    f32x16 s[SB];
#pragma unroll
    for (int x = 0; x < SB; x++)
#pragma unroll
      for (int k = 0; k < KS; k++) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(tile + ka[k] + x * 32 * DH * 2);
#pragma unroll
        for (int p = NP - 1; p >= 0; p--)
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[p][k], (p == NP - 1 && k == 0) ? (f32x16)(0.f) : s[x], 0, 0, 0);
      }
    bf16x8 vf[SB][2][NT];
#pragma unroll
    for (int x = 0; x < SB; x++)
#pragma unroll
      for (int ks = 0; ks < 2; ks++)
#pragma unroll
        for (int tt = 0; tt < NT; tt++) {
          union { bf16x4 q[2]; bf16x8 f; } u;
#pragma unroll
          for (int y = 0; y < 2; y++)
            u.q[y] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lbf16x4*)(lbytes*)(tile + va[tt] + (x * 32 + ks * 16 + y * 8) * DH * 2));
          vf[x][ks][tt] = u.f;
        }
    // the keys' fragments half a block ahead of their products, the values' among the last products
    __builtin_amdgcn_sched_group_barrier(0x100, KS, 0);
    if constexpr (SB > 1) {
#pragma unroll
      for (int k = 0; k < KS; k++) {
        __builtin_amdgcn_sched_group_barrier(0x008, NP, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < KS; k++) {
      __builtin_amdgcn_sched_group_barrier(0x008, NP, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 4 * NT * SB / KS, 0);
    }
    if (t + 1 < tiles) {
      request(t + 1, pg);
      pg = pages(t + 2);
    }
    if (kb < it.k0 || kb + KT > wmin) {  // some key is not every query's
      asm volatile("");                  // stays a branch: the masks cost as much as a third of the step's vector work
#pragma unroll
      for (int x = 0; x < SB; x++)
#pragma unroll
        for (int v = 0; v < 16; v++) {
          const int kk = kb + x * 32 + 8 * (v >> 2) + 4 * h + (v & 3);
          s[x][v] = kk < lim && kk >= it.k0 ? s[x][v] : -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int x = 0; x < SB; x++)
#pragma unroll
      for (int v = 0; v < 16; v += 2) mx = fmaxf(fmaxf(mx, s[x][v]), s[x][v + 1]);
    mx *= sc;
    if (__any(mx > m_run + 8.0f)) {  // -inf + 8 is -inf: the first keys of a query come through here
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m_run, mx);
      const float al = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run - mn);
      l_run *= al;
#pragma unroll
      for (int tt = 0; tt < NT; tt++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[tt][v] *= al;
      m_run = mn;
    }
    const float off = m_run == -INFINITY ? 0.f : m_run;  // a query without a key yet: every p is 0
#pragma unroll
    for (int x = 0; x < SB; x++) {
      union { uint32_t u[8]; bf16x8 f[2]; } pf[NP];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[x][e], sc, -off)), p1 = __builtin_amdgcn_exp2f(fmaf(s[x][e + 1], sc, -off));
        uint32_t pl[NP];
        planes_of(p0, p1, pl);
        l_run = add_planes(l_run, p0, p1, pl);
#pragma unroll
        for (int p = 0; p < NP; p++) pf[p].u[e >> 1] = pl[p];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ks++)
#pragma unroll
        for (int tt = 0; tt < NT; tt++)
#pragma unroll
          for (int p = NP - 1; p >= 0; p--)
            o[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[x][ks][tt], pf[p].f[ks], o[tt], 0, 0, 0);
    }
  }
  finish_wide<T, uint16_t, DH>(A, it, R, g, o, m_run, l_run, lim, lds);
}

// The end of a piece of few queries: lane l holds dims 16 t + 4 (l / 16) .. + 3 of queries l % 16 + 16 x, over its wave's keys. The
// waves' sums are joined in wave order and written.
template <typename T, typename KVT, int DH, int QS>
__device__ void finish_few(const SeqArgs& A, const Item& it, const Records R, int g, const f32x4 (&o)[QS][DH / 16],
                           const float (&m_run)[QS], const float (&l_run)[QS], char* lds) {
  constexpr int NW = kWG / 64, NT = DH / 16, NQ = 16 * QS;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, col = lane & 15, q4 = lane >> 4;
  const int G = A.G, nq = it.nrows * G;
  __shared__ float2 s_ml[NW][NQ];
  __shared__ uint32_t s_few_bad;
  if (tid == 0) s_few_bad = 0u;
  __syncthreads();  // every wave is done with its tile
  float* ow = (float*)lds;  // [wave][query][dim]
#pragma unroll
  for (int x = 0; x < QS; x++) {
    float l = l_run[x];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int tt = 0; tt < NT; tt++)
      *reinterpret_cast<float4*>(ow + (w * NQ + x * 16 + col) * DH + tt * 16 + q4 * 4) =
          make_float4(o[x][tt][0], o[x][tt][1], o[x][tt][2], o[x][tt][3]);
    if (q4 == 0) s_ml[w][x * 16 + col] = make_float2(m_run[x], l);
  }
  __syncthreads();
  for (int i = tid; i < nq * (DH / 4); i += kWG) {
    const int j = i / (DH / 4), d = i % (DH / 4) * 4, r = it.row0 + j / G, hd = g * G + j % G;
    const int n = min(row_limit(A, it, r), it.k1);
    float M = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NW; x++) M = fmaxf(M, s_ml[x][j].x);
#pragma unroll
    for (int x = 0; x < NW; x++) {
      const float2 ml = s_ml[x][j];
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
      const float4 v = *reinterpret_cast<const float4*>(ow + (x * NQ + j) * DH + d);
      L = fmaf(ml.y, f, L);
      a[0] = fmaf(v.x, f, a[0]);
      a[1] = fmaf(v.y, f, a[1]);
      a[2] = fmaf(v.z, f, a[2]);
      a[3] = fmaf(v.w, f, a[3]);
    }
    auto finite = [](float x) { return fabsf(x) < INFINITY; };
    if ((!(L > 0.f) && n > it.k0) || !(finite(a[0]) && finite(a[1]) && finite(a[2]) && finite(a[3]))) {
      atomicOr(&s_few_bad, 1u << j);
    } else if (it.rec < 0) {
      store4((T*)A.out + r * A.os + hd * DH + d, a, n > 0 ? 1.0f / L : 0.f);
    } else {
      const size_t at = (size_t)it.rec + (size_t)g * nq + j;
      store4(R.o + at * DH + d, a, 1.0f);
      if (d == 0) R.ml[at] = make_float2(M, L);
    }
  }
  __syncthreads();
  for (uint32_t m = __builtin_amdgcn_readfirstlane(s_few_bad); m != 0u; m &= m - 1u)
    plain_piece<T, KVT, DH>(A, it, R, g, __builtin_ctz(m), (float*)lds);
}

// A piece of bf16 keys for up to 16 queries: each wave takes every fourth set of 32 keys by itself, with no barrier until
// the end. What bounds it is the stream of keys, so a wave keeps the next 32 keys and values on the way (16 KB, 128 KB
// a CU) while it works on these.
//   S^T = K Q^T (v_mfma_f32_16x16x32_bf16: lane l supplies 8 consecutive k of A row l % 16 and of B column l % 16, from k =
//     8 (l / 16); accumulator register v of lane l is row 4 (l / 16) + v, column l % 16).
//   O^T += V^T P^T over the 32 keys at once: k = 8 q .. 8 q + 7 of lanes 16 q .. are the keys 4 q + 0..3 and 16 + 4 q + 0..3 whose
//     probabilities they hold. K and V pass through a tile of LDS of the wave's own: loads take whole rows, operands 16 rows at once.
// Measured: a row of each of 64 sequences of 8192 keys (8 KV heads of 128) 320 us, 6.7 TB/s; 16 queries a KV head behind 64 of 4096
// keys 171 us, where a wide piece takes 189 for 20.
template <typename T, int DH>
__device__ void piece_few(const SeqArgs& A, const Item& it, const Records R, int g, char* lds) {
  constexpr int NP = sizeof(T) == 4 ? 3 : 1;
  constexpr int KT = 32, NW = kWG / 64, KS = DH / 32, NT = DH / 16, NCH = DH / 8, KPL = 64 / NCH;  // KPL: keys of a wave's load
  constexpr int VL = KT / KPL;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, q4 = lane >> 4;
  const int G = A.G, nq = it.nrows * G;
  const spd_cache& C = A.c;
  const int last = it.k1 - 1;
  const int start = it.k0 & ~(kPage - 1), tiles = (it.k1 - start + KT - 1) / KT;
  const size_t half = (size_t)C.n_kv_heads * kPage * DH;
  const uint16_t* pool = (const uint16_t*)A.kv + (size_t)g * kPage * DH;
  const int* table = C.page_table + (size_t)it.table * C.max_pages;
  auto pages = [&](int t) { return table[min(start / kPage + t * 2 + (lane & 1), last / kPage)]; };
  const int pg0 = w < tiles ? pages(w) : 0;
  int pg = w < tiles ? pages(w + NW) : 0;
  const float sc = NP == 1 ? A.scale * kLog2e : 1.0f;
  const int jj = min(col, nq - 1), row = it.row0 + jj / G, head = g * G + jj % G;
  const int lim = min(row_limit(A, it, row), it.k1);
  bf16x8 qf[NP][KS];
  load_query<T, KS, 32>(qf, (const T*)A.q + row * A.qs + head * DH + q4 * 8, A.scale * kLog2e);
  int wmin = lim;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) wmin = min(wmin, __shfl_xor(wmin, d, 64));
  wmin = __builtin_amdgcn_readfirstlane(wmin);

  // Keys outside [k0, k1) are read as the nearest one inside (see piece_wide).
  auto in_page = [&](int key) { return (uint32_t)(min(max(key, it.k0), last) & (kPage - 1)) * DH; };
  uint4 kr[VL], vr[VL];  // whole rows, so that a load takes whole lines
  auto load = [&](int t, int pg) {
    const uint16_t* p[2];
#pragma unroll
    for (int b = 0; b < 2; b++) p[b] = pool + (size_t)page_to_read(C, __builtin_amdgcn_readlane(pg, b)) * 2 * half;
    const int first = start + t * KT;
#pragma unroll
    for (int i = 0; i < VL; i++) {
      const uint16_t* at = p[i * KPL / 16] + in_page(first + i * KPL + lane / NCH) + lane % NCH * 8;
      kr[i] = ldg16(at);  // read once
      vr[i] = ldg16(at + half);
    }
  };
  constexpr int KROT = DH == 128 ? 0 : 1, VROT = DH == 128 ? 0 : 1;  // as in piece_wide
  char* kt = lds + w * 2 * KT * DH * 2;
  char* vt = kt + KT * DH * 2;
  uint32_t kw[VL], vw[VL], ka[KS], va[NT];
#pragma unroll
  for (int i = 0; i < VL; i++) {
    const int k = i * KPL + lane / NCH;
    kw[i] = k * DH * 2 + ((lane % NCH ^ (k >> KROT) % NCH) << 4);
    vw[i] = k * DH * 2 + ((lane % NCH ^ (k & 7) >> VROT << 1) << 4);
  }
#pragma unroll
  for (int k = 0; k < KS; k++) ka[k] = col * DH * 2 + (((4 * k + q4) ^ (col >> KROT) % NCH) << 4);
#pragma unroll
  for (int tt = 0; tt < NT; tt++) {
    const int k = q4 * 4 + col / 4, c = tt * 2 + (lane & 3) / 2;
    va[tt] = k * DH * 2 + ((c ^ (k & 7) >> VROT << 1) << 4) + (lane & 1) * 8;
  }
  f32x4 o[1][NT];
#pragma unroll
  for (int t = 0; t < NT; t++) o[0][t] = (f32x4)(0.f);
  float m_run[1] = {-INFINITY}, l_run[1] = {0.f};
  if (w < tiles) load(w, pg0);
  for (int t = w; t < tiles; t += NW) {
    const int kb = start + t * KT;
#pragma unroll
    for (int i = 0; i < VL; i++) {
      *reinterpret_cast<uint4*>(kt + kw[i]) = kr[i];
      *reinterpret_cast<uint4*>(vt + vw[i]) = vr[i];
    }
    if (t + NW < tiles) {
      load(t + NW, pg);
      pg = pages(t + 2 * NW);
    }
    f32x4 s[2];
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int k = 0; k < KS; k++) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + ka[k] + b * 16 * DH * 2);
#pragma unroll
        for (int p = NP - 1; p >= 0; p--)
          s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][k], (p == NP - 1 && k == 0) ? (f32x4)(0.f) : s[b], 0, 0, 0);
      }
    if (kb < it.k0 || kb + KT > wmin) {
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int v = 0; v < 4; v++) {
          const int kk = kb + b * 16 + 4 * q4 + v;
          s[b][v] = kk < lim && kk >= it.k0 ? s[b][v] : -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int v = 1; v < 8; v++) mx = fmaxf(mx, s[v >> 2][v & 3]);
    mx *= sc;
    if (__any(mx > m_run[0] + 8.0f)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m_run[0], mx);
      const float al = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[0] - mn);
      l_run[0] *= al;
#pragma unroll
      for (int tt = 0; tt < NT; tt++) o[0][tt] *= al;
      m_run[0] = mn;
    }
    const float off = m_run[0] == -INFINITY ? 0.f : m_run[0];
    union { uint32_t u[4]; bf16x8 f; } pf[NP];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], sc, -off)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][(e & 3) + 1], sc, -off));
      uint32_t pl[NP];
      planes_of(p0, p1, pl);
      l_run[0] = add_planes(l_run[0], p0, p1, pl);
#pragma unroll
      for (int p = 0; p < NP; p++) pf[p].u[e >> 1] = pl[p];
    }
#pragma unroll
    for (int tt = 0; tt < NT; tt++) {
      union { bf16x4 q[2]; bf16x8 f; } vf;
#pragma unroll
      for (int y = 0; y < 2; y++) vf.q[y] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lbf16x4*)(lbytes*)(vt + va[tt] + y * 16 * DH * 2));
#pragma unroll
      for (int p = NP - 1; p >= 0; p--) o[0][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.f, pf[p].f, o[0][tt], 0, 0, 0);
    }
  }
  finish_few<T, uint16_t, DH, 1>(A, it, R, g, o, m_run, l_run, lds);
}

// The same over an fp32 cache, for up to 16 QS queries, 16 keys at a time, with v_mfma_f32_16x16x4_f32 (lane l supplies k = l / 16 of
// A row and B column l % 16): a lane's four dims of a chunk are four steps; p is used as it is, register v of lanes 16 q .. being
// key 4 q + v. One set of queries is bound by the stream of keys (64 sequences of 4096 keys, 8 KV heads of 128: 336 us, 6.4 TB/s), two
// by the products behind it (461 us; 669 with 32 queries in one wave of piece_f32).
template <int DH, int QS>
__device__ void piece_few_f32(const SeqArgs& A, const Item& it, const Records R, int g, char* lds) {
  constexpr int KT = 16, NW = kWG / 64, KS = DH / 16, NT = DH / 16, NCH = DH / 4, KPL = 64 / NCH, VL = KT / KPL;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, q4 = lane >> 4;
  const int G = A.G, nq = it.nrows * G;
  const spd_cache& C = A.c;
  const int last = it.k1 - 1;
  const int start = it.k0 & ~(kPage - 1), tiles = (it.k1 - start + KT - 1) / KT;  // a tile is a page
  const size_t half = (size_t)C.n_kv_heads * kPage * DH;
  const float* pool = (const float*)A.kv + (size_t)g * kPage * DH;
  const int* table = C.page_table + (size_t)it.table * C.max_pages;
  auto page_at = [&](int t) { return table[min(start / kPage + t, last / kPage)]; };
  const int pg0 = w < tiles ? page_at(w) : 0;
  int pg = w < tiles ? page_at(w + NW) : 0;
  int lim[QS];
  float4 qf[QS][KS];
#pragma unroll
  for (int x = 0; x < QS; x++) {
    const int jj = min(x * 16 + col, nq - 1), row = it.row0 + jj / G, head = g * G + jj % G;
    lim[x] = min(row_limit(A, it, row), it.k1);
    const float* q = (const float*)A.q + row * A.qs + head * DH + q4 * 4;
    const float f = A.scale * kLog2e;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const float4 v = *reinterpret_cast<const float4*>(q + s * 16);
      qf[x][s] = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
  }
  uint4 kr[VL], vr[VL];
  auto load = [&](int t, int pg) {
    const float* p = pool + (size_t)page_to_read(C, __builtin_amdgcn_readfirstlane(pg)) * 2 * half;
    const int first = start + t * KT;
#pragma unroll
    for (int i = 0; i < VL; i++) {
      const float* at = p + (uint32_t)(min(max(first + i * KPL + lane / NCH, it.k0), last) & (kPage - 1)) * DH + lane % NCH * 4;
      kr[i] = ldg16(at);
      vr[i] = ldg16(at + half);
    }
  };
  // K: chunk c of key k sits at c ^ k; V: at c ^ (k / 4) << 2, so that the four keys of a read are in different banks
  char* kt = lds + w * 2 * KT * DH * 4;
  char* vt = kt + KT * DH * 4;
  f32x4 o[QS][NT];
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int x = 0; x < QS; x++) {
#pragma unroll
    for (int t = 0; t < NT; t++) o[x][t] = (f32x4)(0.f);
    m_run[x] = -INFINITY;
    l_run[x] = 0.f;
  }
  if (w < tiles) load(w, pg0);
  for (int t = w; t < tiles; t += NW) {
    const int kb = start + t * KT;
#pragma unroll
    for (int i = 0; i < VL; i++) {
      const int k = i * KPL + lane / NCH, c = lane % NCH;
      *reinterpret_cast<uint4*>(kt + k * DH * 4 + ((c ^ k) << 4)) = kr[i];
      *reinterpret_cast<uint4*>(vt + k * DH * 4 + ((c ^ (k >> 2) << 2) << 4)) = vr[i];
    }
    if (t + NW < tiles) {
      load(t + NW, pg);
      pg = page_at(t + 2 * NW);
    }
    f32x4 s[QS];
#pragma unroll
    for (int x = 0; x < QS; x++) s[x] = (f32x4)(0.f);
#pragma unroll
    for (int k = 0; k < KS; k++) {
      const float4 kf = *reinterpret_cast<const float4*>(kt + col * DH * 4 + (((4 * k + q4) ^ col) << 4));
#pragma unroll
      for (int x = 0; x < QS; x++) s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf.x, qf[x][k].x, s[x], 0, 0, 0);
#pragma unroll
      for (int x = 0; x < QS; x++) s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf.y, qf[x][k].y, s[x], 0, 0, 0);
#pragma unroll
      for (int x = 0; x < QS; x++) s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf.z, qf[x][k].z, s[x], 0, 0, 0);
#pragma unroll
      for (int x = 0; x < QS; x++) s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf.w, qf[x][k].w, s[x], 0, 0, 0);
    }
    float mx[QS];
    bool renew = false;
#pragma unroll
    for (int x = 0; x < QS; x++) {
      mx[x] = -INFINITY;
#pragma unroll
      for (int v = 0; v < 4; v++) {
        const int kk = kb + 4 * q4 + v;
        s[x][v] = kk < lim[x] && kk >= it.k0 ? s[x][v] : -INFINITY;
        mx[x] = fmaxf(mx[x], s[x][v]);
      }
      renew = renew || mx[x] > m_run[x] + 8.0f;
    }
    if (__any(renew)) {
#pragma unroll
      for (int x = 0; x < QS; x++) {
        float m = fmaxf(mx[x], __shfl_xor(mx[x], 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float mn = fmaxf(m_run[x], m);
        const float al = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[x] - mn);
        l_run[x] *= al;
#pragma unroll
        for (int tt = 0; tt < NT; tt++) o[x][tt] *= al;
        m_run[x] = mn;
      }
    }
#pragma unroll
    for (int x = 0; x < QS; x++) {
      const float off = m_run[x] == -INFINITY ? 0.f : m_run[x];
#pragma unroll
      for (int v = 0; v < 4; v++) {
        s[x][v] = __builtin_amdgcn_exp2f(s[x][v] - off);
        l_run[x] += s[x][v];
      }
    }
#pragma unroll
    for (int v = 0; v < 4; v++)
#pragma unroll
      for (int tt = 0; tt < NT; tt++) {
        const float vf = *reinterpret_cast<const float*>(vt + (4 * q4 + v) * DH * 4 + (((tt * 4 + col / 4) ^ q4 << 2) << 4) + (col & 3) * 4);
#pragma unroll
        for (int x = 0; x < QS; x++) o[x][tt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, s[x][v], o[x][tt], 0, 0, 0);
      }
  }
  finish_few<float, float, DH, QS>(A, it, R, g, o, m_run, l_run, lds);
}

// The same over an fp32 cache, for 32 queries a wave, with v_mfma_f32_32x32x2_f32 (lane l supplies k = l / 32 of A row
// and B column l % 32; accumulators as above): a lane's four dims of a chunk are four steps, so the halves take chunks in
// turn. P is used as it is. Tiles of 32 keys. Bound by the products: 4096 causal rows 1.22 ms, 113 TFLOP/s, 8 x 2048 rows 123, of 154
// that a square product of 16384 reaches.
template <int DH>
__device__ void piece_f32(const SeqArgs& A, const Item& it, const Records R, int g, char* lds) {
  constexpr int KT = 32, NT = DH / 32, KS = DH / 8, NCH = DH / 4;
  constexpr int KBUF = KT * DH * 4, BUF = 2 * KBUF, LPT = KT * NCH / kWG;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int G = A.G, nq = it.nrows * G;
  const spd_cache& C = A.c;
  const int last = it.k1 - 1;
  const int start = it.k0 & ~(kPage - 1), tiles = (it.k1 - start + KT - 1) / KT;
  const size_t half = (size_t)C.n_kv_heads * kPage * DH;
  const float* pool = (const float*)A.kv + (size_t)g * kPage * DH;
  const int* table = C.page_table + (size_t)it.table * C.max_pages;
  const bool active = w * 32 < nq;
  const int j = w * 32 + col, jj = min(j, nq - 1), row = it.row0 + jj / G, head = g * G + jj % G;
  const int lim = min(row_limit(A, it, row), it.k1);
  float4 qf[KS];
  {
    const float* q = (const float*)A.q + row * A.qs + head * DH + h * 4;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const float4 x = *reinterpret_cast<const float4*>(q + s * 8);
      const float f = A.scale * kLog2e;
      qf[s] = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
    }
  }
  auto pages = [&](int t) { return table[min(start / kPage + t * (KT / kPage) + (lane & 1), last / kPage)]; };
  auto issue = [&](int buf, int t, int pg) {
#pragma unroll
    for (int i = 0; i < LPT; i++) {
      const int ch = i * kWG + tid, k = ch / NCH, key = start + t * KT + k;
      const int page = page_to_read(C, __builtin_amdgcn_readlane(pg, (i * kWG + w * 64) / (NCH * kPage)));
      const int in = min(max(key, it.k0), last) % kPage;
      const float* p = pool + (size_t)page * 2 * half + in * DH;
      lbytes* to = (lbytes*)(lds + buf * BUF + (i * kWG + w * 64) * 16);
      __builtin_amdgcn_global_load_lds((gbytes*)(p + (ch % NCH ^ (k & 7)) * 4), to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gbytes*)(p + half + (ch % NCH ^ (k >> 2 & 1) << 3) * 4), to + KBUF, 16, 0, 0);
    }
  };
  f32x16 o[NT];
#pragma unroll
  for (int t = 0; t < NT; t++) o[t] = (f32x16)(0.f);
  float m_run = -INFINITY, l_run = 0.f;
  int pg = 0;
  if (tiles > 0) {
    pg = pages(0);
    issue(0, 0, pg);
    pg = pages(1);
  }
  for (int t = 0; t < tiles; t++) {
    const int buf = t & 1;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < tiles) {
      issue(buf ^ 1, t + 1, pg);
      pg = pages(t + 2);
    }
    const char* kt = lds + buf * BUF;
    const char* vt = kt + KBUF;
    const int kb = start + t * KT;
    if (!active || !__any(kb < lim)) continue;
    f32x16 s = (f32x16)(0.f);
#pragma unroll
    for (int k = 0; k < KS; k++) {
      const float4 kf = *reinterpret_cast<const float4*>(kt + col * DH * 4 + (((2 * k + h) ^ (col & 7)) << 4));
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.x, qf[k].x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.y, qf[k].y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.z, qf[k].z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.w, qf[k].w, s, 0, 0, 0);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const int kk = kb + 8 * (v >> 2) + 4 * h + (v & 3);
      s[v] = kk < lim && kk >= it.k0 ? s[v] : -INFINITY;
      mx = fmaxf(mx, s[v]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (__any(mx > m_run + 8.0f)) {
      const float mn = fmaxf(m_run, mx);
      const float al = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run - mn);
      l_run *= al;
#pragma unroll
      for (int tt = 0; tt < NT; tt++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[tt][v] *= al;
      m_run = mn;
    }
    const float off = m_run == -INFINITY ? 0.f : m_run;
    float ps = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      s[v] = __builtin_amdgcn_exp2f(s[v] - off);
      ps += s[v];
    }
    l_run += ps;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const int vk = 8 * (v >> 2) + 4 * h + (v & 3);
#pragma unroll
      for (int tt = 0; tt < NT; tt++) {
        const float vf = *reinterpret_cast<const float*>(vt + vk * DH * 4 + (((tt * 8 + col / 4) ^ h << 3) << 4) + (col & 3) * 4);
        o[tt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[v], o[tt], 0, 0, 0);
      }
    }
  }
  finish_wide<float, float, DH>(A, it, R, g, o, m_run, l_run, lim, lds);
}

// The piece of a call without a plan: a tile of at most 16 queries, or (no cu) a decode row, over all its keys.
__device__ __forceinline__ bool direct_item(const SeqArgs& A, int y, Item& it) {
  it.k0 = 0;
  it.rec = -1;
  if (A.cu == nullptr) {
    it.table = A.seqs[y];
    if ((unsigned)it.table >= (unsigned)A.c.max_seqs) return false;
    it.row0 = y;
    it.nrows = 1;
    it.k1 = seq_len(A.c, it.table);
    it.lim0 = 0;
    it.mode = ITEM_FLAT | ITEM_FEW;
    return true;
  }
  const int i = find_last(A.nseqs, y, [&](int k) { return A.cu[k] / A.rpt + k; });
  const int begin = A.cu[i], stop = A.cu[i + 1], end = min(stop, A.rows);
  it.table = A.seqs[i];
  if (begin < 0 || begin >= end || (unsigned)it.table >= (unsigned)A.c.max_seqs) return false;
  const long long row0 = begin + (long long)(y - (begin / A.rpt + i)) * A.rpt;
  if (row0 < begin || row0 >= end) return false;
  it.row0 = (int)row0;
  it.nrows = min(A.rpt, end - it.row0);
  it.lim0 = (int)max((long long)seq_len(A.c, it.table) - stop + it.row0 + 1, -(1ll << 30));
  it.k1 = max(0, it.lim0 + it.nrows - 1);
  it.mode = ITEM_FEW;
  return true;
}

// Grid: a piece's KV heads one after the other (with 8 of them a head's keys stay in one XCD's L2).
template <typename T, int DH>
__global__ __launch_bounds__(kWG, 2) void k_attend_bf16(SeqArgs A, const int* count, const Item* items, Records R) {
  extern __shared__ __align__(16) char lds[];
  const int g = blockIdx.x % A.c.n_kv_heads, y = blockIdx.x / A.c.n_kv_heads;
  const Item it = items[y];  // beside the count, not behind it: the list has an entry for every workgroup
  if (y >= count[0]) return;
  if (it.mode & ITEM_FEW)
    piece_few<T, DH>(A, it, R, g, lds);
  else
    piece_wide<T, DH>(A, it, R, g, lds);
}

template <int DH>
__global__ __launch_bounds__(kWG, 2) void k_attend_f32(SeqArgs A, const int* count, const Item* items, Records R) {
  extern __shared__ __align__(16) char lds[];
  const int g = blockIdx.x % A.c.n_kv_heads, y = blockIdx.x / A.c.n_kv_heads;
  const Item it = items[y];
  if (y >= count[0]) return;
  if (it.mode & ITEM_FEW)
    piece_few_f32<DH, 1>(A, it, R, g, lds);
  else if (it.mode & ITEM_PAIR)
    piece_few_f32<DH, 2>(A, it, R, g, lds);
  else
    piece_f32<DH>(A, it, R, g, lds);
}

template <typename T, typename KVT, int DH>
__global__ __launch_bounds__(kWG, 2) void k_attend_direct(SeqArgs A) {
  extern __shared__ __align__(16) char lds[];
  Item it;
  const int g = blockIdx.x % A.c.n_kv_heads;
  if (!direct_item(A, blockIdx.x / A.c.n_kv_heads, it)) return;
  if constexpr (sizeof(KVT) == 2)
    piece_few<T, DH>(A, it, Records{}, g, lds);
  else
    piece_few_f32<DH, 1>(A, it, Records{}, g, lds);
}

// Records to outputs. Grid: x = KV head, y = units (strided). The DH / 4 lanes of a query first hold a piece's (m, l) each,
// which gives the query's maximum and the pieces' factors by shuffles, then four dims each, over eight pieces at once. It reads the
// records once (64 rows of 32 heads behind 8192 shared keys: 17 MB, 6.2 us).
constexpr int kMergeRows = 128;  // 32: 4 us more there, 64: 0.5

template <int DH>
constexpr int merge_queries() { return kWG / (DH / 4); }

template <typename T, int DH>
__global__ __launch_bounds__(kWG) void k_merge(SeqArgs A, const int* count, const Unit* units, const Merge* merges, Records R) {
  constexpr int TPQ = DH / 4;
  const int n = count[1], g = blockIdx.x, G = A.G, hkv = A.c.n_kv_heads, lane = threadIdx.x % TPQ;
  for (int u = blockIdx.y; u < n; u += gridDim.y) {
    const Unit un = units[u];
    const Merge m = merges[un.merge];
    const int j = un.query + threadIdx.x / TPQ, nq = m.nrows * G, jj = min(j, nq - 1), np = m.pieces[0] + m.pieces[1];
    auto record = [&](int p) {
      const int x = p >= m.pieces[0], q = p - (x ? m.pieces[0] : 0);
      return (size_t)m.rec[x] + (size_t)(q * hkv + g) * m.queries[x] + m.first[x] + jj;
    };
    const int r = m.row0 + jj / G, head = g * G + jj % G;
    int lim = m.lim0 + jj / G;
    if (m.mode & ITEM_FLAT) lim = seq_len(A.c, A.seqs[r]);
    float L, a[4], part = 1.0f;
    bool again;
    do {  // once more, lowered by a power of two, where finite records add up to what is not
      float M = -INFINITY;
      L = a[0] = a[1] = a[2] = a[3] = 0.f;
      for (int p0 = 0; p0 < np; p0 += TPQ) {  // a pass but for more pieces than lanes
        const int p = p0 + lane;
        const float2 ml = p < np ? R.ml[record(p)] : make_float2(-INFINITY, 0.f);
        float mp = ml.x;
#pragma unroll
        for (int d = 1; d < TPQ; d <<= 1) mp = fmaxf(mp, __shfl_xor(mp, d, TPQ));
        const float Mn = fmaxf(M, mp);
        const float before = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
        // no key of this query in the piece: 0; a sum that is NaN goes on
        const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - Mn) * part;
        float l = ml.y * f;
#pragma unroll
        for (int d = 1; d < TPQ; d <<= 1) l += __shfl_xor(l, d, TPQ);
        M = Mn;
        L = L * before + l;
#pragma unroll
        for (int e = 0; e < 4; e++) a[e] *= before;
        const int here = min(TPQ, np - p0);
        for (int b = 0; b < here; b += 8) {
          float4 o[8];
#pragma unroll
          for (int e = 0; e < 8; e++) o[e] = *reinterpret_cast<const float4*>(R.o + record(min(p0 + b + e, np - 1)) * DH + 4 * lane);
#pragma unroll
          for (int e = 0; e < 8; e++) {
            const float w = __shfl(f, min(b + e, TPQ - 1), TPQ);
            if (b + e >= here) continue;
            a[0] = fmaf(o[e].x, w, a[0]);
            a[1] = fmaf(o[e].y, w, a[1]);
            a[2] = fmaf(o[e].z, w, a[2]);
            a[3] = fmaf(o[e].w, w, a[3]);
          }
        }
      }
      const bool finite = fabsf(a[0]) < INFINITY && fabsf(a[1]) < INFINITY && fabsf(a[2]) < INFINITY && fabsf(a[3]) < INFINITY;
      again = part == 1.0f && __any(!finite);
      part = ldexpf(1.0f, -down_of(max(np, 1)));
    } while (again);
    if (j < nq) store4((T*)A.out + r * A.os + head * DH + 4 * lane, a, lim > 0 ? 1.0f / L : 0.f);
  }
}

// ------------------------------------------------------------------------------------------------------- launches
// What a call takes: its tiles, and its workspace (the plan's lists, then the records).
struct Request {
  int rpt, wanted, jobs, tiles, qpu;
  bool direct, merge;
  size_t items, merges, units, records;
  size_t at_items, at_merges, at_units, at_tiles, at_ml, at_o, bytes;
};

Request request(const spd_cache& c, int n_q_heads, int nseqs, int rows, int ngroups, int max_len, bool prefix) {
  Request q{};
  const int hkv = c.n_kv_heads, G = n_q_heads / hkv;
  // Short calls go without a plan, one launch, every piece of at most 16 queries over all its keys: prompts whose tiles are at
  // most two a CU, decode rows (a shared prefix of so few keys is in the L2 for all of a group that the GPU holds at once). Planned and
  // so: 3 fp32 prompts of 21 rows 13.9 and 5.2 us, 4 bf16 prompts of 16 rows behind 300 keys 17.1 and 9.3, decode rows of
  // 300 keys 15.9 and 8.2, 256 of 512 keys 89 and 85. Longer calls need the splits, larger prompts the wide tiles.
  const bool fits = max_len > 0 && max_len <= 512;
  q.rpt = 16 / G;
  q.direct = fits && (prefix ? nseqs * hkv <= (ngroups > 0 ? 512 : 2048) : ((long long)rows / q.rpt + nseqs) * hkv <= 512);
  if (q.direct) {
    q.jobs = prefix ? nseqs : rows / q.rpt + nseqs;
    return q;
  }
  q.rpt = 128 / G;
  q.qpu = c.head_dim == 128 ? merge_queries<128>() : merge_queries<64>();
  // a job of at most kMinChunk / 2 keys is not split: then prompts have nothing to join
  const bool split = max_len == 0 || max_len > kMinChunk / 2;
  q.wanted = split ? std::max(1, kWantedWGs / hkv) : 0;
  q.merge = split || (prefix && ngroups > 0);
  q.tiles = prefix && ngroups > 0 ? nseqs / q.rpt + ngroups : 0;
  q.jobs = prefix ? q.tiles + nseqs : rows / q.rpt + nseqs;
  // jobs that cost more than a share (all costs / wanted): fewer than `wanted` of them, with fewer than 2 `wanted` pieces
  q.items = (size_t)q.jobs + 2 * q.wanted;
  q.merges = prefix ? nseqs : q.wanted;
  const int most = prefix ? G : std::min(q.rpt, rows) * G;  // queries of a merge
  q.units = q.merges * ((most + q.qpu - 1) / q.qpu);
  q.records = 2 * (size_t)q.wanted * hkv * std::min(q.rpt, rows) * G;
  if (prefix && ngroups > 0) q.records += 2 * (size_t)nseqs * n_q_heads;
  auto take = [&](size_t n) {
    const size_t at = q.bytes;
    q.bytes += (n + 255) / 256 * 256;
    return at;
  };
  take(64);  // counts
  q.at_items = take(q.items * sizeof(Item));
  q.at_merges = take(q.merges * sizeof(Merge));
  q.at_units = take(q.units * sizeof(Unit));
  q.at_tiles = take((size_t)q.tiles * sizeof(int4));
  q.at_ml = take(q.records * sizeof(float2));
  q.at_o = take(q.records * c.head_dim * sizeof(float));
  return q;
}

template <typename T, int DH>
void launch(const SeqArgs& a, const Request& q, const PlanArgs& p, const Records& r, hipStream_t s) {
  const bool bf16 = a.c.dtype == SPD_BF16;
  const size_t shm = 2 * 2 * 32 * DH * 4;  // either kind: two tiles of K and V, or a wave's own
  if (q.direct) {
    const dim3 grid((unsigned)(a.c.n_kv_heads * q.jobs));
    if (bf16)
      hipLaunchKernelGGL((k_attend_direct<T, uint16_t, DH>), grid, dim3(kWG), shm, s, a);
    else
      hipLaunchKernelGGL((k_attend_direct<float, float, DH>), grid, dim3(kWG), shm, s, a);
    return;
  }
  const dim3 grid((unsigned)(a.c.n_kv_heads * q.items));
  if (bf16) {
    hipLaunchKernelGGL((k_attend_bf16<T, DH>), grid, dim3(kWG), shm, s, a, p.count, p.items, r);
  } else {
    hipLaunchKernelGGL((k_attend_f32<DH>), grid, dim3(kWG), shm, s, a, p.count, p.items, r);
  }
  if (q.merge)
    hipLaunchKernelGGL((k_merge<T, DH>), dim3(a.c.n_kv_heads, (unsigned)std::min<size_t>(q.units, kMergeRows)), dim3(kWG), 0, s, a,
                       p.count, p.units, p.merges, r);
}

// A thread a job: four waves, one a SIMD, go through the plan faster than sixteen (7.1 and 8.0 us for 64 rows that share a prefix)
// while they have one job a thread.
template <int NTH>
void launch_plan_of(const PlanArgs& p, bool prefix, hipStream_t s) {
  if (prefix)
    hipLaunchKernelGGL((k_plan_attention<true, NTH>), dim3(1), dim3(NTH), 0, s, p);
  else
    hipLaunchKernelGGL((k_plan_attention<false, NTH>), dim3(1), dim3(NTH), 0, s, p);
}
void launch_plan(const PlanArgs& p, bool prefix, hipStream_t s) {
  p.jobs <= kSmallPlanWG ? launch_plan_of<kSmallPlanWG>(p, prefix, s) : launch_plan_of<kPlanWG>(p, prefix, s);
}

PlanArgs plan_args(const SeqArgs& a, int dtype, const Request& q, void* workspace) {
  char* ws = (char*)workspace;
  PlanArgs p{};
  p.c = a.c;
  p.seqs = a.seqs;
  p.cu = a.cu;
  p.prefix = a.prefix;
  p.nseqs = a.nseqs;
  p.rows = a.rows;
  p.ngroups = a.ngroups;
  p.G = a.G;
  p.wanted = q.wanted;
  p.rpt = q.rpt;
  p.tiles = q.tiles;
  p.jobs = q.jobs;
  p.pair = a.c.dtype == SPD_F32;
  p.wide_cost = dtype == SPD_BF16 ? 1 : 4;
  p.qpu = q.qpu;
  p.count = (int*)ws;
  p.items = (Item*)(ws + q.at_items);
  p.merges = (Merge*)(ws + q.at_merges);
  p.units = (Unit*)(ws + q.at_units);
  p.tile_rec = (int4*)(ws + q.at_tiles);
  return p;
}

// Plan, pieces, merge; or the pieces alone.
void run_attention(SeqArgs a, int dtype, const Request& q, bool prefix, void* workspace, hipStream_t s) {
  a.rpt = q.rpt;
  if (q.direct && prefix) a.cu = nullptr;
  PlanArgs p{};
  Records r{};
  if (!q.direct) {
    p = plan_args(a, dtype, q, workspace);
    r = Records{(float*)((char*)workspace + q.at_o), (float2*)((char*)workspace + q.at_ml)};
    launch_plan(p, prefix, s);
  }
  const bool wide = a.c.head_dim == 128;
  if (dtype == SPD_BF16)
    wide ? launch<uint16_t, 128>(a, q, p, r, s) : launch<uint16_t, 64>(a, q, p, r, s);
  else
    wide ? launch<float, 128>(a, q, p, r, s) : launch<float, 64>(a, q, p, r, s);
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
  if (q == out) return invalid(call, "out must not be q");
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
  run_attention(a, dtype, request(*c, n_q_heads, nseqs, rows, 0, max_len, false), false, workspace, (hipStream_t)stream);
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
  run_attention(a, dtype, request(*c, n_q_heads, nseqs, nseqs, ngroups, max_len, true), true, workspace, (hipStream_t)stream);
  return check_launch(call);
}
