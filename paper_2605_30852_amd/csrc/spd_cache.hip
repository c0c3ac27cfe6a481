// The pages of a cache of several sequences: growing (with copies of shared pages), forking, truncating and compacting
// them, and the rows that enter them.
//
// The state (table, lens, refs) lives on the device. Growing, compacting and large forks are two launches. The plan, one
// workgroup, checks the request and decides everything: a call that does not fit changes nothing. It works in tiles of
// entries or page ids with a prefix sum over the workgroup, so that pages are handed out in one fixed order, whatever
// the order in which waves run. Then many workgroups apply the plan: entries, counts (integer atomics, whose order
// does not show) and the copies of pages, which are what takes time: page bytes x layers, read and written once. A fork
// of few children is applied by the workgroup that checks it, and truncating needs no plan: every workgroup checks all of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "spd_cachefn.h"

namespace spd {

spd_status check_cache(const char* call, const spd_cache* c, bool pages) {
  if (!c) return invalid(call, "NULL cache");
  if (!c->kv || !c->page_table || !c->lens || (pages && !c->refs)) return invalid(call, "NULL pointer in the cache");
  if (misaligned(c->kv, 16)) return invalid(call, "kv must be 16-byte aligned");
  if (misaligned(c->page_table, 4) || misaligned(c->lens, 4) || misaligned(c->refs, 4))
    return invalid(call, "page_table, lens and refs must be 4-byte aligned");
  if (c->n_layers < 1 || c->num_pages < 1) return invalid(call, "n_layers and num_pages must be positive");
  if (c->max_seqs < 1 || c->max_seqs > kMaxSeqs) return invalid(call, "max_seqs must be in [1, 65536]");
  if (c->max_pages < 1 || c->max_pages > kMaxPages) return invalid(call, "max_pages must be in [1, 2^26]");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return invalid(call, "n_kv_heads must be in [1, 1024]");
  if (c->head_dim != 64 && c->head_dim != 128) return invalid(call, "head_dim must be 64 or 128");
  if (c->dtype != SPD_F32 && c->dtype != SPD_BF16) return invalid(call, "the cache's dtype must be SPD_F32 or SPD_BF16");
  return SPD_OK;
}

spd_status check_workspace(const char* call, const void* ws, size_t bytes, size_t need) {
  if (need == 0) return SPD_OK;
  if (!ws || misaligned(ws, 256)) return invalid(call, "workspace must be non-NULL and 256-byte aligned");
  if (bytes < need) {
    set_call_error(std::string(call) + ": workspace too small, " + std::to_string(need) + " bytes needed");
    return SPD_E_CAPACITY;
  }
  return SPD_OK;
}

spd_status check_rows(const char* call, const void* p, int64_t stride, int heads, int head_dim, int dtype) {
  const int64_t e = (int64_t)elem_bytes(dtype);
  if (!p) return invalid(call, "NULL pointer");
  if (misaligned(p, 16) || stride % (16 / e)) return invalid(call, "rows must be 16-byte aligned, strides multiples of 16 bytes");
  if (stride < (int64_t)heads * head_dim || stride > ((int64_t)1 << 40)) return invalid(call, "a row's stride is below its length (or past 2^40)");
  return SPD_OK;
}

spd_status check_launch(const char* call) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SPD_OK;
  set_call_error(std::string(call) + " launch: " + hipGetErrorString(e));
  return SPD_E_HIP;
}

namespace {

constexpr int kPlanWG = 1024, kPlanWaves = kPlanWG / 64, kSmallPlanWG = 256;
constexpr int kIdsPerWave = 16 * 64, kIdsPerTile = kPlanWaves * kIdsPerWave;  // page ids of a tile of a plan

// Workspace of a plan, in ints: the header, then what the call needs.
enum { PH_STATUS = 0, PH_MOVES = 1, PH_LIVE = 2, PH_INTS = 16 };
struct Plan {
  int* head;
  int *first, *begin, *want, *src;  // reserve: an entry's first page in `ids`, the logical pages it takes, the page it copies
  int* ids;                         // reserve: free pages; compact: holes
  int* late;                        // compact: held pages that move
  int* map;                         // compact: where page id goes
};

size_t reserve_ints(const spd_cache& c, int n) { return PH_INTS + 4 * (size_t)n + (size_t)c.num_pages; }
size_t compact_ints(const spd_cache& c) { return PH_INTS + 3 * (size_t)c.num_pages; }

Plan reserve_plan(int n, void* ws) {
  Plan p{};
  p.head = (int*)ws;
  p.first = p.head + PH_INTS;
  p.begin = p.first + n;
  p.want = p.begin + n;
  p.src = p.want + n;
  p.ids = p.src + n;
  return p;
}

Plan compact_plan(const spd_cache& c, void* ws) {
  Plan p{};
  p.head = (int*)ws;
  p.ids = p.head + PH_INTS;
  p.late = p.ids + c.num_pages;
  p.map = p.late + c.num_pages;
  return p;
}

__device__ __forceinline__ int pages_of(int keys) { return (keys + kPage - 1) / kPage; }

// Exclusive prefix sum of v over a workgroup of NW waves, and the total; sums: NW entries of LDS.
template <int NW = kPlanWaves>
__device__ __forceinline__ long long plan_scan(long long v, long long* sums, long long* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const long long x = (long long)wave_scan((unsigned long long)v);
  __syncthreads();  // the last tile's sums are read
  if (lane == 63) sums[w] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < NW; i++) {
    if (i < w) before += sums[i];
    all += sums[i];
  }
  *total = all;
  return before + x - v;
}

// Which sequences a call has named.
struct Named {
  uint32_t* bits;
  __device__ __forceinline__ void clear(int max_seqs) const {
    for (int i = threadIdx.x; i < (max_seqs + 31) / 32; i += blockDim.x) bits[i] = 0u;
  }
  __device__ __forceinline__ bool first(int s) const { return !(atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u); }
};

// A chain of loads and barriers, 7.6 us (7.2 at the shortest) for 64 sequences (16 page ids a thread and pass).
template <int NTH>
__global__ __launch_bounds__(NTH) void k_plan_reserve(spd_cache c, const int* seqs, const int* add, int n, int* status,
                                                          Plan P) {
  __shared__ uint32_t bits[kMaxSeqs / 32];
  __shared__ long long sums[NTH / 64];
  __shared__ int s_status;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, cap = kPage * c.max_pages;
  const Named named{bits};
  named.clear(c.max_seqs);
  if (tid == 0) s_status = SPD_CACHE_DONE;
  __syncthreads();
  long long total = 0;
  for (int i0 = 0; i0 < n; i0 += NTH) {
    const int i = i0 + tid;
    int bad = SPD_CACHE_DONE, need = 0;
    if (i < n) {
      const int s = seqs[i], a = add[i];
      if ((unsigned)s >= (unsigned)c.max_seqs || !named.first(s)) {
        bad = SPD_CACHE_BAD_SEQ;
      } else {
        const int len = c.lens[s];
        if (a < 0 || len < 0 || len > cap || a > cap - len) {
          bad = SPD_CACHE_BAD_LEN;
        } else {
          const int have = pages_of(len), want = pages_of(len + a);
          int src = -1;
          if (a > 0 && len % kPage) {
            const int last = c.page_table[(size_t)s * c.max_pages + have - 1];
            if ((unsigned)last < (unsigned)c.num_pages && c.refs[last] > 1) src = last;
          }
          const int begin = src >= 0 ? have - 1 : have;
          need = want - begin;
          P.begin[i] = begin;
          P.want[i] = want;
          P.src[i] = src;
        }
      }
    }
    if (bad) atomicMax(&s_status, bad);
    long long all;
    const long long at = total + plan_scan<NTH / 64>(need, sums, &all);
    if (i < n) P.first[i] = (int)min(at, (long long)c.num_pages);
    total += all;
  }
  __syncthreads();
  // the first `total` free pages: a wave takes 64 ids a load, 16 loads at once
  long long found = 0;
  if (s_status == SPD_CACHE_DONE && total <= c.num_pages) {
    for (long long t0 = 0; t0 < c.num_pages && found < total; t0 += NTH * 16) {
      const long long id0 = t0 + w * kIdsPerWave + lane;
      bool f[16];
#pragma unroll
      for (int k = 0; k < 16; k++) f[k] = id0 + k * 64 < c.num_pages && c.refs[id0 + k * 64] == 0;
      unsigned long long m[16];
      int mine = 0;
#pragma unroll
      for (int k = 0; k < 16; k++) {
        m[k] = __ballot(f[k]);
        mine += __popcll(m[k]);
      }
      long long all, at = found + plan_scan<NTH / 64>(lane == 0 ? mine : 0, sums, &all);
      at = __shfl(at, 0, 64);
#pragma unroll
      for (int k = 0; k < 16; k++) {
        const long long r = at + __popcll(m[k] & ((1ull << lane) - 1ull));
        if (f[k] && r < total) P.ids[r] = (int)(id0 + k * 64);
        at += __popcll(m[k]);
      }
      found += all;
    }
  }
  if (tid == 0) {
    const int st = s_status != SPD_CACHE_DONE ? s_status : found < total ? SPD_CACHE_NO_PAGES : SPD_CACHE_DONE;
    P.head[PH_STATUS] = st;
    *status = st;
  }
}

// A slice of a page, whose bytes are a multiple of 4096: four loads of a thread under way at once, past the caches (what is
// copied is read by none soon). 64 pages of 8 layers: 16.4 us with a page of 64 KB a workgroup, 21.5 us in slices through the caches, 11.3 us so.
constexpr int kSlice = 4 * kWG * 16;
__device__ __forceinline__ void copy_slice(char* dst, const char* src, size_t page_bytes, int slice) {
  uint4 v[4];
  const size_t b = (size_t)slice * kSlice + threadIdx.x * 16;
#pragma unroll
  for (int u = 0; u < 4; u++)
    if (b + (size_t)u * kWG * 16 < page_bytes) v[u] = ldg16(src + b + (size_t)u * kWG * 16);
#pragma unroll
  for (int u = 0; u < 4; u++)
    if (b + (size_t)u * kWG * 16 < page_bytes) stg16(dst + b + (size_t)u * kWG * 16, v[u]);
}

// Grid: x = entry, y = a slice of a layer's copy (strided); the entry's table and counts with y = 0.
__global__ __launch_bounds__(kWG) void k_apply_reserve(spd_cache c, const int* seqs, const int* add, Plan P, size_t page_bytes,
                                                       int slices) {
  if (P.head[PH_STATUS] != SPD_CACHE_DONE) return;
  const int i = blockIdx.x, s = seqs[i], begin = P.begin[i], want = P.want[i], src = P.src[i], first = P.first[i];
  if (src >= 0) {
    const size_t layer = page_bytes * c.num_pages;
    const int dst = P.ids[first];
    for (int x = blockIdx.y; x < c.n_layers * slices; x += gridDim.y) {
      char* base = (char*)c.kv + x / slices * layer;
      copy_slice(base + dst * page_bytes, base + src * page_bytes, page_bytes, x % slices);
    }
  }
  if (blockIdx.y != 0) return;
  for (int j = begin + threadIdx.x; j < want; j += kWG) {
    const int p = P.ids[first + j - begin];
    c.page_table[(size_t)s * c.max_pages + j] = p;
    c.refs[p] = 1;
  }
  if (threadIdx.x == 0) {
    if (src >= 0) atomicSub(&c.refs[src], 1);
    c.lens[s] += add[i];
  }
}

// Fork: sources are read as they were, so a child that is not empty refuses the call, and a source is no child of it unless
// it is empty.
__device__ __forceinline__ void check_fork(const spd_cache& c, const int* src, const int* dst, const int* keep, int n,
                                           const Named& named, int* s_status) {
  for (int i = threadIdx.x; i < n; i += kPlanWG) {
    const int s = src[i], d = dst[i], k = keep[i];
    int bad = SPD_CACHE_DONE;
    if ((unsigned)s >= (unsigned)c.max_seqs || (unsigned)d >= (unsigned)c.max_seqs || !named.first(d) || c.lens[d] != 0)
      bad = SPD_CACHE_BAD_SEQ;
    else if (k < 0 || k > c.lens[s] || k > kPage * c.max_pages)
      bad = SPD_CACHE_BAD_LEN;
    if (bad) atomicMax(s_status, bad);
  }
}

// Child i takes the pages of its source, `step` threads from `at` on.
__device__ __forceinline__ void fork_pages(const spd_cache& c, int s, int d, int keep, int at, int step) {
  const int n = pages_of(keep);
  const int* from = c.page_table + (size_t)s * c.max_pages;
  int* to = c.page_table + (size_t)d * c.max_pages;
#pragma unroll 4
  for (int j = at; j < n; j += step) {
    const int p = from[j];
    to[j] = p;
    if ((unsigned)p < (unsigned)c.num_pages) atomicAdd(&c.refs[p], 1);
  }
}

// SMALL: the same workgroup applies what it has checked, its 16 waves divided among the children; otherwise k_apply_fork does, a
// workgroup a child, a launch more. Fork and a truncate behind it, in one launch and in two, called (and replayed in a graph): 8 children
// of 130 pages 17.7 and 20.4 us (8.1 and 8.9), 64 of them 17.6 and 20.7 (14.5 and 10.5): one saves the host a launch where that bounds
// the calls. 128 of 90 pages 19.7 and 20.8 (20.1 and 12.8), 256 of 48 24.4 and 20.7 (25 and 15.6): two from 65 children on. Many long
// ones want a workgroup each: 16 of 2048 pages 20.1 and 20.4 (20.5 and 13.4); one or two have more threads in one: one of 12288 25.5 and 36.2
// (25 and 35.8). How long the children are only the device knows, so short ones in a wide table go in two as well: 64 of 16 pages,
// 2048 wide, 17.6 and 20.9 us (10.1 and 9.4).
constexpr int kSmallFork = 12288;  // entries of the children's tables
bool small_fork(const spd_cache& c, int n) { return n <= 2 || (n <= 64 && (size_t)n * c.max_pages <= kSmallFork); }

template <bool SMALL>
__global__ __launch_bounds__(kPlanWG) void k_plan_fork(spd_cache c, const int* src, const int* dst, const int* keep, int n,
                                                       int* status, int* head) {
  __shared__ uint32_t bits[kMaxSeqs / 32];
  __shared__ int s_status;
  const Named named{bits};
  named.clear(c.max_seqs);
  if (threadIdx.x == 0) s_status = SPD_CACHE_DONE;
  __syncthreads();
  check_fork(c, src, dst, keep, n, named, &s_status);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (!SMALL) head[PH_STATUS] = s_status;
    *status = s_status;
  }
  if (!SMALL || s_status != SPD_CACHE_DONE) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (n > kPlanWaves / 2) {  // a wave a child at a time
    for (int i = w; i < n; i += kPlanWaves) {
      const int d = dst[i], k = keep[i];
      fork_pages(c, src[i], d, k, lane, 64);
      if (lane == 0) c.lens[d] = k;
    }
  } else if (const int per = kPlanWaves / n; w < n * per) {  // several waves each
    const int i = w / per, d = dst[i], k = keep[i], at = (w - i * per) * 64 + lane;
    fork_pages(c, src[i], d, k, at, 64 * per);
    if (at == 0) c.lens[d] = k;
  }
}

// Grid: x = child.
__global__ __launch_bounds__(kWG) void k_apply_fork(spd_cache c, const int* src, const int* dst, const int* keep, const int* head) {
  if (head[PH_STATUS] != SPD_CACHE_DONE) return;
  const int i = blockIdx.x;
  fork_pages(c, src[i], dst[i], keep[i], threadIdx.x, kWG);
  if (threadIdx.x == 0) c.lens[dst[i]] = keep[i];
}

// Grid: x = sequence (strided). What refuses the call is in its arguments, which nothing changes, so every workgroup checks
// them all and no launch has to come before. That is n entries a workgroup, so there are at most kTruncateWGs of them: 4096
// sequences take 15.6, 13.7 and 19.3 us with 256, 512 and 1024, 65536 sequences 0.18 ms with 512 and 14 ms with one each.
constexpr int kTruncateWGs = 512;
__global__ __launch_bounds__(kWG) void k_truncate(spd_cache c, const int* seqs, const int* keep, int n, int* status) {
  __shared__ uint32_t bits[kMaxSeqs / 32];
  __shared__ int s_status;
  for (int i = threadIdx.x; i < (c.max_seqs + 31) / 32; i += kWG) bits[i] = 0u;
  if (threadIdx.x == 0) s_status = SPD_CACHE_DONE;
  __syncthreads();
  const Named named{bits};
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kWG) {
    const int s = seqs[i];
    const int bad = (unsigned)s >= (unsigned)c.max_seqs || !named.first(s) ? SPD_CACHE_BAD_SEQ : keep[i] < 0 ? SPD_CACHE_BAD_LEN : 0;
    if (bad) atomicMax(&s_status, bad);
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = s_status;
  if (s_status != SPD_CACHE_DONE) return;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = seqs[i], len = seq_len(c, s), k = min(keep[i], len), end = pages_of(len);
    int* row = c.page_table + (size_t)s * c.max_pages;
#pragma unroll 4
    for (int j = pages_of(k) + threadIdx.x; j < end; j += kWG) {
      const int p = row[j];
      row[j] = -1;
      if ((unsigned)p < (unsigned)c.num_pages) atomicSub(&c.refs[p], 1);
    }
    __syncthreads();  // every wave has read the length
    if (threadIdx.x == 0) c.lens[s] = k;
  }
}

// Held pages are counted (n), then those at n and above and the holes below n are listed, in order: as many of each. Two passes over
// refs, 14 us for 8192 pages, beside 120 us of copies.
__global__ __launch_bounds__(kPlanWG) void k_plan_compact(spd_cache c, int* live, Plan P) {
  __shared__ long long sums[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  long long n = 0;
  for (long long t0 = 0; t0 < c.num_pages; t0 += kIdsPerTile) {
    const long long id0 = t0 + w * kIdsPerWave + lane;
    int mine = 0;
#pragma unroll
    for (int k = 0; k < 16; k++) mine += id0 + k * 64 < c.num_pages && c.refs[id0 + k * 64] > 0;
    long long all;
    plan_scan(mine, sums, &all);
    n += all;
  }
  long long moves = 0;  // holes seen; late pages seen
  long long lates = 0;
  for (long long t0 = 0; t0 < c.num_pages; t0 += kIdsPerTile) {
    const long long id0 = t0 + w * kIdsPerWave + lane;
    bool hole[16], late[16];
#pragma unroll
    for (int k = 0; k < 16; k++) {
      const long long id = id0 + k * 64;
      const bool in = id < c.num_pages, held = in && c.refs[id] > 0;
      hole[k] = in && !held && id < n;
      late[k] = held && id >= n;
      if (in && !held && id >= n) P.map[id] = (int)id;
    }
    int h = 0, l = 0;
#pragma unroll
    for (int k = 0; k < 16; k++) {
      h += __popcll(__ballot(hole[k]));
      l += __popcll(__ballot(late[k]));
    }
    long long all;  // both counts in one sum: ids are below 2^31
    long long at = plan_scan(lane == 0 ? (long long)h << 32 | l : 0, sums, &all);
    at = __shfl(at, 0, 64);
    long long ah = moves + (at >> 32), al = lates + (at & 0xffffffffll);
#pragma unroll
    for (int k = 0; k < 16; k++) {
      const unsigned long long mh = __ballot(hole[k]), ml = __ballot(late[k]), below = (1ull << lane) - 1ull;
      if (hole[k]) P.ids[ah + __popcll(mh & below)] = (int)(id0 + k * 64);
      if (late[k]) P.late[al + __popcll(ml & below)] = (int)(id0 + k * 64);
      ah += __popcll(mh);
      al += __popcll(ml);
    }
    moves += all >> 32;
    lates += all & 0xffffffffll;
  }
  __syncthreads();  // the lists are whole
  for (long long k = tid; k < moves; k += kPlanWG) P.map[P.late[k]] = P.ids[k];
  if (tid == 0) {
    P.head[PH_MOVES] = (int)moves;
    P.head[PH_LIVE] = (int)n;
    *live = (int)n;
  }
}

// Sources are at n and above, destinations below: no copy reads what another writes. Bound by HBM, 5.3 TB/s read and written (the
// rate of a copy of 1 GiB is 5.2).
__global__ __launch_bounds__(kWG) void k_apply_compact(spd_cache c, Plan P, size_t page_bytes, int slices) {
  const int moves = P.head[PH_MOVES], n = P.head[PH_LIVE];
  const size_t layer = page_bytes * c.num_pages;
  const unsigned per_move = (unsigned)c.n_layers * slices;
  for (unsigned long long i = blockIdx.x; i < (unsigned long long)moves * per_move; i += gridDim.x) {
    const unsigned k = (unsigned)(i / per_move), x = (unsigned)(i % per_move), src = P.late[k], dst = P.ids[k];
    char* base = (char*)c.kv + x / slices * layer;
    copy_slice(base + dst * page_bytes, base + src * page_bytes, page_bytes, x % slices);
    if (x == 0 && threadIdx.x == 0) {
      c.refs[dst] = c.refs[src];
      c.refs[src] = 0;
    }
  }
  const size_t entries = (size_t)c.max_seqs * c.max_pages;
  for (size_t e = (size_t)blockIdx.x * kWG + threadIdx.x; e < entries; e += (size_t)gridDim.x * kWG) {
    const int p = c.page_table[e];
    if (p >= n && p < c.num_pages) c.page_table[e] = P.map[p];
  }
}

// ------------------------------------------------------------------------------------------------- new rows
struct AppendArgs {
  const void *k, *v, *q;
  void* qo;
  int64_t ks, vs, qs, qos;
  const float *cos, *sin;
  const int *seqs, *cu_rows;
  int layer, hq, nseqs, rows;
};

// A workgroup takes a row. A thread's unit is eight dims of a head and the eight that rotate with them, 16 bytes a load. Bound by HBM:
// fp32 rows of prompts into a bf16 cache, 273 MB, 54 us, 5 TB/s, and 45 us when the rows are those of the last call, part of which
// the caches keep; 64 single rows 4 us, a launch and four dependent loads.
template <typename T, typename KVT, int DH>
__global__ __launch_bounds__(kWG) void k_append(spd_cache c, AppendArgs A) {
  constexpr int H = DH / 2, UPH = H / 8;
  const int r = blockIdx.x;
  const RowAt at = row_at(c, A.seqs, A.cu_rows, A.nseqs, r);
  if (at.seq < 0 || at.key < 0) return;
  const int page = c.page_table[(size_t)at.seq * c.max_pages + at.key / kPage];
  const bool own = (unsigned)page < (unsigned)c.num_pages;
  const size_t half = (size_t)c.n_kv_heads * kPage * DH;  // a page's keys, then as many values
  KVT* base = (KVT*)c.kv + (((size_t)A.layer * c.num_pages + (own ? page : 0)) * 2) * half + (size_t)(at.key % kPage) * DH;
  const int nq = A.hq * UPH, nk = c.n_kv_heads * UPH;
  for (int u = threadIdx.x; u < nq + 2 * nk; u += kWG) {
    const int kind = u < nq ? 0 : u < nq + nk ? 1 : 2;
    const int x = u - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk), h = x / UPH, d = x % UPH * 8;
    const T* in = kind == 0 ? (const T*)A.q + r * A.qs : kind == 1 ? (const T*)A.k + r * A.ks : (const T*)A.v + r * A.vs;
    float a[8], b[8];
    load8(in + h * DH + d, a);
    load8(in + h * DH + H + d, b);
    if (A.cos != nullptr && kind < 2) {
      float cs[8], sn[8];
      load8(A.cos + (size_t)at.key * H + d, cs);
      load8(A.sin + (size_t)at.key * H + d, sn);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float ra = fmaf(a[e], cs[e], -(b[e] * sn[e])), rb = fmaf(b[e], cs[e], a[e] * sn[e]);
        a[e] = ra;
        b[e] = rb;
      }
    }
    if (kind == 0) {
      T* o = (T*)A.qo + r * A.qos + h * DH + d;
      store8(o, a);
      store8(o + H, b);
    } else if (own) {
      KVT* o = base + (kind == 2 ? half : 0) + (size_t)h * kPage * DH + d;
      store8(o, a);
      store8(o + H, b);
    }
  }
}

// The same with norms of the heads before the rotation, and rotations of other layouts. A unit is two chunks of eight dims: the
// rotation partners (half pairs), or two chunks that rotate within themselves (interleaved pairs) or not at all, behind the turned
// dims. The lanes of a head join their sums of squares by moves between lanes; each row is read and written once, and HBM bounds it: 5999
// fp32 rows of 48 heads into a bf16 cache, 272 MB, 55 us, 4.9 TB/s (66 where a lane's two chunks lie side by side); bf16 rows into a bf16
// cache, 149 MB, 29.8, 5.0 TB/s; 64 single rows 4.5 us, as k_append's.
struct HeadArgs : AppendArgs {
  const float *q_gain, *k_gain;
  float eps;
  int rot;
};

template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// Eight dims as four pairs.
__device__ __forceinline__ void turn_pairs(float (&x)[8], const float* cosines, const float* sines) {
  const float4 c = *reinterpret_cast<const float4*>(cosines), s = *reinterpret_cast<const float4*>(sines);
  const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const float a = x[2 * e], b = x[2 * e + 1];
    x[2 * e] = fmaf(a, cs[e], -(b * sn[e]));
    x[2 * e + 1] = fmaf(b, cs[e], a * sn[e]);
  }
}

template <typename T, typename KVT, int DH, bool PAIRS>
__global__ __launch_bounds__(kWG) void k_append_heads(spd_cache c, HeadArgs A) {
  constexpr int UPH = DH / 16;
  const int r = blockIdx.x;
  const RowAt at = row_at(c, A.seqs, A.cu_rows, A.nseqs, r);
  if (at.seq < 0 || at.key < 0) return;
  const int page = c.page_table[(size_t)at.seq * c.max_pages + at.key / kPage];
  const bool own = (unsigned)page < (unsigned)c.num_pages;
  const size_t half = (size_t)c.n_kv_heads * kPage * DH;  // a page's keys, then as many values
  KVT* base = (KVT*)c.kv + (((size_t)A.layer * c.num_pages + (own ? page : 0)) * 2) * half + (size_t)(at.key % kPage) * DH;
  const int nq = A.hq * UPH, nk = c.n_kv_heads * UPH, turned = A.rot / 8, reach = A.rot / 2;
  for (int u = threadIdx.x; u < nq + 2 * nk; u += kWG) {
    const int kind = u < nq ? 0 : u < nq + nk ? 1 : 2;
    const int x = u - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk), h = x / UPH, m = x % UPH;
    // Neighbouring lanes have neighbouring chunks: the halves of the turned dims, then those of the others (interleaved: of the head)
    const int mine = turned / 2;
    const bool halves = !PAIRS && m < mine;
    const int da = PAIRS || halves ? m * 8 : (m + mine) * 8, db = da + (PAIRS ? DH / 2 : halves ? reach : DH / 2 - reach);
    const T* in = (kind == 0 ? (const T*)A.q + r * A.qs : kind == 1 ? (const T*)A.k + r * A.ks : (const T*)A.v + r * A.vs) + h * DH;
    float a[8], b[8];
    load8(in + da, a);
    load8(in + db, b);
    const float* gain = kind == 0 ? A.q_gain : kind == 1 ? A.k_gain : nullptr;
    if (gain != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
      ss = lanes_sum<UPH>(ss);
      const float mean = ss * (1.0f / DH) + A.eps;
      float f = 1.0f / sqrtf(mean);
      if (!(mean > 0x1p-100f && mean < INFINITY)) {  // past fp32's range, or where squares are no normal numbers: the same, scaled
        const float by = mean > 1.0f ? 0x1p-70f : 0x1p60f;
        ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float y = a[e] * by, z = b[e] * by;
          ss = fmaf(y, y, fmaf(z, z, ss));
        }
        f = by / sqrtf(lanes_sum<UPH>(ss) * (1.0f / DH) + A.eps * by * by);
      }
      float ga[8], gb[8];
      load8(gain + da, ga);
      load8(gain + db, gb);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        a[e] = a[e] * f * ga[e];
        b[e] = b[e] * f * gb[e];
      }
    }
    const float *cosines = A.cos + (size_t)at.key * reach, *sines = A.sin + (size_t)at.key * reach;
    if constexpr (PAIRS) {
      if (kind < 2 && da < A.rot) turn_pairs(a, cosines + da / 2, sines + da / 2);
      if (kind < 2 && db < A.rot) turn_pairs(b, cosines + db / 2, sines + db / 2);
    } else if (kind < 2 && halves) {
      float cs[8], sn[8];
      load8(cosines + da, cs);
      load8(sines + da, sn);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float ra = fmaf(a[e], cs[e], -(b[e] * sn[e])), rb = fmaf(b[e], cs[e], a[e] * sn[e]);
        a[e] = ra;
        b[e] = rb;
      }
    }
    if (kind == 0) {
      T* o = (T*)A.qo + r * A.qos + h * DH;
      store8(o + da, a);
      store8(o + db, b);
    } else if (own) {
      KVT* o = base + (kind == 2 ? half : 0) + (size_t)h * kPage * DH;
      store8(o + da, a);
      store8(o + db, b);
    }
  }
}

template <typename T, typename KVT, int DH>
void launch_heads_of(const spd_cache& c, const HeadArgs& a, bool pairs, hipStream_t s) {
  if (pairs)
    hipLaunchKernelGGL((k_append_heads<T, KVT, DH, true>), dim3(a.rows), dim3(kWG), 0, s, c, a);
  else
    hipLaunchKernelGGL((k_append_heads<T, KVT, DH, false>), dim3(a.rows), dim3(kWG), 0, s, c, a);
}
template <typename T, typename KVT>
void launch_heads(const spd_cache& c, const HeadArgs& a, bool pairs, hipStream_t s) {
  c.head_dim == 128 ? launch_heads_of<T, KVT, 128>(c, a, pairs, s) : launch_heads_of<T, KVT, 64>(c, a, pairs, s);
}

template <typename T, typename KVT>
void launch_append(const spd_cache& c, const AppendArgs& a, hipStream_t s) {
  if (c.head_dim == 128)
    hipLaunchKernelGGL((k_append<T, KVT, 128>), dim3(a.rows), dim3(kWG), 0, s, c, a);
  else
    hipLaunchKernelGGL((k_append<T, KVT, 64>), dim3(a.rows), dim3(kWG), 0, s, c, a);
}

size_t page_bytes_of(const spd_cache& c) { return (size_t)2 * c.n_kv_heads * kPage * c.head_dim * elem_bytes(c.dtype); }

int slices_of(const spd_cache& c) { return (int)((page_bytes_of(c) + kSlice - 1) / kSlice); }
constexpr int kCopyWGs = 4096;

// The checks that reserve, fork, truncate and compact share.
spd_status check_change(const char* call, const spd_cache* c, std::initializer_list<const void*> arrays, int n) {
  const spd_status st = check_cache(call, c, true);
  if (st != SPD_OK) return st;
  for (const void* p : arrays)
    if (!p || misaligned(p, 4)) return invalid(call, "NULL or misaligned pointer");
  if (n < 1 || n > c->max_seqs) return invalid(call, "n must be in [1, max_seqs]");
  return SPD_OK;
}

// What both appends check but for the rotation.
spd_status check_append(const char* call, const spd_cache* c, int32_t layer, const void* k, int64_t k_stride, const void* v,
                        int64_t v_stride, const void* q, int64_t q_stride, const void* q_out, int64_t q_out_stride,
                        int32_t n_q_heads, int32_t dtype, const int32_t* seqs, const int32_t* cu_rows, int32_t nseqs, int32_t rows) {
  spd_status st = check_cache(call, c, false);
  if (st != SPD_OK) return st;
  if (dtype != SPD_F32 && dtype != SPD_BF16) return invalid(call, "dtype must be SPD_F32 or SPD_BF16");
  if (layer < 0 || layer >= c->n_layers) return invalid(call, "no such layer");
  if (!seqs || !cu_rows || misaligned(seqs, 4) || misaligned(cu_rows, 4)) return invalid(call, "NULL or misaligned pointer");
  if (nseqs < 1 || nseqs > c->max_seqs) return invalid(call, "nseqs must be in [1, max_seqs]");
  if (rows < 0 || rows >= 1 << 24) return invalid(call, "rows must be in [0, 2^24)");
  if ((st = check_rows(call, k, k_stride, c->n_kv_heads, c->head_dim, dtype)) != SPD_OK) return st;
  if ((st = check_rows(call, v, v_stride, c->n_kv_heads, c->head_dim, dtype)) != SPD_OK) return st;
  if (n_q_heads < 0 || n_q_heads > 16384 || (n_q_heads == 0) != (q == nullptr) || (q == nullptr) != (q_out == nullptr))
    return invalid(call, "q and q_out come with n_q_heads in [1, 16384], or are NULL with n_q_heads 0");
  if (q) {
    if ((st = check_rows(call, q, q_stride, n_q_heads, c->head_dim, dtype)) != SPD_OK) return st;
    if ((st = check_rows(call, q_out, q_out_stride, n_q_heads, c->head_dim, dtype)) != SPD_OK) return st;
  }
  return SPD_OK;
}

spd_status check_rope(const char* call, const spd_cache* c, const float* rope_cos, const float* rope_sin, int32_t rope_positions) {
  if ((rope_cos == nullptr) != (rope_sin == nullptr)) return invalid(call, "cos and sin come together");
  if (misaligned(rope_cos, 16) || misaligned(rope_sin, 16)) return invalid(call, "cos and sin must be 16-byte aligned");
  if (rope_cos ? rope_positions < kPage * c->max_pages : rope_positions != 0)
    return invalid(call, "rope_positions must be at least 16 * max_pages (0 without cos and sin)");
  return SPD_OK;
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" spd_status spd_cache_workspace(const spd_cache* c, int32_t n, size_t* bytes) {
  const spd_status st = check_cache("cache workspace", c, false);
  if (st != SPD_OK) return st;
  if (!bytes || n < 1 || n > c->max_seqs) return invalid("cache workspace", "NULL pointer, or n outside [1, max_seqs]");
  *bytes = (std::max(reserve_ints(*c, n), compact_ints(*c)) * sizeof(int) + 255) / 256 * 256;
  return SPD_OK;
}

extern "C" spd_status spd_cache_reserve(const spd_cache* c, const int32_t* seqs, const int32_t* add, int32_t n, int32_t* status,
                                        void* workspace, size_t ws_bytes, void* stream) {
  spd_status st = check_change("cache reserve", c, {seqs, add, status}, n);
  if (st == SPD_OK) st = check_workspace("cache reserve", workspace, ws_bytes, reserve_ints(*c, n) * sizeof(int));
  if (st != SPD_OK) return st;
  const Plan p = reserve_plan(n, workspace);
  hipStream_t s = (hipStream_t)stream;
  if (n <= kSmallPlanWG && c->num_pages <= 16 * kSmallPlanWG)  // one entry a thread, one tile of page ids: 7.6 us instead of 9.4
    hipLaunchKernelGGL(k_plan_reserve<kSmallPlanWG>, dim3(1), dim3(kSmallPlanWG), 0, s, *c, seqs, add, n, status, p);
  else
    hipLaunchKernelGGL(k_plan_reserve<kPlanWG>, dim3(1), dim3(kPlanWG), 0, s, *c, seqs, add, n, status, p);
  hipLaunchKernelGGL(k_apply_reserve, dim3(n, std::min(c->n_layers * slices_of(*c), std::max(1, kCopyWGs / n))), dim3(kWG), 0, s, *c,
                     seqs, add, p, page_bytes_of(*c), slices_of(*c));
  return check_launch("cache reserve");
}

extern "C" spd_status spd_cache_fork(const spd_cache* c, const int32_t* src, const int32_t* dst, const int32_t* keep, int32_t n,
                                     int32_t* status, void* workspace, size_t ws_bytes, void* stream) {
  spd_status st = check_change("cache fork", c, {src, dst, keep, status}, n);
  if (st == SPD_OK) st = check_workspace("cache fork", workspace, ws_bytes, PH_INTS * sizeof(int));
  if (st != SPD_OK) return st;
  int* head = (int*)workspace;
  hipStream_t s = (hipStream_t)stream;
  if (small_fork(*c, n)) {
    hipLaunchKernelGGL(k_plan_fork<true>, dim3(1), dim3(kPlanWG), 0, s, *c, src, dst, keep, n, status, head);
  } else {
    hipLaunchKernelGGL(k_plan_fork<false>, dim3(1), dim3(kPlanWG), 0, s, *c, src, dst, keep, n, status, head);
    hipLaunchKernelGGL(k_apply_fork, dim3(n), dim3(kWG), 0, s, *c, src, dst, keep, head);
  }
  return check_launch("cache fork");
}

extern "C" spd_status spd_cache_truncate(const spd_cache* c, const int32_t* seqs, const int32_t* keep, int32_t n,
                                         int32_t* status, void*, size_t, void* stream) {
  const spd_status st = check_change("cache truncate", c, {seqs, keep, status}, n);
  if (st != SPD_OK) return st;
  hipLaunchKernelGGL(k_truncate, dim3(std::min(n, kTruncateWGs)), dim3(kWG), 0, (hipStream_t)stream, *c, seqs, keep, n, status);
  return check_launch("cache truncate");
}

extern "C" spd_status spd_cache_compact(const spd_cache* c, int32_t* live, void* workspace, size_t ws_bytes, void* stream) {
  spd_status st = check_change("cache compact", c, {live}, 1);
  if (st == SPD_OK) st = check_workspace("cache compact", workspace, ws_bytes, compact_ints(*c) * sizeof(int));
  if (st != SPD_OK) return st;
  const Plan p = compact_plan(*c, workspace);
  hipStream_t s = (hipStream_t)stream;
  hipLaunchKernelGGL(k_plan_compact, dim3(1), dim3(kPlanWG), 0, s, *c, live, p);
  hipLaunchKernelGGL(k_apply_compact, dim3(kCopyWGs), dim3(kWG), 0, s, *c, p, page_bytes_of(*c), slices_of(*c));
  return check_launch("cache compact");
}

extern "C" spd_status spd_cache_append(const spd_cache* c, int32_t layer, const void* k, int64_t k_stride, const void* v,
                                       int64_t v_stride, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                                       int32_t n_q_heads, int32_t dtype, const float* rope_cos, const float* rope_sin,
                                       int32_t rope_positions, const int32_t* seqs, const int32_t* cu_rows, int32_t nseqs,
                                       int32_t rows, void* stream) {
  const char* call = "cache append";
  spd_status st = check_append(call, c, layer, k, k_stride, v, v_stride, q, q_stride, q_out, q_out_stride, n_q_heads, dtype, seqs,
                               cu_rows, nseqs, rows);
  if (st == SPD_OK) st = check_rope(call, c, rope_cos, rope_sin, rope_positions);
  if (st != SPD_OK) return st;
  if (rows == 0) return SPD_OK;
  if (q && q == q_out && q_stride != q_out_stride && rows > 1) return invalid(call, "q_out may be q with the same stride only");
  const AppendArgs a{k, v, q, q_out, k_stride, v_stride, q_stride, q_out_stride, rope_cos, rope_sin, seqs, cu_rows, layer,
                     n_q_heads, nseqs, rows};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == SPD_BF16)
    c->dtype == SPD_BF16 ? launch_append<uint16_t, uint16_t>(*c, a, s) : launch_append<uint16_t, float>(*c, a, s);
  else
    c->dtype == SPD_BF16 ? launch_append<float, uint16_t>(*c, a, s) : launch_append<float, float>(*c, a, s);
  return check_launch(call);
}

extern "C" spd_status spd_cache_append_heads(const spd_cache* c, int32_t layer, const void* k, int64_t k_stride, const void* v,
                                             int64_t v_stride, const void* q, int64_t q_stride, void* q_out,
                                             int64_t q_out_stride, int32_t n_q_heads, int32_t dtype, const spd_head_rule* rule,
                                             const float* rope_cos, const float* rope_sin, int32_t rope_positions,
                                             const int32_t* seqs, const int32_t* cu_rows, int32_t nseqs, int32_t rows,
                                             void* stream) {
  const char* call = "cache append of heads";
  spd_status st = check_append(call, c, layer, k, k_stride, v, v_stride, q, q_stride, q_out, q_out_stride, n_q_heads, dtype, seqs,
                               cu_rows, nseqs, rows);
  if (st == SPD_OK) st = check_rope(call, c, rope_cos, rope_sin, rope_positions);
  if (st != SPD_OK) return st;
  if (!rule) return invalid(call, "NULL rule");
  if (misaligned(rule->q_gain, 16) || misaligned(rule->k_gain, 16)) return invalid(call, "gains must be 16-byte aligned");
  if (rule->q_gain && !q) return invalid(call, "a gain of queries without queries");
  if ((rule->q_gain || rule->k_gain) && !(rule->eps > 0.f && std::isfinite(rule->eps))) return invalid(call, "eps must be finite and above 0");
  if (rule->rot < 0 || rule->rot % 16 || rule->rot > c->head_dim || (rule->rot > 0) != (rope_cos != nullptr))
    return invalid(call, "rot must be a multiple of 16 up to head_dim with cos and sin, 0 without");
  if (rule->interleaved != 0 && rule->interleaved != 1) return invalid(call, "interleaved must be 0 or 1");
  if (rows == 0) return SPD_OK;
  if (q && q == q_out && q_stride != q_out_stride && rows > 1) return invalid(call, "q_out may be q with the same stride only");
  const HeadArgs a{AppendArgs{k, v, q, q_out, k_stride, v_stride, q_stride, q_out_stride, rope_cos, rope_sin, seqs, cu_rows, layer,
                              n_q_heads, nseqs, rows},
                   rule->q_gain, rule->k_gain, rule->eps, rule->rot};
  const bool pairs = rule->interleaved != 0;
  hipStream_t s = (hipStream_t)stream;
  if (dtype == SPD_BF16)
    c->dtype == SPD_BF16 ? launch_heads<uint16_t, uint16_t>(*c, a, pairs, s) : launch_heads<uint16_t, float>(*c, a, pairs, s);
  else
    c->dtype == SPD_BF16 ? launch_heads<float, uint16_t>(*c, a, pairs, s) : launch_heads<float, float>(*c, a, pairs, s);
  return check_launch(call);
}
