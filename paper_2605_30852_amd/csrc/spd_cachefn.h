// Device helpers of the calls on a spd_cache: which sequence a packed row belongs to, the key it stands for, and
// pages read from a table that only the device knows.
#pragma once
#include "spd_cache.h"
#include "spd_devfn.h"

namespace spd {

// Last i in [0, n) with at(i) <= r, for at that ascends from at(0) <= r; by a whole wave, 64 probes a round (two rounds
// up to 4096 entries, where a binary search waits for twelve loads one after the other).
template <typename F>
__device__ __forceinline__ int find_last(int n, int r, F at) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool le = lane * step < n && at(lo + lane * step) <= r;
    const int k = max(__popcll(__ballot(le)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int seq_len(const spd_cache& c, int s) { return min(max(c.lens[s], 0), kPage * c.max_pages); }

// The sequence of a packed row and the key it stands for; seq < 0: the row belongs to none. key < 0: before the first.
struct RowAt {
  int seq, key;
};

__device__ __forceinline__ RowAt row_at(const spd_cache& c, const int* seqs, const int* cu_rows, int nseqs, int r) {
  const int i = find_last(nseqs, r, [&](int k) { return cu_rows[k]; });
  const int begin = cu_rows[i], end = cu_rows[i + 1], s = seqs[i];
  RowAt a{-1, -1};
  if (begin > r || r >= end || begin < 0 || (unsigned)s >= (unsigned)c.max_seqs) return a;
  a.seq = s;
  const int len = seq_len(c, s);
  a.key = end - r <= len ? len - (end - r) : -1;
  return a;
}

// A page to read: an id that is none becomes page 0.
__device__ __forceinline__ int page_to_read(const spd_cache& c, int id) { return (unsigned)id < (unsigned)c.num_pages ? id : 0; }

// A lane's value plus those of the lanes before it, and the largest of a wave in lane 63, by moves between lanes that do not go
// through LDS: 64 bits in six steps take about 0.1 us, shuffles 0.5.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long dpp64(unsigned long long x) {  // 0 where no lane is the source
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return (unsigned long long)(uint32_t)hi << 32 | (uint32_t)lo;
}
__device__ __forceinline__ unsigned long long wave_scan(unsigned long long x) {
  x += dpp64<0x111, 0xf>(x);  // one lane on in a row of 16, then two, four, eight
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);  // the last lane of rows 0 and 2 to rows 1 and 3
  x += dpp64<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ unsigned long long wave_top(unsigned long long x) {
  x = max(x, dpp64<0x111, 0xf>(x));
  x = max(x, dpp64<0x112, 0xf>(x));
  x = max(x, dpp64<0x114, 0xf>(x));
  x = max(x, dpp64<0x118, 0xf>(x));
  x = max(x, dpp64<0x142, 0xa>(x));
  return max(x, dpp64<0x143, 0xc>(x));
}

// Two fp32 values as bf16, to nearest even; infinities and NaN stay what they are.
typedef float fp32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(fp32x2{a, b}, bf16x2));
}

// 16-byte store past the caches.
__device__ __forceinline__ void stg16(void* p, const uint4& u) {
  const v4u v = {u.x, u.y, u.z, u.w};
  __builtin_nontemporal_store(v, (__attribute__((address_space(1))) v4u*)(p));
}

// Eight elements (16-byte aligned) as floats, and back.
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&f)[8]) {
  unpack16<uint16_t>(*reinterpret_cast<const uint4*>(p), f);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; i++) u[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

}  // namespace spd
