// Rotary positions: frequencies, scaled for contexts longer than the trained one, and their tables of cosines and sines.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "spd_cache.h"
#include "spd_devfn.h"

namespace spd {
namespace {

constexpr int kMaxPairs = 128;
constexpr int kTableWGs = 4096;
constexpr double kTwoPi = 6.283185307179586476925;
constexpr double kPerQuarter = 0.6366197723675814, kPerQuarterLow = -3.935735335036497e-17;  // 2 / pi, the sum of both

// Quarter turns a position of each pair, as the sum of two doubles.
struct Turns {
  double hi[kMaxPairs], lo[kMaxPairs];
};

// cos and sin of u quarter turns, u in [-1/2, 1/2], each within 5e-12 of itself: polynomials of u^2 that were fitted to the least largest
// relative error. (Of fp32 they take 11 FMAs and two multiplications; Taylor's series 14 and three.)
__device__ __forceinline__ void cos_sin(double u, double& c, double& s) {
  const double v = u * u;
  double a = -2.485220715473308e-05, b = 0.00015819507016715984;
  a = fma(a, v, 0.0009191629220490869);
  b = fma(b, v, -0.0046812606257090415);
  a = fma(a, v, -0.020863468401264795);
  b = fma(b, v, 0.07969258184265056);
  a = fma(a, v, 0.2536695072116401);
  b = fma(b, v, -0.6459640961024081);
  a = fma(a, v, -1.2337005501235698);
  b = fma(b, v, 1.570796326787748);
  c = fma(a, v, 1.0);
  s = u * b;
}

// A thread has V pairs of every n-th position. The angle is the position times the frequency in quarter turns: its product, with the
// error that an FMA gives, loses its whole quarters exactly (1.5 2^52 leaves them in the sum's low bits), and what is left is right for
// any position. Both values are rounded once, from 64 bits. Some 20 fp64 instructions a pair take as long as its 8 bytes to memory:
// 131072 positions of 64 pairs, 67 MB, 15.4 us a launch into buffers in turn, 4.4 TB/s (a copy reaches 5.1), 13.7 into the same ones,
// which the last-level cache holds in part.
template <int V>
__global__ __launch_bounds__(kWG) void k_rope_table(Turns T, int pairs, long long first, int positions, double amplitude, float* cosines,
                                                    float* sines) {
  const int units = pairs / V, rows = kWG / units, j = (int)threadIdx.x % units * V;
  if ((int)threadIdx.x >= rows * units) return;
  double hi[V], lo[V];
#pragma unroll
  for (int e = 0; e < V; e++) {
    hi[e] = T.hi[j + e];
    lo[e] = T.lo[j + e];
  }
  for (long long row = (long long)blockIdx.x * rows + threadIdx.x / units; row < positions; row += (long long)gridDim.x * rows) {
    const double p = (double)(first + row);
    float c[V], s[V];
#pragma unroll
    for (int e = 0; e < V; e++) {
#pragma clang fp contract(off)  // `at` is the rounded product in all of its uses
      const double at = p * hi[e], big = at + 0x1.8p52;
      const double u = (at - (big - 0x1.8p52)) + fma(p, lo[e], fma(p, hi[e], -at));
      const uint32_t q = (uint32_t)__builtin_bit_cast(unsigned long long, big);  // its low two bits: the quarter
      double x, y;
      cos_sin(u, x, y);
      const float cu = (float)(x * amplitude), su = (float)(y * amplitude);
      c[e] = __uint_as_float(__float_as_uint(q & 1 ? su : cu) ^ ((q + 1) & 2) << 30);
      s[e] = __uint_as_float(__float_as_uint(q & 1 ? cu : su) ^ (q & 2) << 30);
    }
    const size_t to = (size_t)row * pairs + j;
    if constexpr (V == 4) {
      *reinterpret_cast<float4*>(cosines + to) = make_float4(c[0], c[1], c[2], c[3]);
      *reinterpret_cast<float4*>(sines + to) = make_float4(s[0], s[1], s[2], s[3]);
    } else {
      cosines[to] = c[0];
      sines[to] = s[0];
    }
  }
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" spd_status spd_rope_frequencies(int32_t dims, double base, const spd_rope_scaling* scaling, double* freq) {
  const char* call = "rope frequencies";
  if (!freq) return invalid(call, "NULL pointer");
  if (dims < 2 || dims % 2 || dims > 2 * kMaxPairs) return invalid(call, "dims must be even, in [2, 256]");
  if (!(base > 1.0) || !std::isfinite(base)) return invalid(call, "base must be finite and above 1");
  const int kind = scaling ? scaling->kind : SPD_ROPE_PLAIN;
  if (kind < SPD_ROPE_PLAIN || kind > SPD_ROPE_PARTS) return invalid(call, "no such scaling");
  const double f = kind != SPD_ROPE_PLAIN ? scaling->factor : 1.0;
  if (!(f > 0.0) || !std::isfinite(f)) return invalid(call, "factor must be finite and above 0");
  if (kind == SPD_ROPE_BASE && dims < 4) return invalid(call, "a changed base needs at least 4 dims");
  if (kind == SPD_ROPE_PARTS) {
    if (scaling->original < 1) return invalid(call, "original must be at least 1");
    if (!(scaling->low < scaling->high) || !std::isfinite(scaling->low) || !std::isfinite(scaling->high))
      return invalid(call, "low must be below high, both finite");
  }
  if (kind == SPD_ROPE_BASE) base *= std::pow(f, (double)dims / (dims - 2));
  if (!std::isnormal(base)) return invalid(call, "the changed base is no normal number");  // subnormal ones have fewer bits
  for (int i = 0; i < dims / 2; i++) {
    double t = std::pow(base, -2.0 * i / dims);
    if (kind == SPD_ROPE_LINEAR) t /= f;
    if (kind == SPD_ROPE_PARTS) {
      const double turns = scaling->original * t / kTwoPi;
      const double part = std::min(1.0, std::max(0.0, (turns - scaling->low) / (scaling->high - scaling->low)));
      t = (1.0 - part) * t / f + part * t;
    }
    if (!std::isfinite(t)) return invalid(call, "a frequency is not finite");
    freq[i] = t;
  }
  return SPD_OK;
}

extern "C" spd_status spd_rope_table(const double* freq, int32_t pairs, int64_t first, int32_t positions, double amplitude,
                                     float* cosines, float* sines, void* stream) {
  const char* call = "rope table";
  if (pairs < 1 || pairs > kMaxPairs) return invalid(call, "pairs must be in [1, 128]");
  if (positions < 0 || first < -(1ll << 30) || first > 1ll << 30) return invalid(call, "positions must not be negative, first within 2^30");
  if (!std::isfinite(amplitude)) return invalid(call, "amplitude must be finite");
  if (!freq) return invalid(call, "NULL pointer");
  Turns t{};
  for (int i = 0; i < pairs; i++) {
    if (!(std::fabs(freq[i]) <= 1e3)) return invalid(call, "a frequency is not finite, or above 1000");
    t.hi[i] = freq[i] * kPerQuarter;
    t.lo[i] = std::fma(freq[i], kPerQuarter, -t.hi[i]) + freq[i] * kPerQuarterLow;
  }
  if (positions == 0) return SPD_OK;
  if (!cosines || !sines || misaligned(cosines, 16) || misaligned(sines, 16)) return invalid(call, "NULL or misaligned pointer");
  const size_t bytes = (size_t)positions * pairs * sizeof(float);
  if ((uintptr_t)cosines < (uintptr_t)sines + bytes && (uintptr_t)sines < (uintptr_t)cosines + bytes)
    return invalid(call, "cosines and sines overlap");
  const bool fours = pairs % 4 == 0;
  const int rows = kWG / (fours ? pairs / 4 : pairs);
  const dim3 grid(std::min((positions - 1) / rows + 1, kTableWGs));
  hipStream_t st = (hipStream_t)stream;
  if (fours)
    hipLaunchKernelGGL((k_rope_table<4>), grid, dim3(kWG), 0, st, t, pairs, (long long)first, positions, amplitude, cosines, sines);
  else
    hipLaunchKernelGGL((k_rope_table<1>), grid, dim3(kWG), 0, st, t, pairs, (long long)first, positions, amplitude, cosines, sines);
  return check_launch(call);
}
