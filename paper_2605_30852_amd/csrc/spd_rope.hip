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
constexpr double kTwoPi = 6.283185307179586476925, kPerTurn = 0.15915494309189535, kPerTurnLow = -9.839338337591243e-18;

// Turns a position of each pair, as the sum of two doubles.
struct Turns {
  double hi[kMaxPairs], lo[kMaxPairs];
};

// cos and sin of `turns` turns in [-1/8, 1/8], the Taylor series of 2 pi times it, to 2^-37 of themselves.
__device__ __forceinline__ void cos_sin(double turns, double& c, double& s) {
  const double x = turns * kTwoPi, y = x * x;
  double a = 1.0 / 479001600, b = -1.0 / 39916800;
  a = fma(a, y, -1.0 / 3628800);
  b = fma(b, y, 1.0 / 362880);
  a = fma(a, y, 1.0 / 40320);
  b = fma(b, y, -1.0 / 5040);
  a = fma(a, y, -1.0 / 720);
  b = fma(b, y, 1.0 / 120);
  a = fma(a, y, 1.0 / 24);
  b = fma(b, y, -1.0 / 6);
  a = fma(a, y, -0.5);
  c = fma(a, y, 1.0);
  s = fma(x * y, b, x);
}

// A thread has V pairs of every n-th position. The angle is the position times the frequency in turns: its product, with the error
// that an FMA gives, loses its whole turns exactly, and what is left is right for any position. Both values are rounded once, from 64 bits.
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
#pragma clang fp contract(off)  // `at` is the rounded product in both of its uses
      const double at = p * hi[e];
      const double r = (at - rint(at)) + fma(p, lo[e], fma(p, hi[e], -at));
      const double quarter = rint(4.0 * r);
      double x, y;
      cos_sin(fma(quarter, -0.25, r), x, y);
      const int q = (int)quarter & 3;
      const double cc = q & 1 ? y : x, ss = q & 1 ? x : y;
      c[e] = (float)((q == 1 || q == 2 ? -cc : cc) * amplitude);
      s[e] = (float)((q & 2 ? -ss : ss) * amplitude);
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
  for (int i = 0; i < dims / 2; i++) {
    double t = std::pow(base, -2.0 * i / dims);
    if (kind == SPD_ROPE_LINEAR) t /= f;
    if (kind == SPD_ROPE_PARTS) {
      const double turns = scaling->original * t / kTwoPi;
      const double part = std::min(1.0, std::max(0.0, (turns - scaling->low) / (scaling->high - scaling->low)));
      t = (1.0 - part) * t / f + part * t;
    }
    freq[i] = t;
  }
  return SPD_OK;
}

extern "C" spd_status spd_rope_table(const double* freq, int32_t pairs, int64_t first, int32_t positions, double amplitude,
                                     float* cosines, float* sines, void* stream) {
  const char* call = "rope table";
  if (pairs < 1 || pairs > kMaxPairs) return invalid(call, "pairs must be in [1, 128]");
  if (positions < 0 || first < -(1ll << 40) || first > 1ll << 40) return invalid(call, "positions must not be negative, first within 2^40");
  if (!std::isfinite(amplitude)) return invalid(call, "amplitude must be finite");
  if (!freq) return invalid(call, "NULL pointer");
  Turns t{};
  for (int i = 0; i < pairs; i++) {
    if (!(std::fabs(freq[i]) <= 1e6)) return invalid(call, "a frequency is not finite, or above 1e6");
    t.hi[i] = freq[i] * kPerTurn;
    t.lo[i] = std::fma(freq[i], kPerTurn, -t.hi[i]) + freq[i] * kPerTurnLow;
  }
  if (positions == 0) return SPD_OK;
  if (!cosines || !sines || misaligned(cosines, 16) || misaligned(sines, 16)) return invalid(call, "NULL or misaligned pointer");
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
