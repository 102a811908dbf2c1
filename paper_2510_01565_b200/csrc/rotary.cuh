// Rotary positions: channel pairs of every head turned by angles that grow with the row's position,
//   (a, b) -> magnitude * (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair
// Pairs are neighbours (interleaved) or half the rotated part apart.  Angles are products of up to 2^31 with a frequency, so they are taken
// in 64 bits, as turns, and only their fraction is narrowed.
#pragma once
#include "block_quant.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

constexpr int kRotaryMaxPairs = 128;
constexpr int kRotaryRows = 4;                 // rows per CTA at most
constexpr int kRotaryThreads = 256;

struct RotaryParams {
  const void* x;
  void* out;
  long long ld_x, ld_out;
  long long rows;
  const int* positions;      // [rows], or NULL: by the batch
  int n_heads, head_dim, pairs, interleaved, inverse;
  int rows_per_cta;
  float magnitude;
  int n;                     // requests
  int cu[DIT_MAX_REQUESTS + 1];
  int first[DIT_MAX_REQUESTS];
  double turns[kRotaryMaxPairs];               // frequency / (2 pi)
};

template <int kType>
__device__ __forceinline__ typename QuantIn<kType>::Elem narrow(float v) {
  if constexpr (kType == 2) return v;
  else if constexpr (kType == 1) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
  else return __half_as_ushort(__float2half_rn(v));
}
template <int kType>
__device__ __forceinline__ uint4 narrow16(const float (&v)[QuantIn<kType>::EPL]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kType == 2) w[i] = __float_as_uint(v[i]);
    else w[i] = static_cast<uint32_t>(narrow<kType>(v[2 * i])) | static_cast<uint32_t>(narrow<kType>(v[2 * i + 1])) << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A CTA takes a few rows: it computes their cosines and sines once, for all heads, and then walks (row, head, unit), a unit being the
// channels that one lane reads, 16 bytes and, where pairs are apart, the 16 bytes of their partners; channels behind the rotated
// part are copied (not at all in place).  Bound by HBM, each element read and written once.
// kVec: rows, heads and halves start on 16-byte boundaries; otherwise a unit is a pair.
template <int kType, bool kVec>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_kernel(const __grid_constant__ RotaryParams p) {
  using In = QuantIn<kType>;
  using Elem = typename In::Elem;
  constexpr int EPL = In::EPL;
  __shared__ float2 cs[kRotaryRows][kRotaryMaxPairs];
  const long long row0 = static_cast<long long>(blockIdx.x) * p.rows_per_cta;
  const int n_rows = static_cast<int>(min(static_cast<long long>(p.rows_per_cta), p.rows - row0));
  for (int i = threadIdx.x; i < n_rows * p.pairs; i += kRotaryThreads) {
    const int r = i / p.pairs, f = i - r * p.pairs;
    const long long row = row0 + r;
    int position;
    if (p.positions) {
      position = __ldg(p.positions + row);
    } else {
      int lo = 0, hi = p.n - 1;                // the row's request: the last one that begins at or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.cu[mid] <= row) lo = mid; else hi = mid - 1;
      }
      position = p.first[lo] + static_cast<int>(row - p.cu[lo]);
    }
    const double t = position * p.turns[f];
    float s, c;
    sincospif(static_cast<float>(2.0 * (t - rint(t))), &s, &c);
    cs[r][f] = make_float2(c * p.magnitude, (p.inverse ? -s : s) * p.magnitude);
  }
  __syncthreads();
  const Elem* x = static_cast<const Elem*>(p.x);
  Elem* out = static_cast<Elem*>(p.out);
  const int rotated = 2 * p.pairs;
  const bool copy = p.x != p.out && rotated < p.head_dim;
  if constexpr (kVec) {
    const int turning = p.interleaved ? rotated / EPL : p.pairs / EPL;              // units of a head that turn
    const int units = turning + (copy ? (p.head_dim - rotated) / EPL : 0);
    const int total = n_rows * p.n_heads * units;
    constexpr int BATCH = 2;
    for (int i0 = threadIdx.x; i0 < total; i0 += BATCH * kRotaryThreads) {
      uint4 a[BATCH], b[BATCH];
      long long at[BATCH], to[BATCH];
      int row[BATCH], unit[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int i = i0 + k * kRotaryThreads;
        unit[k] = -1;
        if (i >= total) continue;
        const int rh = i / units, u = i - rh * units, r = rh / p.n_heads, h = rh - r * p.n_heads;
        const int c = u < turning ? u * EPL : rotated + (u - turning) * EPL;
        unit[k] = u; row[k] = r;
        at[k] = (row0 + r) * p.ld_x + h * p.head_dim + c;
        to[k] = (row0 + r) * p.ld_out + h * p.head_dim + c;
        a[k] = *reinterpret_cast<const uint4*>(x + at[k]);
        if (!p.interleaved && u < turning) b[k] = *reinterpret_cast<const uint4*>(x + at[k] + p.pairs);
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (unit[k] < 0) continue;
        if (unit[k] >= turning) {
          *reinterpret_cast<uint4*>(out + to[k]) = a[k];
          continue;
        }
        float v[EPL];
        In::widen16(a[k], v);
        if (p.interleaved) {
          const float2* t = &cs[row[k]][unit[k] * (EPL / 2)];
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            const float va = v[e], vb = v[e + 1];
            v[e] = va * t[e / 2].x - vb * t[e / 2].y;
            v[e + 1] = va * t[e / 2].y + vb * t[e / 2].x;
          }
          *reinterpret_cast<uint4*>(out + to[k]) = narrow16<kType>(v);
        } else {
          float w[EPL];
          In::widen16(b[k], w);
          const float2* t = &cs[row[k]][unit[k] * EPL];
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            const float va = v[e], vb = w[e];
            v[e] = va * t[e].x - vb * t[e].y;
            w[e] = va * t[e].y + vb * t[e].x;
          }
          *reinterpret_cast<uint4*>(out + to[k]) = narrow16<kType>(v);
          *reinterpret_cast<uint4*>(out + to[k] + p.pairs) = narrow16<kType>(w);
        }
      }
    }
  } else {
    const int units = p.pairs + (copy ? p.head_dim - rotated : 0);
    const int total = n_rows * p.n_heads * units;
    for (int i = threadIdx.x; i < total; i += kRotaryThreads) {
      const int rh = i / units, u = i - rh * units, r = rh / p.n_heads, h = rh - r * p.n_heads;
      const long long from = (row0 + r) * p.ld_x + h * p.head_dim, to = (row0 + r) * p.ld_out + h * p.head_dim;
      if (u >= p.pairs) {
        const int c = rotated + u - p.pairs;
        out[to + c] = x[from + c];
        continue;
      }
      const int ca = p.interleaved ? 2 * u : u, cb = p.interleaved ? 2 * u + 1 : u + p.pairs;
      const float va = In::widen(x[from + ca]), vb = In::widen(x[from + cb]);
      const float2 t = cs[r][u];
      out[to + ca] = narrow<kType>(va * t.x - vb * t.y);
      out[to + cb] = narrow<kType>(va * t.y + vb * t.x);
    }
  }
}

}  // namespace dit
