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
  int n_heads, head_dim, pairs, inverse;
  int rows_per_cta;          // 1 or 4
  int pieces;                // of a head, kUnits at most
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

// A CTA takes a few rows: it computes their cosines and sines once, for all heads, and then turns their heads; channels behind the rotated
// part are copied (not at all in place).  Bound by HBM, each element read and written once.
//
// kUnits > 0: rows, heads and halves start on boundaries of kBytes (16 or 8), and the pieces of a head of that size, a piece and its
// partner counted once where pairs are apart, are at most kUnits.  A lane keeps its place in the head and the cosines and sines of it, and
// walks the heads of a row; its first pieces are requested before the sines are computed.  23058 rows of 40 heads of 128, fp16: 72-78 us, 6.0-6.5 TB/s
// (98 with a division per piece and the sines from shared memory, and as much with twice the pieces in flight and half the CTAs).
// kUnits == 0: a lane per pair, whatever the alignment.
template <int kBytes>
__device__ __forceinline__ uint4 load_piece(const void* p) {
  if constexpr (kBytes == 16) return *static_cast<const uint4*>(p);
  const uint2 v = *static_cast<const uint2*>(p);
  return make_uint4(v.x, v.y, 0u, 0u);
}
template <int kBytes>
__device__ __forceinline__ void store_piece(void* p, const uint4& v) {
  if constexpr (kBytes == 16) *static_cast<uint4*>(p) = v;
  else *static_cast<uint2*>(p) = make_uint2(v.x, v.y);
}

template <int kType, int kUnits, int kBytes, bool kInterleaved>
__global__ void __launch_bounds__(kRotaryThreads, 4)
rotary_kernel(const __grid_constant__ RotaryParams p) {
  using In = QuantIn<kType>;
  using Elem = typename In::Elem;
  constexpr int EPL = In::EPL, EPP = EPL * kBytes / 16;                            // elements of a 16-byte load, of a piece
  __shared__ float2 cs[kRotaryRows][kRotaryMaxPairs];
  dependents_may_start();
  await_predecessor();
  const long long row0 = static_cast<long long>(blockIdx.x) * p.rows_per_cta;
  const int n_rows = static_cast<int>(min(static_cast<long long>(p.rows_per_cta), p.rows - row0));
  const int rotated = 2 * p.pairs;

  constexpr int BATCH = kInterleaved ? 4 : 2, UNITS = kUnits > 0 ? kUnits : 1;
  constexpr int WARPS = kRotaryThreads / 32, PER = 32 / UNITS;                     // heads of a warp
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int mine = warp % p.rows_per_cta, step = WARPS / p.rows_per_cta * PER;
  const int turning = (kInterleaved ? rotated : p.pairs) / EPP;                    // pieces of a head that turn
  const int unit = lane % UNITS;
  const bool turns = unit < turning;
  const bool works = kUnits > 0 && mine < n_rows && unit < p.pieces && (turns || p.x != p.out);
  const int c = turns ? unit * EPP : rotated + (unit - turning) * EPP;
  int h0 = works ? warp / p.rows_per_cta * PER + lane / UNITS : p.n_heads;
  const Elem* x = static_cast<const Elem*>(p.x) + (row0 + mine) * p.ld_x + c;
  uint4 a[BATCH], b[BATCH];
  auto load = [&]() {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int h = h0 + k * step;
      if (h >= p.n_heads) break;
      a[k] = load_piece<kBytes>(x + h * p.head_dim);
      if (!kInterleaved && turns) b[k] = load_piece<kBytes>(x + h * p.head_dim + p.pairs);
    }
  };
  if constexpr (kUnits > 0) load();

  for (int i = threadIdx.x; i < n_rows * p.pairs; i += kRotaryThreads) {
    const int r = i / p.pairs, f = i - r * p.pairs;
    const long long row = row0 + r;
    int position;
    if (p.positions) {
      position = p.positions[row];
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
  if constexpr (kUnits > 0) {
    Elem* out = static_cast<Elem*>(p.out) + (row0 + mine) * p.ld_out + c;
    constexpr int ANGLES = kInterleaved ? EPP / 2 : EPP;                           // of a piece
    float2 t[ANGLES];
    if (turns && works) {
#pragma unroll
      for (int e = 0; e < ANGLES; ++e) t[e] = cs[mine][unit * ANGLES + e];
    }
    while (h0 < p.n_heads) {
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int h = h0 + k * step;
        if (h >= p.n_heads) break;
        Elem* to = out + h * p.head_dim;
        if (!turns) {
          store_piece<kBytes>(to, a[k]);
          continue;
        }
        float v[EPL];
        In::widen16(a[k], v);
        if constexpr (kInterleaved) {
#pragma unroll
          for (int e = 0; e < EPP; e += 2) {
            const float va = v[e], vb = v[e + 1];
            v[e] = va * t[e / 2].x - vb * t[e / 2].y;
            v[e + 1] = va * t[e / 2].y + vb * t[e / 2].x;
          }
        } else {
          float w[EPL];
          In::widen16(b[k], w);
#pragma unroll
          for (int e = 0; e < EPP; ++e) {
            const float va = v[e], vb = w[e];
            v[e] = va * t[e].x - vb * t[e].y;
            w[e] = va * t[e].y + vb * t[e].x;
          }
          store_piece<kBytes>(to + p.pairs, narrow16<kType>(w));
        }
        store_piece<kBytes>(to, narrow16<kType>(v));
      }
      h0 += BATCH * step;
      if (h0 < p.n_heads) load();
    }
  } else {
    const Elem* x = static_cast<const Elem*>(p.x);
    Elem* out = static_cast<Elem*>(p.out);
    const int units = p.pairs + (p.x != p.out ? p.head_dim - rotated : 0);
    const int total = n_rows * p.n_heads * units;
    for (int i = threadIdx.x; i < total; i += kRotaryThreads) {
      const int rh = i / units, u = i - rh * units, r = rh / p.n_heads, h = rh - r * p.n_heads;
      const long long from = (row0 + r) * p.ld_x + h * p.head_dim, to = (row0 + r) * p.ld_out + h * p.head_dim;
      if (u >= p.pairs) {
        const int c = rotated + u - p.pairs;
        out[to + c] = x[from + c];
        continue;
      }
      const int ca = kInterleaved ? 2 * u : u, cb = kInterleaved ? 2 * u + 1 : u + p.pairs;
      const float va = In::widen(x[from + ca]), vb = In::widen(x[from + cb]);
      const float2 t = cs[r][u];
      out[to + ca] = narrow<kType>(va * t.x - vb * t.y);
      out[to + cb] = narrow<kType>(va * t.y + vb * t.x);
    }
  }
}

}  // namespace dit
