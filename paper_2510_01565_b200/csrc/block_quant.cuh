// Quantisation to e4m3 codes with one fp32 scale per 128 columns of a row (activations) or per
// 128 x 128 block (weights, transposed on the way):
//   top = max(max|x|, 2^-100),  scale = top / 448,  code = e4m3(x * (448 / top))
// Both divisions and the product are single IEEE fp32 operations, so the codes are a function of the
// inputs alone that any fp32 implementation reproduces bit for bit.  The floor keeps 448 / top finite
// for groups of zeros and of tiny numbers.  A NaN passes through the maximum into scale and codes.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

constexpr float kQuantFloor = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ void quant_factors(float top, float& inv, float& scale) {
  top = fmax_nan(top, kQuantFloor);
  inv = __fdiv_rn(448.0f, top);
  scale = __fdiv_rn(top, 448.0f);
}

// Two values -> two e4m3 codes (low byte first), nearest even, clamped to +-448.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// kType: 0 = fp16, 1 = bf16, 2 = fp32.  Elements per 16-byte load and the widening of one load.
template <int kType>
struct QuantIn {
  static constexpr int EPL = kType == 2 ? 4 : 8;
  using Elem = typename std::conditional<kType == 2, float, uint16_t>::type;
  static __device__ __forceinline__ float widen(Elem e) {
    if constexpr (kType == 2) return e;
    else if constexpr (kType == 1) return __uint_as_float(static_cast<uint32_t>(e) << 16);
    else return __half2float(__ushort_as_half(e));
  }
  // Magnitudes by their bit patterns, whose integer order is the numbers' with infinity above every number and NaN above it.
  static __device__ __forceinline__ uint32_t max_bits(uint32_t top, uint32_t word) {
    if constexpr (kType == 2) return max(top, word & 0x7FFFFFFFu);
    else return __vmaxu2(top, word & 0x7FFF7FFFu);
  }
  static __device__ __forceinline__ uint32_t fold_bits(uint32_t top) { return kType == 2 ? top : max(top & 0xFFFFu, top >> 16); }
  static __device__ __forceinline__ float from_bits(uint32_t top) {
    if constexpr (kType == 2) return __uint_as_float(top);
    else return widen(static_cast<uint16_t>(top));
  }
  static __device__ __forceinline__ void widen16(const uint4& r, float (&v)[EPL]) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kType == 2) v[i] = __uint_as_float(u[i]);
      else if constexpr (kType == 1) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
      else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i])); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
    }
  }
};

struct QuantParams {
  const void* x;
  uint8_t* codes;
  float* scales;
  long long ld, ld_codes, ld_scales;
  int rows, cols, groups;      // groups of 128 columns
  int rows_per_task;           // 8 or 32
};

// One warp per (group of 128 columns, run of rows): a 16-byte load per lane covers the group in two rows
// (16-bit inputs) or one (fp32), the maximum is a shuffle reduction over the lanes of a row, and the
// run's scales leave as one coalesced store (they lie group-major).  Neighbouring warps take
// neighbouring groups, so a CTA reads runs of 2 KB.  Bound by HBM: 3 bytes per 16-bit element; four loads
// per lane are in flight (two or eight, a second batch ahead, more warps by fewer registers: all slower).  9216 x 12288 fp16: 58 us, 5.8 TB/s
// (66 us while every lane did the divisions of its rows).
// kVec: rows start on 16-byte boundaries; otherwise elements are loaded one by one.
constexpr int kQuantBlockWarps = 8;

template <int kType, bool kVec>
__global__ void __launch_bounds__(kQuantBlockWarps * 32)
quantize_block128_kernel(const QuantParams p) {
  using In = QuantIn<kType>;
  constexpr int EPL = In::EPL, LPR = 128 / EPL, RPI = 32 / LPR;   // lanes per row, rows per iteration
  constexpr int BATCH = 4;
  const int lane = threadIdx.x & 31;
  const long long task = static_cast<long long>(blockIdx.x) * kQuantBlockWarps + (threadIdx.x >> 5);
  const int group = static_cast<int>(task % p.groups);
  const long long row0 = task / p.groups * p.rows_per_task;
  if (row0 >= p.rows) return;
  const int n_rows = static_cast<int>(min(static_cast<long long>(p.rows_per_task), p.rows - row0));
  const int sub = lane / LPR, c0 = group * 128 + (lane % LPR) * EPL;
  const int n_in = min(EPL, p.cols - c0);                         // this lane's columns inside the matrix (may be <= 0)
  const typename In::Elem* src = static_cast<const typename In::Elem*>(p.x) + row0 * p.ld + c0;
  uint8_t* dst = p.codes + row0 * p.ld_codes + c0;
  float my_scale = 0.f;
  for (int b = 0; b < n_rows; b += BATCH * RPI) {
    float v[BATCH][EPL];
    if (kVec && n_in == EPL) {
      uint4 raw[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int r = b + i * RPI + sub;
        raw[i] = r < n_rows ? load_once(src + r * p.ld) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) In::widen16(raw[i], v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int r = b + i * RPI + sub;
#pragma unroll
        for (int e = 0; e < EPL; ++e) v[i][e] = (r < n_rows && e < n_in) ? In::widen(src[r * p.ld + e]) : 0.f;
      }
    }
    float top[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      top[i] = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; e += 2) top[i] = fmax3_nan(top[i], fabsf(v[i][e]), fabsf(v[i][e + 1]));
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) top[i] = fmax_nan(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
    }
    // The divisions of the batch's rows are shared out over the lanes: lane k works for row b + k % ROWS, which is also the
    // row of the run whose scale it keeps.
    constexpr int ROWS = BATCH * RPI;
    float row_top = 0.f, inv, scale;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float t = __shfl_sync(0xffffffffu, top[i], lane % RPI * LPR);
      if (lane % ROWS / RPI == i) row_top = t;
    }
    quant_factors(row_top, inv, scale);
    if (lane / ROWS == b / ROWS) my_scale = scale;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int r = b + i * RPI + sub;
      const float my_inv = __shfl_sync(0xffffffffu, inv, i * RPI + sub);
      if (r < n_rows && n_in > 0) {
        uint8_t* d = dst + r * p.ld_codes;
        uint32_t w[EPL / 4];
#pragma unroll
        for (int q = 0; q < EPL / 4; ++q)
          w[q] = e4m3x2(v[i][4 * q] * my_inv, v[i][4 * q + 1] * my_inv) | (e4m3x2(v[i][4 * q + 2] * my_inv, v[i][4 * q + 3] * my_inv) << 16);
        if (n_in == EPL) {                                        // rows of codes start on 16-byte boundaries
          if constexpr (EPL == 8) *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[1]);
          else *reinterpret_cast<uint32_t*>(d) = w[0];
        } else {
#pragma unroll
          for (int e = 0; e < EPL; ++e)
            if (e < n_in) d[e] = static_cast<uint8_t>(w[e / 4] >> (8 * (e % 4)));
        }
      }
    }
  }
  if (lane < n_rows) p.scales[group * p.ld_scales + row0 + lane] = my_scale;
}

// Weights w [in, out] -> codes [out, in] with one scale per 128 x 128 block: a CTA holds its block in
// registers (8 vectors of 16 bytes of 16-bit input per thread), reduces the maximum, and turns the block
// through shared memory as packed quadruples of codes along `in`.  A thread's vectors are four
// consecutive `in` rows at the same eight columns, so each of its 16 words holds four consecutive
// codes of one output row; word kq of row n lies at kq ^ 2 (n / 8), which keeps both phases free of
// bank conflicts.  HBM is the floor: 3 bytes per element.  3072 x 12288 bf16: 23.6 us, 4.8 TB/s (46 us with the widened values held: half the
// CTAs); what keeps it from 17.6 us is not known (2304 blocks of 32 KB on 592 resident CTAs: the tail is 3 %).
struct QuantWeightParams {
  const void* w;
  uint8_t* codes;
  float* scales;
  long long ld, ld_codes;
  int in_dim, out_dim, in_groups;
};

template <int kType, bool kVec>
__global__ void __launch_bounds__(256, kType == 2 ? 3 : 4)
quantize_weight_block128_kernel(const QuantWeightParams p) {
  using In = QuantIn<kType>;
  constexpr int COLS = 8, VECS = COLS / In::EPL;                  // 16-byte loads per eight columns: 1 (16-bit) or 2 (fp32)
  __shared__ uint32_t turned[128 * 32];
  __shared__ float warp_top[8];
  const int gk = blockIdx.x % p.in_groups, gn = blockIdx.x / p.in_groups;
  const int k0 = gk * 128, n0 = gn * 128;
  const int c = threadIdx.x & 15, rq = threadIdx.x >> 4;          // columns n0 + 8c .., rows k0 + 4 rq + 64 i + j
  const typename In::Elem* src = static_cast<const typename In::Elem*>(p.w);
  uint4 raw[2][4][VECS];                                          // as loaded: half the registers of the widened values
  uint32_t top_bits = 0;                                          // largest magnitude as bits (a pair of them for 16-bit inputs)
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + 4 * rq + 64 * i + j, n = n0 + 8 * c;
      const typename In::Elem* at = src + static_cast<long long>(k) * p.ld + n;
#pragma unroll
      for (int q = 0; q < VECS; ++q) {
        raw[i][j][q] = make_uint4(0, 0, 0, 0);
        if (kVec && k < p.in_dim && n + COLS <= p.out_dim) {
          raw[i][j][q] = __ldg(reinterpret_cast<const uint4*>(at) + q);
        } else if (k < p.in_dim) {
          typename In::Elem part[In::EPL];
#pragma unroll
          for (int e = 0; e < In::EPL; ++e) part[e] = n + q * In::EPL + e < p.out_dim ? at[q * In::EPL + e] : typename In::Elem(0);
          memcpy(&raw[i][j][q], part, 16);
        }
      }
    }
  auto value = [&](int i, int j, int e) {                         // column n0 + 8c + e of row k0 + 4 rq + 64 i + j
    float t[In::EPL];
    In::widen16(raw[i][j][e / In::EPL], t);
    return t[e % In::EPL];
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < VECS; ++q) {
        const uint32_t u[4] = {raw[i][j][q].x, raw[i][j][q].y, raw[i][j][q].z, raw[i][j][q].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) top_bits = In::max_bits(top_bits, u[w]);
      }
  top_bits = __reduce_max_sync(0xffffffffu, In::fold_bits(top_bits));
  float top = In::from_bits(top_bits);
  if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmax_nan(top, warp_top[i]);
  float inv, scale;
  quant_factors(top, inv, scale);
  if (threadIdx.x == 0) p.scales[static_cast<long long>(gn) * p.in_groups + gk] = scale;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < COLS; ++e) {
      const int n = 8 * c + e, kq = rq + 16 * i;
      turned[n * 32 + (kq ^ (2 * c))] = e4m3x2(value(i, 0, e) * inv, value(i, 1, e) * inv) | (e4m3x2(value(i, 2, e) * inv, value(i, 3, e) * inv) << 16);
    }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_in = min(4, p.in_dim - (k0 + 4 * lane));
#pragma unroll 4
  for (int r = 0; r < 16; ++r) {
    const int n = warp * 16 + r;
    if (n0 + n >= p.out_dim || n_in <= 0) continue;
    const uint32_t word = turned[n * 32 + (lane ^ (2 * (n >> 3)))];
    uint8_t* d = p.codes + static_cast<long long>(n0 + n) * p.ld_codes + k0 + 4 * lane;
    if (n_in == 4) *reinterpret_cast<uint32_t*>(d) = word;
    else
      for (int e = 0; e < n_in; ++e) d[e] = static_cast<uint8_t>(word >> (8 * e));
  }
}

}  // namespace dit
