// Microscaled 4-bit floating point: e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), two to a byte, the even column
// in the low half, under one of two scales (`kGroup` columns of a row share one):
//   32   scale = 2^e, e the smallest integer with top <= 6 * 2^e           (byte e + 127), code = e2m1(x * 2^-e)
//   16   scale = s * 2^e, e the smallest integer with row top <= 6 * 448 * 2^e (one fp32 2^e per row),
//        s = e4m3(top * 2^-e / 6), code = e2m1((x * 2^-e) / s), zero where s is zero
// with top = max(max|x|, 2^-100) of the group or row.  The row's factor is a power of two, so every product above is exact and each
// decision rests on one quotient, rounded to fp32: for 16-bit inputs it lies on a border between two codes exactly where the true one does, and
// codes can be tested bit for bit.
//
// Scale bytes lie in the order in which the tensor cores take them: tiles of 128 rows x 4 groups, 512 bytes,
//   byte (row % 32) * 16 + (row % 128) / 32 * 4 + group % 4   of tile [row / 128][group / 4]
// Whole tiles are written, zeros where no row or group is.
#pragma once
#include "block_quant.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

// Eight values -> eight codes, nearest with ties to the even code, |x| > 6 clamped.
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}\n"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
__device__ __forceinline__ uint32_t e2m1x4(float v0, float v1, float v2, float v3) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b;\n\t.reg .b16 h;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "mov.b16 h, {a, b};\n\tcvt.u32.u16 %0, h;\n\t}\n"
      : "=r"(r) : "f"(v0), "f"(v1), "f"(v2), "f"(v3));
  return r;
}
// Eight codes -> eight values.
__device__ __forceinline__ void e2m1_values(uint32_t codes, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }   // -126 <= e <= 127

// Smallest e with top <= limit * 2^e, where limit = (1 + kMantissa / 2^23) * 2^kExponent; top is finite and >= 2^-100.
template <uint32_t kMantissa, int kExponent>
__device__ __forceinline__ int scale_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  return static_cast<int>(u >> 23) - 127 - kExponent + ((u & 0x7FFFFFu) > kMantissa ? 1 : 0);
}
__device__ __forceinline__ int group_exponent(float top) { return scale_exponent<0x400000u, 2>(top); }        // 6 = 1.5 * 4
__device__ __forceinline__ int row_exponent(float top) { return scale_exponent<0x280000u, 11>(top); }         // 2688 = 1.3125 * 2048

// Values of scale bytes.
__device__ __forceinline__ float e8m0_value(uint32_t b) { return b == 0 ? __uint_as_float(0x00400000u) : (b == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(b << 23)); }
__device__ __forceinline__ float e4m3_value(uint32_t b) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(b), __NV_E4M3))); }

// What a lane needs to code values of its group: codes are e2m1(x * up * (high + low)).
struct GroupScale {
  uint32_t byte;
  float up, high, low;       // 2^-e; the reciprocal of the e4m3 number in two parts (groups of 16)
  bool none;                 // every code is zero
};
// up: 2^-e of the row (groups of 16); bad: the row (16) or group (32) holds a NaN or an infinity.
//
// There are no divisions.  A quotient x / s of a 24-bit x and an s of four bits (or 6, two bits) that fp32 does not hold is at least 2^-29 of
// itself away from the middle between two fp32 numbers.  With the reciprocal in two parts, low = (1 - s high) high, the sum x high + x low is off
// by less than 2^-44 before its one rounding: it is the correctly rounded quotient.
template <int kGroup>
__device__ __forceinline__ GroupScale group_scale(float top, float up, bool bad) {
  GroupScale g;
  if constexpr (kGroup == 32) {
    const int e = group_exponent(fmaxf(bad ? 0.f : top, kQuantFloor));
    g.byte = bad ? 255u : static_cast<uint32_t>(e + 127);
    g.up = pow2(-e);
    g.high = 1.f; g.low = 0.f;
    g.none = bad;
  } else {
    const float t = top * up;
    constexpr float kSixth = 0.16666667163372039794921875f, kRest = -4.967053879312289e-09f;      // 1/6 = kSixth + kRest, |error| < 2^-50
    g.byte = bad ? 0u : __nv_cvt_float_to_fp8(fmaf(t, kSixth, t * kRest), __NV_SATFINITE, __NV_E4M3);
    g.none = g.byte == 0;
    g.up = up;
    const float s = e4m3_value(g.byte);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(g.high) : "f"(s));
    g.low = g.high * fmaf(-s, g.high, 1.0f);
  }
  return g;
}

// Codes of eight (16-bit inputs) or four values.
template <int kGroup, int N>
__device__ __forceinline__ uint32_t encode(const float (&v)[N], const GroupScale& g) {
  float q[N];
  const float2 up = make_float2(g.up, g.up), high = make_float2(g.high, g.high), low = make_float2(g.low, g.low);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    float2 x = fmul2(make_float2(v[i], v[i + 1]), up);
    if constexpr (kGroup == 16) x = ffma2(x, high, fmul2(x, low));
    q[i] = x.x; q[i + 1] = x.y;
  }
  uint32_t code;
  if constexpr (N == 8) code = e2m1x8(q);
  else code = e2m1x4(q[0], q[1], q[2], q[3]);
  return g.none ? 0u : code;
}

// EPL consecutive elements from any element address, as the words of a 16-byte load; `n` of them exist (may be <= 0), the rest are zero.  kVec: the
// address is a multiple of 16.  Otherwise whole runs come as 32-bit words, of 16-bit elements that start in the middle of a word as the
// words around them, shifted (`before`: the element in front of the run may be read as well, and so may the one behind it where n > EPL).
template <int kType, bool kVec>
__device__ __forceinline__ uint4 load_run(const typename QuantIn<kType>::Elem* src, int n, bool before) {
  constexpr int EPL = QuantIn<kType>::EPL;
  if (n >= EPL) {
    if constexpr (kVec) return load_passing(src);
    if constexpr (kType == 2) {
      return make_uint4(__float_as_uint(*src), __float_as_uint(src[1]), __float_as_uint(src[2]), __float_as_uint(src[3]));
    } else {
      const uintptr_t at = reinterpret_cast<uintptr_t>(src);
      const uint32_t* words = reinterpret_cast<const uint32_t*>(at & ~static_cast<uintptr_t>(3));
      if (!(at & 2)) return make_uint4(words[0], words[1], words[2], words[3]);
      if (before && n > EPL) {
        const uint32_t w0 = words[0], w1 = words[1], w2 = words[2], w3 = words[3], w4 = words[4];
        return make_uint4(__funnelshift_r(w0, w1, 16), __funnelshift_r(w1, w2, 16), __funnelshift_r(w2, w3, 16), __funnelshift_r(w3, w4, 16));
      }
    }
  }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < EPL; ++e)
    if (e < n) {
      if constexpr (kType == 2) w[e] = __float_as_uint(src[e]);
      else w[e >> 1] |= static_cast<uint32_t>(src[e]) << (16 * (e & 1));
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Fp4QuantParams {
  const void* x;             // [rows, cols], row stride ld
  uint8_t* codes;
  uint8_t* scales;
  float* row_scales;         // groups of 16 only
  long long ld, ld_codes;    // ld_codes in bytes
  int rows, cols, chunks;    // chunks: scale tiles of a row
};

__device__ __forceinline__ long long scale_at(int row, int group, int chunks) {
  return (static_cast<long long>(row >> 7) * chunks + (group >> 2)) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4 + (group & 3);
}

// A row per THREADS lanes (a warp of a CTA of eight, or a whole CTA), kBytes of consecutive columns per lane and load: EPL values, kGroup / EPL
// lanes to a group.  A row of up to THREADS * kLoads loads stays in registers between its maximum and its codes; a longer one
// is read twice.  Rows behind the last one up to the tile's end get their zero scales only.  Bound by HBM and the issue of instructions:
// 9216 x 12288 fp16 49 us, 5.9 TB/s (groups of 32, without the meeting of the CTA, 43).
// kBytes: what rows' starts are multiples of, 32 (one load per group of 16 16-bit numbers: its scale is found once), 16, or 0: anywhere,
// loads of 16 bytes' worth made up of smaller ones.
// Registers are held down to what lets as many whole CTAs as go into 1280 threads (1536 with little to hold) fit an SM: five of 256 threads, two of 512 (one
// without the bound; 4096 x 40000 fp16, read twice, 140 -> 92 us, 10630 x 6480 44 -> 40).
template <int kType, int kGroup, int kBytes, int THREADS, int kLoads>
__global__ void __launch_bounds__(THREADS == 32 ? 256 : THREADS, (kLoads * (kBytes == 32 ? 2 : 1) <= 4 ? 1536 : 1280) / (THREADS == 32 ? 256 : THREADS))
quantize_fp4_kernel(const Fp4QuantParams p) {
  using In = QuantIn<kType>;
  constexpr int W = kBytes == 32 ? 2 : 1;                         // 16-byte words of a load
  constexpr int EPW = In::EPL, EPL = EPW * W, LPG = kGroup / EPL; // values of a word, of a load; lanes per group
  constexpr int CTA = THREADS == 32 ? 256 : THREADS;
  __shared__ uint32_t warp_top[CTA / 32];
  dependents_may_start();
  await_predecessor();
  const int at = threadIdx.x % THREADS;                           // lane of the row
  const long long row_l = static_cast<long long>(blockIdx.x) * (CTA / THREADS) + threadIdx.x / THREADS;
  const int padded = (p.rows + 127) / 128 * 128;
  if (row_l >= padded) return;                                    // (a whole warp; with a row per CTA none)
  const int row = static_cast<int>(row_l);
  const bool there = row < p.rows;
  const int span = THREADS * EPL * kLoads;                        // columns held at a time
  const int wide = p.chunks * 4 * kGroup;                         // columns with a scale byte
  const typename In::Elem* src = static_cast<const typename In::Elem*>(p.x) + (there ? row : 0) * p.ld;
  uint4 raw[kLoads][W];
  auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = base + (i * THREADS + at) * EPL, n = there ? p.cols - c : 0;
      if (W == 2 && n >= EPL) {
        if constexpr (W == 2) load_passing_v8(raw[i], src + c);
      } else {
#pragma unroll
        for (int w = 0; w < W; ++w) raw[i][w] = load_run<kType, (kBytes > 0)>(src + c + w * EPW, n - w * EPW, c + w > 0);
      }
    }
  };
  auto top_of = [&](const uint4 (&r)[W]) {
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) top = In::max_bits(In::max_bits(In::max_bits(In::max_bits(top, r[w].x), r[w].y), r[w].z), r[w].w);
    return top;
  };
  load(0);
  float up = 0.f;
  bool bad = false;
  if constexpr (kGroup == 16) {
    uint32_t top = 0;
    for (int base = 0;;) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) top = kType == 2 ? max(top, top_of(raw[i])) : __vmaxu2(top, top_of(raw[i]));
      base += span;
      if (base >= p.cols) break;
      load(base);
    }
    top = In::fold_bits(top);
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (THREADS > 32) {
      if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = top;
      __syncthreads();
      top = warp_top[threadIdx.x & (CTA / 32 - 1)];
      top = __reduce_max_sync(0xffffffffu, top);
    }
    const float row_top = In::from_bits(top);
    bad = !(row_top < INFINITY);
    const int e = row_exponent(fmaxf(bad ? 1.f : row_top, kQuantFloor));
    up = pow2(-e);
    if (there && at == 0) p.row_scales[row] = bad ? __uint_as_float(0x7FC00000u) : pow2(e);
    if (span < p.cols) load(0);
  }
  // the lane's first byte and code of the row; a load further on they are fixed distances away
  uint8_t* scale = p.scales + scale_at(row, at * EPL / kGroup, p.chunks);
  uint8_t* codes = p.codes + row * p.ld_codes + at * (EPL / 2);
  for (int base = 0; base < wide; base += span) {
    if (base > 0) load(base);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = base + (i * THREADS + at) * EPL;
      if (base + i * THREADS * EPL >= wide) break;
      uint32_t bits = In::fold_bits(top_of(raw[i]));
#pragma unroll
      for (int o = 1; o < LPG; o <<= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
      const float top = In::from_bits(bits);
      const GroupScale g = group_scale<kGroup>(top, up, kGroup == 32 ? !(top < INFINITY) : bad);
      // (THREADS * EPL columns are whole tiles of four groups: 512 bytes each)
      if (c < wide && (at % LPG) == 0) scale[static_cast<long long>((base / EPL + i * THREADS) / (4 * LPG)) * 512] = there && c < p.cols ? static_cast<uint8_t>(g.byte) : 0;
      if (there && c < p.cols) {
        uint32_t code[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
          float v[EPW];
          In::widen16(raw[i][w], v);
          code[w] = encode<kGroup, EPW>(v, g);
        }
        uint8_t* dst = codes + (base + i * THREADS * EPL) / 2;
        if (c + EPL <= p.cols) {
          if constexpr (EPL == 16) *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[1]);
          else if constexpr (EPL == 8 && W == 2) *reinterpret_cast<uint32_t*>(dst) = code[0] | code[1] << 16;
          else if constexpr (EPL == 8) *reinterpret_cast<uint32_t*>(dst) = code[0];
          else *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(code[0]);
        } else {
          for (int b = 0; 2 * b < p.cols - c; ++b) dst[b] = static_cast<uint8_t>(code[b / (EPW / 2)] >> (8 * (b % (EPW / 2))));
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ weights
struct Fp4QuantWeightParams {
  const void* w;             // [in_dim, out_dim], row stride ld
  uint8_t* codes;            // [out_dim, ld_codes]
  uint8_t* scales;
  float* row_scales;         // [out_dim], groups of 16 only
  long long ld, ld_codes;
  int in_dim, out_dim, chunks;
};

// Row scales of a weight for groups of 16: the largest 2^e over a column, by an atomic maximum of positive numbers' bits (whose order does
// not matter), over row_scales cleared to zero before.  A CTA takes 64 columns x kColumnRows rows.
constexpr int kColumnRows = 256;
template <int kType, bool kVec>
__global__ void __launch_bounds__(256)
fp4_column_scales_kernel(const Fp4QuantWeightParams p) {
  using In = QuantIn<kType>;
  constexpr int EPL = In::EPL, LPR = 64 / EPL, RPI = 256 / LPR;    // lanes per row, rows per iteration
  __shared__ uint32_t tops[64];
  dependents_may_start();
  const int tiles = (p.out_dim + 63) / 64;
  const int col0 = blockIdx.x % tiles * 64;
  const long long row0 = static_cast<long long>(blockIdx.x / tiles) * kColumnRows;
  const int c = col0 + threadIdx.x % LPR * EPL, sub = threadIdx.x / LPR;
  if (threadIdx.x < 64) tops[threadIdx.x] = 0;
  __syncthreads();
  const typename In::Elem* src = static_cast<const typename In::Elem*>(p.w) + row0 * p.ld + c;
  const int n = static_cast<int>(min(static_cast<long long>(kColumnRows), p.in_dim - row0));
  uint4 top = make_uint4(0, 0, 0, 0);
  auto take = [&](uint32_t a, uint32_t b) { return kType == 2 ? max(a, b & 0x7FFFFFFFu) : __vmaxu2(a, b & 0x7FFF7FFFu); };
  constexpr int BATCH = kColumnRows / RPI < 8 ? kColumnRows / RPI : 8;             // all are requested before the first is used
  for (int r0 = sub; r0 < n; r0 += BATCH * RPI) {
    uint4 v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int r = r0 + i * RPI;
      v[i] = load_run<kType, kVec>(src + r * p.ld, r < n ? p.out_dim - c : 0, c > 0);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) top = make_uint4(take(top.x, v[i].x), take(top.y, v[i].y), take(top.z, v[i].z), take(top.w, v[i].w));
  }
  const uint32_t t[4] = {top.x, top.y, top.z, top.w};
  const int at = threadIdx.x % LPR * EPL;
#pragma unroll
  for (int i = 0; i < EPL; ++i) atomicMax(&tops[at + i], kType == 2 ? t[i] : (t[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
  __syncthreads();
  if (threadIdx.x < 64 && col0 + threadIdx.x < p.out_dim) {
    const float x = In::from_bits(tops[threadIdx.x]);
    const bool bad = !(x < INFINITY);
    const uint32_t bits = bad ? 0x7FC00000u : __float_as_uint(pow2(row_exponent(fmaxf(x, kQuantFloor))));
    atomicMax(reinterpret_cast<unsigned int*>(p.row_scales) + col0 + threadIdx.x, bits);
  }
}

// A CTA transposes 128 x 64 weights through shared memory.  Neighbouring lanes then take the groups of one output row, so that a row's codes leave as
// 64 consecutive bytes and its scales as words.
constexpr int kWeightOut = 64;
template <int kType, int kGroup, bool kVec>
__global__ void __launch_bounds__(256)
quantize_weight_fp4_kernel(const Fp4QuantWeightParams p) {
  using In = QuantIn<kType>;
  using Elem = typename In::Elem;
  constexpr int EPL = In::EPL, kIn = 128, LPR = kWeightOut / EPL, RPI = 256 / LPR;
  // rows an odd number of words apart, and groups shifted against one another: lanes of several groups and rows meet in different banks
  constexpr int PITCH = kWeightOut + (kType == 2 ? 1 : 2), SHIFT = kGroup == 32 ? 8 : 4;
  auto place = [](int r) { return r * PITCH + r / kGroup * SHIFT; };
  __shared__ __align__(16) Elem tile[kIn * PITCH + kIn / kGroup * SHIFT];          // (16-bit weights are written in pairs)
  dependents_may_start();
  await_predecessor();
  const int out_tiles = (p.out_dim + 127) / 128 * 2;               // whole scale tiles
  const int n0 = blockIdx.x % out_tiles * kWeightOut;
  const int k0 = blockIdx.x / out_tiles * kIn;
  {
    const int c = threadIdx.x % LPR * EPL;
    const Elem* src = static_cast<const Elem*>(p.w) + static_cast<long long>(k0) * p.ld + n0 + c;
    uint4 v[kIn / RPI];                                            // all are requested before the first is used
#pragma unroll
    for (int i = 0; i < kIn / RPI; ++i) {
      const int r = i * RPI + threadIdx.x / LPR;
      v[i] = load_run<kType, kVec>(src + r * p.ld, k0 + r < p.in_dim ? p.out_dim - n0 - c : 0, n0 + c > 0);
    }
#pragma unroll
    for (int i = 0; i < kIn / RPI; ++i) {
      const int r = i * RPI + threadIdx.x / LPR;
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      if constexpr (kType == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[place(r) + c + e] = __uint_as_float(w[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(&tile[place(r) + c + 2 * e]) = w[e];
      }
    }
  }
  __syncthreads();
  constexpr int GROUPS = kIn / kGroup;                             // of the tile's columns: 8 or 4, two scale tiles or one
  const int gi = threadIdx.x % GROUPS, group = k0 / kGroup + gi, k = k0 + gi * kGroup;
  const bool tiled = group < 4 * p.chunks;
#pragma unroll
  for (int turn = 0; turn < GROUPS * kWeightOut / 256; ++turn) {
    const int n = turn * (256 / GROUPS) + threadIdx.x / GROUPS, row = n0 + n;
    const bool there = row < p.out_dim && k < p.in_dim;
    float v[kGroup];
    float top = 0.f;
    const Elem* from = tile + place(gi * kGroup) + n;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      v[i] = In::widen(from[i * PITCH]);
      top = fmax_nan(top, fabsf(v[i]));
    }
    float up = 0.f;
    bool bad = !(top < INFINITY);
    if constexpr (kGroup == 16) {
      const uint32_t u = there ? __float_as_uint(p.row_scales[row]) : 0x3F800000u;
      bad = u >= 0x7F800000u;
      up = bad ? 1.f : pow2(127 - static_cast<int>(u >> 23));
    }
    const GroupScale g = group_scale<kGroup>(bad ? 0.f : top, up, bad);
    uint32_t word = there ? g.byte << (8 * (gi & 3)) : 0u;         // four neighbouring groups' bytes
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    if (tiled && (gi & 3) == 0) *reinterpret_cast<uint32_t*>(p.scales + scale_at(row, group, p.chunks)) = word;
    if (!there) continue;
    uint32_t code[kGroup / 8];
#pragma unroll
    for (int b = 0; b < kGroup / 8; ++b) {
      float part[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) part[i] = v[8 * b + i];
      code[b] = encode<kGroup, 8>(part, g);
    }
    uint8_t* dst = p.codes + row * p.ld_codes + k / 2;
    const int bytes = min(kGroup, p.in_dim - k + 1) / 2;           // of the group: all of its kGroup / 2, or the row's last ones
    if (bytes == kGroup / 2) {
      if constexpr (kGroup == 32) *reinterpret_cast<uint4*>(dst) = make_uint4(code[0], code[1], code[2], code[3]);
      else *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[1]);
    } else {
      for (int b = 0; b < bytes; ++b) dst[b] = static_cast<uint8_t>(code[b >> 2] >> (8 * (b & 3)));
    }
  }
}

// ------------------------------------------------------------------------------------------------ the values
struct Fp4ValuesParams {
  const uint8_t *codes, *scales;
  const float* row_scales;   // or NULL
  void* out;
  long long ld_codes, ld_out;
  int rows, cols, chunks;
};

// code * scale (exact) * row scale, rounded to fp32 and then to the output's type.  A lane takes `PER` consecutive codes of a row at a time, a warp a
// row, a CTA kTurns rows per warp.  Bound by HBM: 9216 x 12288 to fp16 45 us, 6.4 TB/s.
// kBytes: what rows of out are known to start on multiples of, 32: sixteen codes per lane, one scale of either group and whole sectors
// to write; 16: eight codes, so that a 16-bit type's neighbouring stores still fill sectors; 0: anywhere.
constexpr int kValueWarps = 8;
template <int kType, int kGroup, int kBytes, int kTurns>
__global__ void __launch_bounds__(kValueWarps * 32)
dequantize_fp4_kernel(const Fp4ValuesParams p) {
  constexpr int PER = kBytes == 32 ? 16 : 8, WORDS = PER / 8;
  using Out = typename QuantIn<kType>::Elem;
  const int col_tiles = (p.cols + 32 * PER - 1) / (32 * PER);
  __shared__ float lines[kBytes ? 1 : kValueWarps][kBytes ? 1 : 32 * 9];
  dependents_may_start();
  await_predecessor();
  const int lane = threadIdx.x & 31;
  const int row0 = blockIdx.x / col_tiles * (kValueWarps * kTurns) + (threadIdx.x >> 5), c = blockIdx.x % col_tiles * (32 * PER) + lane * PER;
  if (kBytes && c >= p.cols) return;
  const uint8_t* codes = p.codes + row0 * p.ld_codes + c / 2;
  uint32_t code[kTurns][WORDS], byte[kTurns];
  float factor[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int row = row0 + i * kValueWarps;
    byte[i] = 0; factor[i] = 1.f;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) code[i][w] = 0;
    if (row >= p.rows) continue;
    const uint8_t* src = codes + i * kValueWarps * p.ld_codes;
    if (WORDS == 2 && c + 16 <= p.cols) {
      const uint2 x = *reinterpret_cast<const uint2*>(src);
      code[i][0] = x.x; code[i][WORDS - 1] = x.y;
    } else {
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const int n = p.cols - c - 8 * w;
        if (n >= 8) code[i][w] = *reinterpret_cast<const uint32_t*>(src + 4 * w);
        else
          for (int b = 0; 2 * b < n; ++b) code[i][w] |= static_cast<uint32_t>(src[4 * w + b]) << (8 * b);
      }
    }
    if (c < p.cols) byte[i] = p.scales[scale_at(row, c / kGroup, p.chunks)];
    if (p.row_scales) factor[i] = p.row_scales[row];
  }
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int row = row0 + i * kValueWarps;
    if (row >= p.rows) break;                                      // (the whole warp)
    float scale = kGroup == 16 ? e4m3_value(byte[i]) : e8m0_value(byte[i]), times = factor[i];
    // 6 * 2^126 is no fp32 number, but may be one under a row factor below 1: a part of the scale goes there (exactly, both are far from their limits)
    if (kGroup == 32 && byte[i] >= 253 && fabsf(times) < 1.f) { scale *= 0.125f; times *= 8.f; }
    Out* out = static_cast<Out*>(p.out) + row * p.ld_out + c;
    float v[WORDS][8];
    uint32_t packed[WORDS][4];                                     // (16-bit types)
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      e2m1_values(code[i][w], v[w]);
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float2 x = fmul2(fmul2(make_float2(v[w][j], v[w][j + 1]), make_float2(scale, scale)), make_float2(times, times));
        v[w][j] = x.x; v[w][j + 1] = x.y;
        if constexpr (kType != 2) packed[w][j / 2] = pack16x2<kType == 1>(x.x, x.y);
      }
    }
    if constexpr (kBytes > 0) {
      if (kType != 2 && WORDS == 2 && c + 16 <= p.cols) {
        st_global_v8(out, *reinterpret_cast<const uint32_t(*)[8]>(packed));
        continue;
      }
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        Out* dst = out + 8 * w;
        const int n = p.cols - c - 8 * w;
        if (n >= 8) {
          if constexpr (kType != 2) *reinterpret_cast<uint4*>(dst) = make_uint4(packed[w][0], packed[w][1], packed[w][2], packed[w][3]);
          else if constexpr (kBytes == 32) st_global_v8(dst, *reinterpret_cast<const uint32_t(*)[8]>(v[w]));
          else {
            reinterpret_cast<float4*>(dst)[0] = make_float4(v[w][0], v[w][1], v[w][2], v[w][3]);
            reinterpret_cast<float4*>(dst)[1] = make_float4(v[w][4], v[w][5], v[w][6], v[w][7]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < n) {
              if constexpr (kType == 2) dst[j] = v[w][j];
              else dst[j] = pack16<kType == 1>(v[w][j]);
            }
        }
      }
    } else {
      // through shared memory, so that neighbouring lanes write neighbouring elements
      float* line = lines[threadIdx.x >> 5];
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) line[lane * 9 + j] = v[0][j];    // (nine words apart: no two lanes in a bank)
      __syncwarp();
      const int c0 = c - lane * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        if (c0 + e < p.cols) {
          const float x = line[e / 8 * 9 + e % 8];
          if constexpr (kType == 2) out[e - lane * 8] = x;
          else out[e - lane * 8] = pack16<kType == 1>(x);
        }
      }
    }
  }
}

}  // namespace dit
