// Product of two microscaled 4-bit operands (fp4_quant.cuh) for sm_100a:
//   C[m, n] = ra[m] * rb[n] * sum_k (code_a[m, k] sa[m, k / G]) (code_b[n, k] sb[n, k / G])   (+ bias[n])
// The tensor cores apply the group scales themselves (kind::mxf4nvf4 with four e4m3 scales per 64 k, kind::mxf4 with two powers of two), four
// times the 16-bit rate.  They read them from tensor memory: a 512-byte tile of scales (128 rows x 4 groups) becomes four columns,
// copied there from shared memory by tcgen05.cp, which the tensor pipe takes in order with the products.  The row factors, one per
// row and per column of C, are applied to the finished sums.
#pragma once
#include "block_gemm.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

struct Fp4GemmParams {
  int M, N, K;
  int band;                  // tile order, see tile_coords
  const float* ra;           // [M] or NULL
  const float* rb;           // [N] or NULL
  const float* bias;         // [N] or NULL
  void* out;
  long long ld_out;
  int vec_out;               // rows of out start on 16-byte boundaries
  int* status;
};

// ----------------------------------------------------------------------------------- block-scaled MMA
// Instruction descriptor: e2m1 operands, both K-major, M x N, K = 64; scale type e4m3 or power of two; the scale words' first byte.
template <int kGroup>
__host__ __device__ constexpr uint32_t idesc_fp4(int m, int n, int sf_id) {
  return (static_cast<uint32_t>(sf_id) << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | ((kGroup == 32 ? 1u : 0u) << 23)
         | (static_cast<uint32_t>(m >> 4) << 24) | (static_cast<uint32_t>(sf_id) << 29);
}
#define DIT_MMA_FP4(group, kind)                                                                                                            \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, [%5], [%6], p;\n\t}\n" \
               ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(sa_tmem), "r"(sb_tmem) : "memory")
template <int kGroup, bool kPair>
__device__ __forceinline__ void umma_fp4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem, uint32_t accumulate) {
  if constexpr (kGroup == 16 && kPair) DIT_MMA_FP4("2", "mxf4nvf4.block_scale.scale_vec::4X");
  else if constexpr (kGroup == 16) DIT_MMA_FP4("1", "mxf4nvf4.block_scale.scale_vec::4X");
  else if constexpr (kPair) DIT_MMA_FP4("2", "mxf4.block_scale.scale_vec::2X");
  else DIT_MMA_FP4("1", "mxf4.block_scale.scale_vec::2X");
}
// 512 bytes of shared memory (32 rows of 16 bytes) to four columns of tensor memory, the same in every quarter of the lanes; pair:
// from each CTA's own memory to its own.  Taken in order with the products that the same thread issues.
template <bool kPair>
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint64_t desc) {
  if constexpr (kPair) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Rows of 16 bytes one after the other, eight to 128 bytes, no swizzle.
__device__ __forceinline__ uint64_t smem_desc_rows16(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFF) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}
// 3-D tiled load of either CTA of a pair (see tma_load_2d_pair).
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const void* tmap, int x, int y, int z, uint32_t bar_cluster) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar_cluster)
      : "memory");
}

// A finished sum with its row's and its column's factor and the bias.  A caller's factors may be of any size (a quantiser's row factors span 2^-111 to
// 2^117): the result leaves fp32's range where the whole product does.  Where the sum times the row's factor is already outside it, and the column's
// factor leads back, the product of the two factors comes first, whose size lies between theirs.
__device__ __forceinline__ float fp4_finish(float sum, float fr, float fc, float bias) {
  const float t = sum * fr;
  const bool outside = !(fabsf(t) < INFINITY) || (fabsf(t) < 0x1p-126f && sum != 0.f);
  const bool across = outside && (fabsf(fr) > 1.f) != (fabsf(fc) > 1.f);
  return fmaf(across ? sum : t, across ? fr * fc : fc, bias);
}

// Scale tiles per stage of 256 k, and how a step of 64 k finds its scales in them.
template <int kGroup>
struct Fp4Scales {
  static constexpr int TILES = 256 / (4 * kGroup);                     // 4 (16) or 2 (32) per 128 rows
  static constexpr int STEPS = kGroup == 16 ? 1 : 2;                   // MMAs per tile
  static constexpr int BYTES = TILES * 512;                            // per 128 rows and stage
};

namespace fgemm {
constexpr int BM = 128, BN = 256;
constexpr int A_BYTES = BM * 128, B_BYTES = (BN / 2) * 128;            // 256 k are 128 bytes
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 128 + 32 * EPI_WARPS;
constexpr int REGS_ISSUE = 56, REGS_EPILOGUE = 224;                    // (56 + 2 * 224) * 32 <= 16384 per scheduler
constexpr int BOX_BYTES = 4096;                                        // 128 bytes x 32 rows of the output, one per epilogue warp
constexpr int COL_BYTES = 2 * 512;                                     // column factors and bias of 128 columns, shared by four warps
constexpr int kOverlap = 64;                                           // columns that the two accumulators share
constexpr int kScaleCols = 512 - (2 * BN - kOverlap);                  // 64 columns for scales behind them
template <int kGroup>
struct Cfg {
  using S = Fp4Scales<kGroup>;
  static constexpr int STAGES = 5;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + 3 * S::BYTES;
  static constexpr int SLOT = 12;                                      // columns of one tile of a's scales and two of b's
  static constexpr int SLOTS = kScaleCols / SLOT;
  static constexpr int OFF_OUT = (STAGES * STAGE_BYTES + 1023) / 1024 * 1024;
  static constexpr int OFF_COL = OFF_OUT + EPI_WARPS * BOX_BYTES, OFF_BAR = OFF_COL + 2 * COL_BYTES;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  static_assert(STAGE_BYTES % 1024 == 0, "swizzled tiles start on 1 KB boundaries");
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};
}  // namespace fgemm

// Writes a warp's box (32 rows of 128 bytes, 16-byte units XOR-swizzled by the row) to an output whose rows start off 16-byte boundaries, row by
// row in 32-bit words; 16-bit rows that start in the middle of a word are shifted by one element on the way.  `cols` columns from c0 on exist
// (may be <= 0).
// Whole boxes take a loop of a few instructions per row, without bounds.  Sectors written in part are what is left (9472 x 8191 x 1024
// fp16 137 us, 8190 columns 90, 8192 columns 46).
template <int EPI>
__device__ __forceinline__ void fp4_store_box(const Fp4GemmParams& p, const uint8_t* box, int lane, int row0, int c0, int cols) {
  constexpr bool kWide = EPI == kBlkF32;
  const int rows = min(32, p.M - row0);
  const long long first = static_cast<long long>(row0) * p.ld_out + c0;
  // a lane's word of row r: 16-byte unit lane / 4, XORed with r % 8
  const uint8_t* word = box + ((lane & 3) << 2);
  const int unit = lane >> 2;
  auto read = [&](int r) { return *reinterpret_cast<const uint32_t*>(word + r * 128 + ((unit ^ (r & 7)) << 4)); };
  if (rows == 32 && cols >= (kWide ? 32 : 64)) {
    if constexpr (kWide) {
      float* at = static_cast<float*>(p.out) + first + lane;
#pragma unroll 8
      for (int r = 0; r < 32; ++r, at += p.ld_out) *at = __uint_as_float(read(r));
    } else {
      uint16_t* at = static_cast<uint16_t*>(p.out) + first;
      const bool edge = lane == 0 || lane == 31;
#pragma unroll 8
      for (int r = 0; r < 32; ++r, at += p.ld_out) {
        uint32_t v = read(r);
        if ((reinterpret_cast<uintptr_t>(at) & 2) == 0) {              // (warp-uniform)
          *reinterpret_cast<uint32_t*>(at + 2 * lane) = v;
        } else {                                                       // elements 1 .. 62 as words, 0 and 63 alone
          const uint32_t next = __shfl_down_sync(0xffffffffu, v, 1);
          if (lane < 31) *reinterpret_cast<uint32_t*>(at + 2 * lane + 1) = __funnelshift_r(v, next, 16);
          if (edge) at[lane == 0 ? 0 : 63] = static_cast<uint16_t>(lane == 0 ? v : v >> 16);
        }
      }
    }
    return;
  }
  for (int r = 0; r < rows; ++r) {
    const uint32_t v = read(r);
    if constexpr (kWide) {
      if (lane < cols) static_cast<float*>(p.out)[first + r * p.ld_out + lane] = __uint_as_float(v);
    } else {
      uint16_t* at = static_cast<uint16_t*>(p.out) + first + r * p.ld_out + 2 * lane;
      if (2 * lane + 1 < cols && (reinterpret_cast<uintptr_t>(at) & 2) == 0) {
        *reinterpret_cast<uint32_t*>(at) = v;
      } else {
        if (2 * lane < cols) at[0] = static_cast<uint16_t>(v);
        if (2 * lane + 1 < cols) at[1] = static_cast<uint16_t>(v >> 16);
      }
    }
  }
}

// Persistent, one 256 x 256 tile per CTA pair, 256 k per stage.  Roles: warp 0 TMA producer, warp 1 issues scale copies and MMAs (leader CTA;
// it owns tensor memory), warps 4..11 take finished tiles out: two per quarter of the tile's rows, one for each 128 columns.
// Two accumulators of 256 columns and the scales need more than tensor memory's 512 columns, so the accumulators share 64: the warps
// that hold the shared ones take them out first, and the next tile's products begin once that is done.
template <int EPI, int kGroup>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(fgemm::THREADS, 1)
gemm_fp4_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmSA,
                     const __grid_constant__ CUtensorMap tmSB, const __grid_constant__ CUtensorMap tmOut, const Fp4GemmParams p) {
  using namespace fgemm;
  using C = Cfg<kGroup>;
  using S = Fp4Scales<kGroup>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + 2 + b); };
  const uint32_t shared_bar = bar0 + 8u * (2 * STAGES + 4);            // the shared columns of the last tile are out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * (2 * STAGES + 5));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int num_m = (p.M + 2 * BM - 1) / (2 * BM), num_n = (p.N + BN - 1) / BN;
  const int num_tiles = num_m * num_n;
  const int steps = (p.K + 63) / 64, stages = (steps + 3) / 4;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * EPI_WARPS); }
    mbar_init(shared_bar, EPI_WARPS);                                  // four warps of each CTA
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmA); prefetch_tmap(&tmB); prefetch_tmap(&tmSA); prefetch_tmap(&tmSB); }
  if (warp == 1) { tmem_alloc_pair(smem_u32(tmem_slot), 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  dependents_may_start();
  await_predecessor();
  const uint32_t tmem_base = *tmem_slot;
  auto acc_of = [&](int b) { return tmem_base + b * (BN - kOverlap); };

  if (warp < 4) {
    DIT_SETMAXNREG_DEC(REGS_ISSUE);
    if (warp == 0) {
      if (lane == 0) {
        int stage = 0; uint32_t phase = 0;
        for (int t = pair; t < num_tiles; t += num_pairs) {
          int mb, nb;
          tile_coords(t, num_m, num_n, p.band, mb, nb);
          const int m0 = mb * (2 * BM) + rank * BM, n0 = nb * BN + rank * (BN / 2);
          for (int k = 0; k < stages; ++k) {
            if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) goto done;
            const uint32_t full_leader = map_to_cta(full_bar(stage), 0);
            if (rank == 0) mbar_arrive_expect_tx(full_bar(stage), 2 * C::STAGE_BYTES);
            const uint32_t s = base + stage * C::STAGE_BYTES;
            tma_load_2d_pair(s, &tmA, k * 128, m0, full_leader);
            tma_load_2d_pair(s + A_BYTES, &tmB, k * 128, n0, full_leader);
            tma_load_3d_pair(s + A_BYTES + B_BYTES, &tmSA, 0, k * S::TILES, m0 >> 7, full_leader);
            tma_load_3d_pair(s + A_BYTES + B_BYTES + S::BYTES, &tmSB, 0, k * S::TILES, nb * 2, full_leader);   // all 256 columns' in either CTA
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      const bool issuer = elect_one();
      int stage = 0, slot = 0; uint32_t phase = 0;
      int n = 0;                                                       // tiles of this pair so far
      for (int t = pair; t < num_tiles; t += num_pairs, ++n) {
        const int buf = n & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(tempty_bar(buf), ((n >> 1) & 1u) ^ 1u, abort_flag) && mbar_wait(shared_bar, (n & 1u) ^ 1u, abort_flag))) goto done;
        const uint32_t acc = acc_of(buf);
        for (int k = 0; k < stages; ++k) {
          if (!__all_sync(0xffffffffu, mbar_wait(full_bar(stage), phase, abort_flag))) goto done;
          tc_fence_after();
          const uint32_t s = base + stage * C::STAGE_BYTES;
          const uint64_t adesc = smem_desc_sw128(s, 16, 1024), bdesc = smem_desc_sw128(s + A_BYTES, 16, 1024);
          const uint64_t sdesc = smem_desc_rows16(s + A_BYTES + B_BYTES);
          const int here = min(4, steps - 4 * k);
          if (issuer) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (i >= here) break;
              const int tile = i / S::STEPS, half = i % S::STEPS;
              if (half == 0) {                                         // the next scales, to the columns used longest ago
                if (++slot == C::SLOTS) slot = 0;
                const uint32_t at = tmem_base + 512 - kScaleCols + slot * C::SLOT;
                tmem_copy_scales<true>(at, sdesc + tile * (512 >> 4));
                tmem_copy_scales<true>(at + 4, sdesc + (S::BYTES + tile * 512 >> 4));
                tmem_copy_scales<true>(at + 8, sdesc + (2 * S::BYTES + tile * 512 >> 4));
              }
              const uint32_t at = tmem_base + 512 - kScaleCols + slot * C::SLOT;
              umma_fp4<kGroup, true>(acc, adesc + 2 * i, bdesc + 2 * i, half == 0 ? idesc_fp4<kGroup>(2 * BM, BN, 0) : idesc_fp4<kGroup>(2 * BM, BN, 2), at, at + 4,
                                     k > 0 || i > 0);
            }
            umma_commit_pair(empty_bar(stage), 3);
            if (k == stages - 1) umma_commit_pair(tfull_bar(buf), 3);
          }
          __syncwarp();
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else {
    DIT_SETMAXNREG_INC(REGS_EPILOGUE);
    const int quarter = warp & 3, chalf = (warp - 4) >> 2;
    const uint32_t lane_sel = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tempty_leader = map_to_cta(tempty_bar(0), 0), shared_leader = map_to_cta(shared_bar, 0);
    uint8_t* box = aligned + C::OFF_OUT + (warp - 4) * BOX_BYTES;
    float* col_of = reinterpret_cast<float*>(aligned + C::OFF_COL + chalf * COL_BYTES);      // factors, then bias
    bool ok = true;                            // after a failed wait the warps still meet at their barriers, tile after tile
    int n = 0;
    for (int t = pair; t < num_tiles; t += num_pairs, ++n) {
      const int buf = n & 1;
      int mb, nb;
      tile_coords(t, num_m, num_n, p.band, mb, nb);
      const int row0 = mb * (2 * BM) + rank * BM + quarter * 32, n0 = nb * BN + chalf * 128;
      const bool mine = n0 < p.N && row0 < p.M;                        // something of this warp's part exists (warp-uniform)
      const float fr = p.ra && row0 + lane < p.M ? p.ra[row0 + lane] : 1.f;
      {
        const int c = quarter * 32 + lane;                             // the four warps of these columns fetch 32 each
        const float f = p.rb && n0 + c < p.N ? p.rb[n0 + c] : 1.f, b = p.bias && n0 + c < p.N ? p.bias[n0 + c] : 0.f;
        asm volatile("bar.sync %0, 128;" ::"r"(1 + chalf) : "memory"); // the last tile's have been read
        col_of[c] = f;
        col_of[128 + c] = b;
        asm volatile("bar.sync %0, 128;" ::"r"(1 + chalf) : "memory");
      }
      ok = ok && __all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), (n >> 1) & 1u, abort_flag));
      if (!ok) continue;
      tc_fence_after();
      float2 acc[64];
      const uint32_t from = acc_of(buf) + lane_sel + chalf * 128;
      uint32_t* words = reinterpret_cast<uint32_t*>(acc);
      if (chalf != buf) {                                              // the accumulators share the second one's first and the first one's last 64 columns
        const int first = buf == 0 ? 64 : 0;
        if (first == 64) { tmem_ld32p(from + 64, words + 64); tmem_ld32p(from + 96, words + 96); }
        else { tmem_ld32p(from, words); tmem_ld32p(from + 32, words + 32); }
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_light(shared_leader);
        if (first == 64) { tmem_ld32p(from, words); tmem_ld32p(from + 32, words + 32); }
        else { tmem_ld32p(from + 64, words + 64); tmem_ld32p(from + 96, words + 96); }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32p(from + c * 32, words + c * 32);
      }
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_light(tempty_leader + 8u * buf);
      if (!mine) continue;                     // (its warps of the next tile wait at its column factors)
      // Whether a sum times the row's factor may be outside fp32's range.  Sums under e4m3 scales are 0 or 2^-20 .. 2^53 in size; under powers of two they
      // may be anything, and are looked through where there are factors.
      bool far = __any_sync(0xffffffffu, kGroup == 16 ? fabsf(fr) < 0x1p-100f || fabsf(fr) > 0x1p73f : fr != 1.f);
      if (kGroup == 32 && far) {
        uint32_t most = 0, least = 0xffffffffu;                        // of the sums' magnitudes, of those that are not zero (less one)
#pragma unroll
        for (int i = 0; i < 128; ++i) {
          most = max(most, words[i] & 0x7FFFFFFFu);
          least = min(least, (words[i] & 0x7FFFFFFFu) - 1);
        }
        const float size = fabsf(fr);
        far = __any_sync(0xffffffffu, !(__uint_as_float(most) * size < INFINITY) || (least != 0xffffffffu && __uint_as_float(least + 1) * size < 0x1p-126f));
      }
      if (far) {                                                       // by way of the box, 32 columns at a time: in registers alone it would spill
        if (lane == 0) bulk_store_read_done();
        __syncwarp();
        volatile float* line = reinterpret_cast<volatile float*>(box) + lane;                // the lane's own words
#pragma unroll
        for (int c = 0; c < 4; ++c) {
#pragma unroll
          for (int i = 0; i < 32; ++i) line[i * 32] = __uint_as_float(words[c * 32 + i]);
#pragma unroll 1
          for (int i0 = 0; i0 < 32; i0 += 4) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = line[(i0 + i) * 32];
#pragma unroll
            for (int i = 0; i < 4; ++i) line[(i0 + i) * 32] = fp4_finish(x[i], fr, col_of[c * 32 + i0 + i], col_of[128 + c * 32 + i0 + i]);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) words[c * 32 + i] = __float_as_uint(line[i * 32]);
        }
        __syncwarp();
      }
      // through shared memory, and out by TMA where rows start on 16-byte boundaries
      constexpr bool kWide = EPI == kBlkF32;
      constexpr bool kBf = EPI == kBlkBF16;
      constexpr int COLS = kWide ? 32 : 64;
#pragma unroll
      for (int round = 0; round < 128 / COLS; ++round) {
        if (!far) {                                                    // (row factor * sum) * column factor + bias
#pragma unroll
          for (int i = round * (COLS / 2); i < (round + 1) * (COLS / 2); i += 2) {
            const float4 f = *reinterpret_cast<const float4*>(col_of + 2 * i), b = *reinterpret_cast<const float4*>(col_of + 128 + 2 * i);
            const float2 r = make_float2(fr, fr);
            acc[i] = ffma2(fmul2(acc[i], r), make_float2(f.x, f.y), make_float2(b.x, b.y));
            acc[i + 1] = ffma2(fmul2(acc[i + 1], r), make_float2(f.z, f.w), make_float2(b.z, b.w));
          }
        }
        if (lane == 0) bulk_store_read_done();                         // the previous box has left
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          uint4 w;
          if constexpr (kWide) {
            const float2 a = acc[round * 16 + 2 * q], b = acc[round * 16 + 2 * q + 1];
            w = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
          } else {
            const float2* a = acc + round * 32 + 4 * q;
            w = make_uint4(pack16x2<kBf>(a[0].x, a[0].y), pack16x2<kBf>(a[1].x, a[1].y), pack16x2<kBf>(a[2].x, a[2].y), pack16x2<kBf>(a[3].x, a[3].y));
          }
          *reinterpret_cast<uint4*>(box + lane * 128 + ((q ^ (lane & 7)) << 4)) = w;
        }
        const int x = n0 + round * COLS;
        if (p.vec_out) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0 && x < p.N) {
            tma_store_2d_hint(&tmOut, smem_u32(box), x, row0, evict_first_policy());
            bulk_store_commit();
          }
        } else {
          __syncwarp();
          fp4_store_box<EPI>(p, box, lane, row0, x, min(COLS, p.N - x));
        }
      }
      __syncwarp();
    }
  }

done:
  bulk_store_done();                                                   // (threads that stored nothing pass at once)
  tc_fence_before();
  __syncthreads();
  settle_if_aborted(abort_flag);
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) { tc_fence_after(); tmem_dealloc_pair(tmem_base, 512); }
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusGemmTimeout);
}

// ------------------------------------------------------------------------------------------------
// Few rows, in tiles of BT = 16, 32 or 64: as in the 8-bit product the operands change roles, 128 rows of B (output columns) are the
// MMA's M and up to BT rows of A its N.  Reading B once is the bound: k is split over the CTAs of a cluster until the launch fills the
// device, each CTA adds its part up in tensor memory, and the partial sums meet in distributed shared memory, where rank r sums its share
// of the rows in rank order.  Scales come by plain bulk copies (a row tile's lie one after the other).  Row tiles start on multiples of BT
// inside a scale tile of 128 rows: 32-row tiles of scale words are a column each, so BT = 16 takes one row tile only.
// ------------------------------------------------------------------------------------------------
template <int BT, int kGroup>
struct Fp4SplitCfg {
  using S = Fp4Scales<kGroup>;
  static constexpr int W_BYTES = 128 * 128, T_BYTES = BT * 128;
  static constexpr int STAGE_BYTES = (W_BYTES + T_BYTES + 2 * S::BYTES + 1023) / 1024 * 1024;
  static constexpr int STAGES = BT <= 32 ? 4 : 3;                      // two CTAs per SM (one with twice the ring: 13.5 us where this takes 10.6)
  static constexpr int SLOT = 8, SLOTS = BT == 64 ? 8 : 7;             // scale columns in turn, behind the accumulator
  static constexpr int COLS = 128;
  static constexpr int OFF_BAR = STAGES * STAGE_BYTES, OFF_ROWS = OFF_BAR + 256;   // row factors [BT]
  static constexpr int SMEM_BYTES = OFF_ROWS + 256 + 1024;
  static constexpr int THREADS = 192;
  static_assert(BT + SLOT * SLOTS <= COLS, "tensor memory of one CTA");
  static_assert(BT * 128 * 4 <= STAGES * STAGE_BYTES, "the partial sums reuse the ring");
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
  static_assert(5 * SMEM_BYTES > 227 * 1024, "CTAs that fit an SM's shared memory must fit its tensor memory (4 x 128 columns)");
};

template <int EPI>
__device__ __forceinline__ void fp4_store_one(const Fp4GemmParams& p, int row, int col, float v) {
  const long long at = row * p.ld_out + col;
  if constexpr (EPI == kBlkF16) static_cast<uint16_t*>(p.out)[at] = pack16<false>(v);
  else if constexpr (EPI == kBlkBF16) static_cast<uint16_t*>(p.out)[at] = pack16<true>(v);
  else static_cast<float*>(p.out)[at] = v;
}

template <int EPI, int kGroup, int BT>
__global__ void __launch_bounds__(Fp4SplitCfg<BT, kGroup>::THREADS)
gemm_fp4_split_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const uint8_t* sa, const uint8_t* sb,
                      const Fp4GemmParams p, const int splits) {
  using C = Fp4SplitCfg<BT, kGroup>;
  using S = Fp4Scales<kGroup>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  const uint32_t tfull_bar = bar0 + 8u * (2 * C::STAGES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * (2 * C::STAGES + 1));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int tile = blockIdx.x / splits;
  const int num_n = (p.N + 127) >> 7;
  const int n0 = (tile % num_n) * 128, m0 = (tile / num_n) * BT;
  const int steps = (p.K + 63) / 64, stages = (steps + 3) / 4, chunks = (p.K + 4 * kGroup - 1) / (4 * kGroup);
  const int g0 = static_cast<int>(static_cast<long long>(stages) * rank / splits), g1 = static_cast<int>(static_cast<long long>(stages) * (rank + 1) / splits);

  // The producer's thread sets the barriers up and requests the first stages before tensor memory is there and the CTA meets.
  const uint8_t *wa = sb + static_cast<long long>(n0 >> 7) * chunks * 512, *ta = sa + static_cast<long long>(m0 >> 7) * chunks * 512;
  auto load = [&](int g, int stage) {
    const uint32_t s = base + stage * C::STAGE_BYTES;
    const uint32_t bytes = min(S::TILES, chunks - g * S::TILES) * 512;
    mbar_arrive_expect_tx(full_bar(stage), C::W_BYTES + C::T_BYTES + 2 * bytes);
    tma_load_2d(s, &tmB, g * 128, n0, full_bar(stage));
    tma_load_2d(s + C::W_BYTES, &tmA, g * 128, m0, full_bar(stage));
    bulk_load(s + C::W_BYTES + C::T_BYTES, wa + static_cast<long long>(g) * S::BYTES, bytes, full_bar(stage));
    bulk_load(s + C::W_BYTES + C::T_BYTES + S::BYTES, ta + static_cast<long long>(g) * S::BYTES, bytes, full_bar(stage));
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(tfull_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmA); prefetch_tmap(&tmB);
    await_predecessor();
    for (int s = 0; s < min(C::STAGES, g1 - g0); ++s) load(g0 + s, s);
  }
  if (warp == 1) { tmem_alloc(smem_u32(tmem_slot), C::COLS); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  dependents_may_start();                      // not before: a CTA of the next kernel that took the SM's tensor memory first would wait for this one's end
  const uint32_t tmem_base = *tmem_slot;
  const int quarter = warp & 3;                                        // warps 2..5 -> quarters 2, 3, 0, 1
  const int col = n0 + quarter * 32 + lane;                            // this lane's output column (warps 2..5)
  float* row_of = reinterpret_cast<float*>(aligned + C::OFF_ROWS);
  float fc = 1.f, bias = 0.f;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      for (int g = g0 + C::STAGES; g < g1; ++g) {
        if (!mbar_wait(empty_bar(stage), phase, abort_flag)) break;
        load(g, stage);
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0, slot = 0; uint32_t phase = 0;
      bool ok = true;
      const uint32_t sc0 = tmem_base + BT, word = (m0 & 127) >> 5;     // the row tile's first scale word
      for (int g = g0; g < g1; ++g) {
        if (!(ok = mbar_wait(full_bar(stage), phase, abort_flag))) break;
        tc_fence_after();
        const uint32_t s = base + stage * C::STAGE_BYTES;
        const uint64_t wdesc = smem_desc_sw128(s, 16, 1024), tdesc = smem_desc_sw128(s + C::W_BYTES, 16, 1024);
        const uint64_t sdesc = smem_desc_rows16(s + C::W_BYTES + C::T_BYTES);
        const int here = min(4, steps - 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= here) break;
          const int tl = i / S::STEPS, half = i % S::STEPS;
          if (half == 0) {
            if (++slot == C::SLOTS) slot = 0;
            tmem_copy_scales<false>(sc0 + slot * C::SLOT, sdesc + tl * (512 >> 4));
            tmem_copy_scales<false>(sc0 + slot * C::SLOT + 4, sdesc + (S::BYTES + tl * 512 >> 4));
          }
          umma_fp4<kGroup, false>(tmem_base, wdesc + 2 * i, tdesc + 2 * i, half == 0 ? idesc_fp4<kGroup>(128, BT, 0) : idesc_fp4<kGroup>(128, BT, 2),
                                  sc0 + slot * C::SLOT, sc0 + slot * C::SLOT + 4 + word, g > g0 || i > 0);
        }
        umma_commit(empty_bar(stage));
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
      if (ok) umma_commit(tfull_bar);
    }
  } else {
    // what the sums are finished with is fetched under the stream
    await_predecessor();
    const int row = threadIdx.x - 64;
    if (row < BT) row_of[row] = p.ra && m0 + row < p.M ? p.ra[m0 + row] : 1.f;
    if (col < p.N) {
      fc = p.rb ? p.rb[col] : 1.f;
      bias = p.bias ? p.bias[col] : 0.f;
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const bool ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar, 0, abort_flag));
    if (ok) {
      tc_fence_after();
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
      float* part = reinterpret_cast<float*>(aligned);                 // every MMA has completed: the sums may take the ring's place
#pragma unroll
      for (int c = 0; c < BT / 16; ++c) {
        uint32_t r[16];
        __syncwarp();
        tmem_ld16p(t_row + c * 16, r);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = c * 16 + i;
          if (splits > 1) {
            part[row * 128 + quarter * 32 + lane] = __uint_as_float(r[i]);
          } else if (col < p.N && m0 + row < p.M) {
            fp4_store_one<EPI>(p, m0 + row, col, fp4_finish(__uint_as_float(r[i]), row_of[row], fc, bias));
          }
        }
      }
    }
  }
  if (splits > 1) {
    __syncwarp();
    cluster_sync_all();                        // (a CTA that gave up may have copies under way: it settles below)
    if (warp >= 2 && col < p.N) {
      const int rows = min(BT, p.M - m0);
      const uint32_t mine = base + (quarter * 32 + lane) * 4;
      for (int i0 = rank; i0 < rows; i0 += 4 * splits) {               // four rows at a time: their loads are in flight together
        float v[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int r = 0; r < 8; ++r)
            v[k][r] = (r < splits && i0 + k * splits < rows) ? ld_cluster_f32(map_to_cta(mine + (i0 + k * splits) * 512, r)) : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float sum = 0.f;
#pragma unroll
          for (int r = 0; r < 8; ++r) sum += v[k][r];
          const int row = m0 + i0 + k * splits;
          if (i0 + k * splits < rows) fp4_store_one<EPI>(p, row, col, fp4_finish(sum, row_of[row - m0], fc, bias));
        }
      }
    }
    __syncwarp();
    cluster_sync_all();                                                // peers may still read this CTA's partials until here
  }
  tc_fence_before();
  __syncthreads();
  settle_if_aborted(abort_flag);
  __syncwarp();
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, C::COLS); }
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusGemmTimeout);
}

}  // namespace dit
