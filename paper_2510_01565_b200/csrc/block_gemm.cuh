// Product of two e4m3 operands with block scales for sm_100a:
//   C[m, n] = sum_g sa[g, m] * sb[n / 128, g] * (sum over the 128 k of group g of A[m, k] B[n, k])   (+ fused epilogue)
// Both operands are K-major.  The scales are general fp32 numbers, so the tensor cores cannot apply them:
// every group's partial tile is taken out of tensor memory and added to accumulators in registers with
// one packed multiply-add per pair.  That costs the epilogue warps 128 x 256 values per 128 k of a
// CTA's half of a 256 x 256 tile, 512 cycles of the tensor pipe, against about 256 cycles of
// tensor-memory reads and 256 of multiply-adds that run beside each other: tensor memory holds two
// partial tiles, so the next group's MMAs run while the last one's sums are added.
//
// Two kernels.  gemm_block128_pair_kernel: persistent, one 256 x 256 tile per CTA pair, for shapes with
// enough tiles.  gemm_block128_split_kernel: 128 output columns x up to 64 rows per CTA, k split over a
// cluster and joined through distributed shared memory in rank order, for few rows, where reading B once is
// the bound.
//
// Measured (pair kernel, m 16896, n 12288, k 3072, fp16 out): 568 us = 2.25 PFLOP/s in a single call, 640-690 us in long runs under
// the power cap.  Trial builds of the same kernel with parts left out, in short runs of 577 us: no additions 496 us, no tensor-memory
// reads 539 us, neither 490 us, a quarter of the MMAs 502 us.  So what remains at 490 us is the way of the operands into this
// kernel's ring (64 KB per group and pair, 10 TB/s over the device), and reads and additions beside it cost 15 %.  It is not a
// limit of L2: the 16-bit product on the same tile, with six stages, takes in 12.4 TB/s.  Four stages (64 KB stage the outputs) and a
// stage given back after two commits are the differences; which of them counts has not been measured.
// Split kernel, m 1, n 18432, k 3072 (57 MB of weights): 10.7 us when they are in L2, 16.1 us (3.5 TB/s) from DRAM.
#pragma once
#include "common.cuh"
#include "gemm.cuh"
#include "ptx.cuh"

namespace dit {

// kBlkF16 / kBlkBF16 / kBlkF32: out = acc + bias in that type.
// kBlkGeluF16: out = gelu_tanh(acc + bias) as fp16.  kBlkGateResidF32: out = resid + gate[request(row)] * (acc + bias).
enum BlockGemmEpilogue : int { kBlkF16 = 0, kBlkBF16 = 1, kBlkF32 = 2, kBlkGeluF16 = 3, kBlkGateResidF32 = 4 };

struct BlockGemmParams {
  int M, N, K;
  int band;                  // tile order, see tile_coords
  const float* sa;           // [groups, ld_sa]
  const float* sb;           // [ceil(N / 128), groups]
  const float* bias;         // [N] or NULL
  void* out;                 // row stride ld_out elements
  long long ld_sa, ld_out;
  int vec_out;               // rows of out start on 16-byte boundaries
  int* status;
  // kBlkGateResidF32 only (row strides of resid and out are ld_out)
  int row0;                  // packed row index of row 0 (a launch may cover a slice of the batch's rows)
  const float* resid;
  const float* gate;         // gate vector of request 0; request r at gate + r * gate_stride
  long long gate_stride;
};

namespace bgemm {
constexpr int BM = 128, BN = 256;
constexpr int A_BYTES = BM * 128, B_BYTES = (BN / 2) * 128;
constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 128 + 32 * EPI_WARPS;
constexpr int REGS_ISSUE = 56, REGS_EPILOGUE = 224;   // (56 + 2 * 224) * 32 <= 16384 per scheduler
constexpr int BOX_BYTES = 4096;                       // 128 bytes x 32 rows of the output
// Per epilogue warp: two boxes of its 32 rows, or, where a residual is added, all four of its 32 rows x 128 fp32 columns: the
// residual arrives there by TMA during the main loop and is replaced by the result in place.  Three stages of operands
// are left room for then instead of four (five and six measured no faster than four).
template <int EPI>
struct Cfg {
  static constexpr bool kResid = EPI == kBlkGateResidF32;
  static constexpr int STAGES = kResid ? 3 : 4;
  static constexpr int STAGE_OUT_BYTES = (kResid ? 4 : 2) * BOX_BYTES;
  static constexpr int BIAS_BYTES = kResid ? 0 : 512;         // the bias of the warp's 128 columns
  static constexpr int OFF_OUT = STAGES * STAGE_BYTES, OFF_BAR = OFF_OUT + EPI_WARPS * (STAGE_OUT_BYTES + BIAS_BYTES);
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};
}  // namespace bgemm

// Writes a warp's 32 rows x 128 columns (this lane's row in acc) to an output whose rows start off 16-byte boundaries, which TMA cannot
// address: through `stage` (16-byte units XOR-swizzled by the row), then row by row in 32-bit words.  A 16-bit row that
// starts in the middle of a word is shifted by one element on the way (a whole warp works on one row, so nothing
// diverges), its first and last element may go out alone.  m 4000, n 4001, k 1000: fp16 39 us, fp32 35, against 26 and 31 for
// n 4000 (42 and 39 with an element per lane and store, 43 and 37 row by row without the batches, 61 and 68 in 16-byte
// segments put together by each lane): the stores hold the warps where TMA would not.
template <int EPI>
__device__ __forceinline__ void block_store_unaligned(const BlockGemmParams& p, uint8_t* stage, const float2 (&acc)[64], int lane, int row0, int n0) {
  constexpr bool kWide = EPI == kBlkF32;
  constexpr bool kBf = EPI == kBlkBF16;
  constexpr int ROUNDS = kWide ? 2 : 1, COLS = 128 / ROUNDS;          // 64 words of a row at a time
  auto word = [&](int r, int w) { return *reinterpret_cast<const uint32_t*>(stage + r * 256 + ((((w >> 2) ^ (r & 15)) << 4) | ((w & 3) << 2))); };
#pragma unroll
  for (int round = 0; round < ROUNDS; ++round) {
    const int c0 = n0 + round * COLS, cols = min(COLS, p.N - c0);      // may be <= 0
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      uint4 w;
      if constexpr (kWide) {
        const float2 a = acc[round * 32 + 2 * q], b = acc[round * 32 + 2 * q + 1];
        w = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
      } else {
        w = make_uint4(pack16x2<kBf>(acc[4 * q].x, acc[4 * q].y), pack16x2<kBf>(acc[4 * q + 1].x, acc[4 * q + 1].y),
                       pack16x2<kBf>(acc[4 * q + 2].x, acc[4 * q + 2].y), pack16x2<kBf>(acc[4 * q + 3].x, acc[4 * q + 3].y));
      }
      *reinterpret_cast<uint4*>(stage + lane * 256 + ((q ^ (lane & 15)) << 4)) = w;
    }
    __syncwarp();
    const int rows = min(32, p.M - row0);
    constexpr int BATCH = 8;                   // rows whose words are read before the first is written
    for (int r0 = 0; r0 < rows; r0 += BATCH) {
      uint32_t v[BATCH][2];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) { v[k][0] = word(r0 + k, lane); v[k][1] = word(r0 + k, 32 + lane); }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (r0 + k >= rows) break;
        const long long first = (static_cast<long long>(row0) + r0 + k) * p.ld_out + c0;
        if constexpr (kWide) {
          float* at = static_cast<float*>(p.out) + first;
          if (lane < cols) at[lane] = __uint_as_float(v[k][0]);
          if (32 + lane < cols) at[32 + lane] = __uint_as_float(v[k][1]);
        } else {
          uint16_t* at = static_cast<uint16_t*>(p.out) + first;
          if ((reinterpret_cast<uintptr_t>(at) >> 1) & 1) {            // the row starts in the middle of a word (warp-uniform)
            if (lane == 0 && cols > 0) at[0] = static_cast<uint16_t>(v[k][0]);
            const uint32_t wrap = __shfl_sync(0xffffffffu, v[k][1], 0);
            uint32_t n0 = __shfl_down_sync(0xffffffffu, v[k][0], 1), n1 = __shfl_down_sync(0xffffffffu, v[k][1], 1);
            if (lane == 31) n0 = wrap;
            v[k][0] = __funnelshift_r(v[k][0], n0, 16); v[k][1] = __funnelshift_r(v[k][1], n1, 16);
            ++at;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = 2 * (h * 32 + lane);
              if (c + 2 < cols) *reinterpret_cast<uint32_t*>(at + c) = v[k][h];
              else if (c + 1 < cols) at[c] = static_cast<uint16_t>(v[k][h]);
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = 2 * (h * 32 + lane);
              if (c + 1 < cols) *reinterpret_cast<uint32_t*>(at + c) = v[k][h];
              else if (c < cols) at[c] = static_cast<uint16_t>(v[k][h]);
            }
          }
        }
      }
    }
    __syncwarp();
  }
}

// Roles: warp 0 TMA producer, warps 1 and 2 MMA issuers (leader CTA; warp 1 owns tensor memory), warps 4..11 accumulate and
// write: two per quarter of the tile's rows, one for each 128 columns (so a warp's columns share one scale of B per
// group, and a lane's row one scale of A).
// A group's partial tile is made and taken out in two halves: half h multiplies rows 64 h .. 64 h + 63 of each CTA's
// B box, i.e. columns 64 h.. of both scale blocks.  Tensor memory holds two groups x two halves: a half's round
// trip (MMAs, commit, wake-up, read-out, arrival at the leader: about 1100 cycles, of which 256 are MMAs) then fits
// under the other three, which it did not with two whole partial tiles (900 cycles per group measured).  Issuer h owns half h;
// its commit reports both that its part of the stage has been read and that the half is complete: producer and
// accumulating warps wait on the same barrier.
template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(bgemm::THREADS, 1)
gemm_block128_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                          const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmResid, const BlockGemmParams p,
                          const __grid_constant__ SeqInfo seq) {
  using namespace bgemm;
  using C = Cfg<EPI>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto done_bar = [&](int s, int h) { return bar0 + 8u * (STAGES + 2 * s + h); };      // half h's MMAs of stage s have completed
  auto tempty_bar = [&](int buf, int h) { return bar0 + 8u * (3 * STAGES + 2 * buf + h); };
  auto resid_bar = [&](int w) { return bar0 + 8u * (3 * STAGES + 4 + w); };            // epilogue warp w's residual rows have arrived
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * (3 * STAGES + 4 + EPI_WARPS));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int num_m = (p.M + 2 * BM - 1) / (2 * BM), num_n = (p.N + BN - 1) / BN;
  const int num_tiles = num_m * num_n;
  const int groups = (p.K + 127) / 128;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(done_bar(s, 0), 1); mbar_init(done_bar(s, 1), 1); }
    for (int a = 0; a < 4; ++a) mbar_init(tempty_bar(a >> 1, a & 1), 2 * EPI_WARPS);
    for (int w = 0; w < EPI_WARPS; ++w) mbar_init(resid_bar(w), 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmA); prefetch_tmap(&tmB); }
  if (warp == 1) { tmem_alloc_pair(smem_u32(tmem_slot), 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp < 4) {
    DIT_SETMAXNREG_DEC(REGS_ISSUE);
    if (warp == 0) {
      if (lane == 0) {
        int stage = 0; uint32_t phase = 0;
        for (int t = pair; t < num_tiles; t += num_pairs) {
          int mb, nb;
          tile_coords(t, num_m, num_n, p.band, mb, nb);
          const int m0 = mb * (2 * BM) + rank * BM, n0 = nb * BN + rank * (BN / 2);
          for (int g = 0; g < groups; ++g) {
            if (!mbar_wait(done_bar(stage, 0), phase ^ 1u, abort_flag) || !mbar_wait(done_bar(stage, 1), phase ^ 1u, abort_flag)) goto done;
            const uint32_t full_leader = map_to_cta(full_bar(stage), 0);
            if (rank == 0) mbar_arrive_expect_tx(full_bar(stage), 2 * STAGE_BYTES);
            const uint32_t sa = base + stage * STAGE_BYTES;
            tma_load_2d_pair(sa, &tmA, g * 128, m0, full_leader);
            tma_load_2d_pair(sa + A_BYTES, &tmB, g * 128, n0, full_leader);
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
        }
      }
    } else if (warp < 3 && rank == 0) {
      // the whole warp runs the loop, so that descriptors and addresses live in uniform registers; one thread issues
      constexpr uint32_t idesc = idesc_e4m3(2 * BM, BN / 2);
      const int h = warp - 1;
      const bool issuer = elect_one();
      const int uses = groups * ((num_tiles - pair + num_pairs - 1) / num_pairs);
      int stage = 0; uint32_t phase = 0;
      for (int use = 0; use < uses; ++use) {                           // partial tiles of this pair, in order
        const int buf = use & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(tempty_bar(buf, h), ((use >> 1) & 1u) ^ 1u, abort_flag) && mbar_wait(full_bar(stage), phase, abort_flag))) goto done;
        tc_fence_after();
        const uint32_t sa = base + stage * STAGE_BYTES;
        const uint64_t adesc = smem_desc_sw128(sa, 16, 1024), bdesc = smem_desc_sw128(sa + A_BYTES + h * (B_BYTES / 2), 16, 1024);
        if (issuer) {
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_f8_pair(tmem_base + buf * BN + h * (BN / 2), adesc + 2 * k, bdesc + 2 * k, idesc, k != 0);
          umma_commit_pair(done_bar(stage, h), 3);                     // in both CTAs
        }
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else {
    DIT_SETMAXNREG_INC(REGS_EPILOGUE);
    const int quarter = warp & 3, chalf = (warp - 4) >> 2;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + chalf * 64;
    const uint32_t tempty_leader = map_to_cta(tempty_bar(0, 0), 0);
    uint8_t* stage = aligned + C::OFF_OUT + (warp - 4) * C::STAGE_OUT_BYTES;
    float* bias_of = reinterpret_cast<float*>(aligned + C::OFF_OUT + EPI_WARPS * C::STAGE_OUT_BYTES + (warp - 4) * C::BIAS_BYTES);
    uint32_t resid_phase = 0;
    // What a tile needs from memory before its first group: requested for the next tile before the current one is
    // written.  Lane l holds the bias of columns l, 32 + l, 64 + l, 96 + l; scales run two groups ahead of their use.
    struct Ahead { int row0, n0; const float *sa, *sb; float bias[4], sa_at[3], sb_at[3]; } next;
    auto request = [&](int t) {
      int mb, nb;
      tile_coords(t, num_m, num_n, p.band, mb, nb);
      next.row0 = mb * (2 * BM) + rank * BM + quarter * 32; next.n0 = nb * BN + chalf * 128;
      next.sa = p.sa + (next.row0 + lane < p.M ? next.row0 + lane : 0);
      next.sb = p.sb + static_cast<long long>(next.n0 < p.N ? next.n0 >> 7 : 0) * groups;
#pragma unroll
      for (int c = 0; c < 4; ++c) next.bias[c] = (!C::kResid && p.bias && next.n0 + c * 32 + lane < p.N) ? __ldg(p.bias + next.n0 + c * 32 + lane) : 0.f;
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int at = min(d, groups - 1);
        next.sa_at[d] = __ldg(next.sa + at * p.ld_sa); next.sb_at[d] = __ldg(next.sb + at);
      }
    };
    int stage_of = 0; uint32_t phase = 0; int buf = 0;                 // of the next group
    bool ready = false;                                                // its first half is known to be complete
    if (pair < num_tiles) request(pair);
    for (int t = pair; t < num_tiles; t += num_pairs) {
      const int row0 = next.row0, n0 = next.n0;
      const float *sa = next.sa, *sb = next.sb;
      float sa_at[3] = {next.sa_at[0], next.sa_at[1], 0.f}, sb_at[3] = {next.sb_at[0], next.sb_at[1], 0.f};
      const bool mine = n0 < p.N && row0 < p.M;                        // something of this warp's part exists (warp-uniform)
      if constexpr (C::kResid) {
        if (mine && lane == 0) {
          bulk_store_read_done();                                      // the previous tile's rows have left
          mbar_arrive_expect_tx(resid_bar(warp - 4), 4 * BOX_BYTES);
          for (int c = 0; c < 4; ++c) tma_load_2d(smem_u32(stage) + c * BOX_BYTES, &tmResid, n0 + c * 32, row0, resid_bar(warp - 4));
        }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) bias_of[c * 32 + lane] = next.bias[c];
      }
      float2 acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.f, 0.f);
      // A group's half is read out in two pieces of 32 columns; the next piece is on its way (into the other buffer)
      // while one is added.  Piece by piece with nothing ahead, waits, reads and additions of a half took about 550 cycles
      // one after the other, and with two warps per scheduler these, not the MMAs, set the pace.
      uint32_t ra[32], rb[32];
      auto await = [&](int h) { return __all_sync(0xffffffffu, ready || mbar_wait(done_bar(stage_of, h), phase, abort_flag)); };
      auto fetch = [&](int h, int piece, uint32_t (&r)[32]) { tmem_ld32(t_row + buf * BN + h * 128 + piece * 32, r); };
      auto release = [&](int h) {              // the half is in registers: hand its columns back
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_light(tempty_leader + 8u * (2 * buf + h));
      };
      if (!await(0)) goto done;
      tc_fence_after();
      fetch(0, 0, ra);
      tmem_ld_wait();
      for (int g = 0; g < groups; ++g) {
        {
          const int at = min(g + 2, groups - 1);
          sa_at[2] = __ldg(sa + at * p.ld_sa); sb_at[2] = __ldg(sb + at);
        }
        const float fs = sa_at[0] * sb_at[0];
        const float2 f = make_float2(fs, fs);
        auto add = [&](const uint32_t (&r)[32], int first) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            ffma2_here(acc[first + i], make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), f);
        };
        fetch(0, 1, rb);
        add(ra, 0);
        tmem_ld_wait();
        release(0);
        ready = mbar_test_wait(done_bar(stage_of, 1), phase);
        if (!await(1)) goto done;
        tc_fence_after();
        fetch(1, 0, ra);
        add(rb, 16);
        tmem_ld_wait();
        fetch(1, 1, rb);
        add(ra, 32);
        tmem_ld_wait();
        release(1);
        if (++stage_of == STAGES) { stage_of = 0; phase ^= 1u; }
        buf ^= 1;
        ready = mbar_test_wait(done_bar(stage_of, 0), phase);
        if (g + 1 < groups) {
          if (!await(0)) goto done;
          tc_fence_after();
          fetch(0, 0, ra);
        }
        add(rb, 48);
        tmem_ld_wait();
#pragma unroll
        for (int d = 0; d < 2; ++d) { sa_at[d] = sa_at[d + 1]; sb_at[d] = sb_at[d + 1]; }
      }
      if (t + num_pairs < num_tiles) request(t + num_pairs);
      if (!mine) continue;
      if constexpr (C::kResid) {
        // out = resid + gate (acc + bias), where the residual lies in the boxes: column 32 c + 4 q of the lane's row in 16-byte unit q of box c
        const int row = row0 + lane;
        const float* gate = p.gate + (row < p.M ? find_request(seq, p.row0 + row) : 0) * p.gate_stride + n0;
        if (!__all_sync(0xffffffffu, mbar_wait(resid_bar(warp - 4), resid_phase, abort_flag))) goto done;
        resid_phase ^= 1u;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (n0 + c * 32 >= p.N) break;                               // warp-uniform; N is a multiple of 32 here
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int at = c * 32 + q * 4;
            const float4 g = __ldg(reinterpret_cast<const float4*>(gate + at));
            const float4 b = p.bias ? __ldg(reinterpret_cast<const float4*>(p.bias + n0 + at)) : make_float4(0.f, 0.f, 0.f, 0.f);
            float4* cell = reinterpret_cast<float4*>(stage + c * BOX_BYTES + lane * 128 + ((q ^ (lane & 7)) << 4));
            const float4 x = *cell;
            const float2 lo = fadd2(acc[at / 2], make_float2(b.x, b.y)), hi = fadd2(acc[at / 2 + 1], make_float2(b.z, b.w));
            const float2 o0 = ffma2(make_float2(g.x, g.y), lo, make_float2(x.x, x.y)), o1 = ffma2(make_float2(g.z, g.w), hi, make_float2(x.z, x.w));
            *cell = make_float4(o0.x, o0.y, o1.x, o1.y);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          for (int c = 0; c < 4; ++c)
            if (n0 + c * 32 < p.N) tma_store_2d(&tmOut, smem_u32(stage) + c * BOX_BYTES, n0 + c * 32, row0);
          bulk_store_commit();
        }
        __syncwarp();
        continue;
      }
      __syncwarp();                                                    // bias_of is complete
      auto finished = [&](int i) {                                     // columns 2i .. 2i + 3 of the warp's 128, i even
        const float4 b4 = *reinterpret_cast<const float4*>(bias_of + 2 * i);
        const float2 lo = fadd2(acc[i], make_float2(b4.x, b4.y)), hi = fadd2(acc[i + 1], make_float2(b4.z, b4.w));
        return make_float4(lo.x, lo.y, hi.x, hi.y);
      };
      if constexpr (!C::kResid) {
      if (p.vec_out) {
        // Through shared memory and out by TMA: the warp is free again as soon as its rows lie there, and what lies
        // outside the matrix is dropped.  A box is 128 bytes x 32 rows, 16-byte units XOR-swizzled by the row.
        constexpr bool kWide = EPI == kBlkF32;
        constexpr int COLS = kWide ? 32 : 64;                          // columns per box; two boxes per round
#pragma unroll
        for (int round = 0; round < (kWide ? 2 : 1); ++round) {
          if (lane == 0) bulk_store_read_done();                       // the previous boxes have left
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            uint4 w;
            if constexpr (kWide) {
              const float4 v = finished(round * 32 + 2 * q);
              w = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
            } else {
              float4 a = finished(4 * q), b = finished(4 * q + 2);
              if (EPI == kBlkGeluF16) {
                float2 t0 = gelu_tanh_f32x2(make_float2(a.x, a.y)), t1 = gelu_tanh_f32x2(make_float2(a.z, a.w));
                a = make_float4(t0.x, t0.y, t1.x, t1.y);
                t0 = gelu_tanh_f32x2(make_float2(b.x, b.y)); t1 = gelu_tanh_f32x2(make_float2(b.z, b.w));
                b = make_float4(t0.x, t0.y, t1.x, t1.y);
              }
              constexpr bool kBf = EPI == kBlkBF16;
              w = make_uint4(pack16x2<kBf>(a.x, a.y), pack16x2<kBf>(a.z, a.w), pack16x2<kBf>(b.x, b.y), pack16x2<kBf>(b.z, b.w));
            }
            *reinterpret_cast<uint4*>(stage + (q >> 3) * 4096 + lane * 128 + (((q & 7) ^ (lane & 7)) << 4)) = w;
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int x = n0 + round * 2 * COLS;
            if (x < p.N) tma_store_2d(&tmOut, smem_u32(stage), x, row0);
            if (x + COLS < p.N) tma_store_2d(&tmOut, smem_u32(stage) + 4096, x + COLS, row0);
            bulk_store_commit();
          }
        }
        __syncwarp();
        continue;
      }
      if constexpr (EPI != kBlkGeluF16) {                              // (always vec_out there)
        if (p.bias) {
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const float4 v = finished(i);
            acc[i] = make_float2(v.x, v.y); acc[i + 1] = make_float2(v.z, v.w);
          }
        }
        block_store_unaligned<EPI>(p, stage, acc, lane, row0, n0);
      }
      }
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
// Few rows, in tiles of BT = 16, 32 or 64 (128 lost to two of 64 at every size: one CTA per SM).  The roles of the operands are
// swapped: 128 rows of B (output columns) are the MMA's M, up to BT rows of A its N, so that a lane owns one output column and the MMA wastes nothing on absent rows beyond the rounding to 16.
// Reading B once is the bound (1 byte per 2 M flops): the k groups are split over the CTAs of a cluster until the
// launch fills the device, each CTA streams its part through a ring of TMA boxes, and the partial
// accumulators meet in distributed shared memory, where rank r sums its share of the rows in rank order.
// Two CTAs fit on an SM (shared memory and tensor memory alike), so one CTA's set-up and join run under the
// other's stream.
// ------------------------------------------------------------------------------------------------
template <int BT>
struct SplitCfg {
  static constexpr int A_BYTES = 128 * 128, T_BYTES = BT * 128, STAGE_BYTES = A_BYTES + T_BYTES;
  static constexpr int STAGES = BT <= 32 ? 5 : 4;
  static constexpr int BUFS = 4;                                       // partial tiles in tensor memory
  static constexpr int COLS = BUFS * BT;                               // 64, 128, 256
  static constexpr int SCALE_GROUPS = 8;                               // groups of row scales staged at a time
  static constexpr int OFF_SCALE = STAGES * STAGE_BYTES;
  static constexpr int OFF_BAR = OFF_SCALE + 2 * SCALE_GROUPS * BT * 4;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  static constexpr int THREADS = 192;
  static_assert(BT * 128 * 4 <= STAGES * STAGE_BYTES, "the partial accumulators reuse the ring");
  static_assert(3 * SMEM_BYTES > 227 * 1024 || 3 * COLS <= 512, "CTAs that fit an SM's shared memory must fit its tensor memory");
  static_assert(2 * COLS <= 512 && 4 * SMEM_BYTES > 227 * 1024, "at most three CTAs per SM");
};

template <int EPI>
__device__ __forceinline__ void block_store_one(const BlockGemmParams& p, const SeqInfo& seq, int row, int col, float v) {
  const long long at = row * p.ld_out + col;
  if constexpr (EPI == kBlkF16) static_cast<uint16_t*>(p.out)[at] = pack16<false>(v);
  else if constexpr (EPI == kBlkBF16) static_cast<uint16_t*>(p.out)[at] = pack16<true>(v);
  else if constexpr (EPI == kBlkGeluF16) static_cast<uint16_t*>(p.out)[at] = pack16<false>(gelu_tanh_f32(v));
  else if constexpr (EPI == kBlkF32) static_cast<float*>(p.out)[at] = v;
  else static_cast<float*>(p.out)[at] = fmaf(p.gate[find_request(seq, p.row0 + row) * p.gate_stride + col], v, p.resid[at]);
}

template <int EPI, int BT>
__global__ void __launch_bounds__(SplitCfg<BT>::THREADS)
gemm_block128_split_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const BlockGemmParams p,
                           const __grid_constant__ SeqInfo seq, const int splits) {
  using C = SplitCfg<BT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * C::STAGES + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * C::STAGES + C::BUFS + b); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * (2 * C::STAGES + 2 * C::BUFS));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int tile = blockIdx.x / splits;
  const int num_n = (p.N + 127) >> 7;
  const int n0 = (tile % num_n) * 128, m0 = (tile / num_n) * BT;
  const int groups = (p.K + 127) / 128;
  const int g0 = static_cast<int>(static_cast<long long>(groups) * rank / splits), g1 = static_cast<int>(static_cast<long long>(groups) * (rank + 1) / splits);

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < C::BUFS; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 4); }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmA); prefetch_tmap(&tmB); }
  if (warp == 1) { tmem_alloc(smem_u32(tmem_slot), C::COLS); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  float acc[BT];
  const int quarter = warp & 3;                                        // warps 2..5 -> quarters 2, 3, 0, 1
  const int col = n0 + quarter * 32 + lane;                            // this lane's output column (warps 2..5)
#pragma unroll
  for (int i = 0; i < BT; ++i) acc[i] = 0.f;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      for (int g = g0; g < g1; ++g) {
        if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) break;
        const uint32_t s = base + stage * C::STAGE_BYTES;
        mbar_arrive_expect_tx(full_bar(stage), C::STAGE_BYTES);
        tma_load_2d(s, &tmB, g * 128, n0, full_bar(stage));
        tma_load_2d(s + C::A_BYTES, &tmA, g * 128, m0, full_bar(stage));
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_e4m3(128, BT);
      int stage = 0; uint32_t phase = 0;
      for (int g = g0; g < g1; ++g) {
        const int use = g - g0, buf = use % C::BUFS;
        if (!mbar_wait(tempty_bar(buf), ((use / C::BUFS) & 1u) ^ 1u, abort_flag)) break;
        if (!mbar_wait(full_bar(stage), phase, abort_flag)) break;
        tc_fence_after();
        const uint32_t s = base + stage * C::STAGE_BYTES;
        const uint64_t wdesc = smem_desc_sw128(s, 16, 1024), tdesc = smem_desc_sw128(s + C::A_BYTES, 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k) umma_f8(tmem_base + buf * BT, wdesc + 2 * k, tdesc + 2 * k, idesc, k != 0);
        umma_commit(empty_bar(stage));
        umma_commit(tfull_bar(buf));
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else {
    const float* sb = p.sb + static_cast<long long>(n0 >> 7) * groups;
    float* scales = reinterpret_cast<float*>(aligned + C::OFF_SCALE);  // [2][SCALE_GROUPS][BT]: sa * sb of the coming groups
    const int et = threadIdx.x - 64;
    auto stage_scales = [&](int first) {                               // groups first .. first + 7 into their half
      float* dst = scales + (((first - g0) / C::SCALE_GROUPS) & 1) * C::SCALE_GROUPS * BT;
      for (int i = et; i < C::SCALE_GROUPS * BT; i += 128) {
        const int g = first + i / BT, m = m0 + i % BT;
        dst[i] = (g < g1 && m < p.M) ? __ldg(p.sa + g * p.ld_sa + m) * __ldg(sb + g) : 0.f;
      }
    };
    stage_scales(g0);
    bool ok = true;
    for (int g = g0; g < g1; ++g) {                                    // after a failed wait the warps still meet at their barrier
      const int use = g - g0, buf = use % C::BUFS, in = use % C::SCALE_GROUPS;
      if (in == 0) {
        asm volatile("bar.sync 1, 128;" ::: "memory");                 // this half is written, the other one read
        if (g + C::SCALE_GROUPS < g1) stage_scales(g + C::SCALE_GROUPS);
      }
      const float* sc = scales + ((use / C::SCALE_GROUPS) & 1) * C::SCALE_GROUPS * BT + in * BT;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), (use / C::BUFS) & 1u, abort_flag));
      if (!ok) continue;
      tc_fence_after();
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + buf * BT;
      constexpr int CH = BT < 32 ? BT : 32;
#pragma unroll
      for (int c = 0; c < BT / CH; ++c) {
        uint32_t r[CH];
        __syncwarp();
        if constexpr (CH == 16) tmem_ld16p(t_row + c * CH, r); else tmem_ld32p(t_row + c * CH, r);
        tmem_ld_wait();
        if (c == BT / CH - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(tempty_bar(buf));
        }
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
          const float4 s = *reinterpret_cast<const float4*>(sc + c * CH + i);
          acc[c * CH + i] = fmaf(__uint_as_float(r[i]), s.x, acc[c * CH + i]);
          acc[c * CH + i + 1] = fmaf(__uint_as_float(r[i + 1]), s.y, acc[c * CH + i + 1]);
          acc[c * CH + i + 2] = fmaf(__uint_as_float(r[i + 2]), s.z, acc[c * CH + i + 2]);
          acc[c * CH + i + 3] = fmaf(__uint_as_float(r[i + 3]), s.w, acc[c * CH + i + 3]);
        }
      }
    }
    const float bias = (p.bias && col < p.N) ? __ldg(p.bias + col) : 0.f;
    if (splits == 1) {
      if (ok && col < p.N) {
#pragma unroll
        for (int i = 0; i < BT; ++i)
          if (m0 + i < p.M) block_store_one<EPI>(p, seq, m0 + i, col, acc[i] + bias);
      }
    } else if (ok) {
      // every MMA of this CTA has completed and with it every read of the ring: the partials may take its place
      float* part = reinterpret_cast<float*>(aligned);
#pragma unroll
      for (int i = 0; i < BT; ++i) part[i * 128 + quarter * 32 + lane] = acc[i];
    }
  }
  if (splits > 1) {
    __syncwarp();
    cluster_sync_all();                        // (a CTA that gave up may have copies under way: it settles below)
    if (warp >= 2 && col < p.N) {
      const float bias = p.bias ? __ldg(p.bias + col) : 0.f;
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
          float sum = bias;
#pragma unroll
          for (int r = 0; r < 8; ++r) sum += v[k][r];
          if (i0 + k * splits < rows) block_store_one<EPI>(p, seq, m0 + i0 + k * splits, col, sum);
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
