// Attention over selected key blocks (128 rows each), and the selection by the product of block means.
//
// block_attention_kernel   256 query rows of a head per CTA on the tensor cores, for query blocks of many rows
// block_rows_kernel        up to 16 query rows of a head per cluster, for a few rows that read a long context
// block_means_kernel, block_select_kernel   the selector
#pragma once
#include <type_traits>

#include "attention.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

// Packed batch with separate query and key lengths, passed by value.  `order` lists requests by query rows, most first.
struct BlockBatch {
  int n;
  int cu_q[DIT_MAX_REQUESTS + 1], cu_kv[DIT_MAX_REQUESTS + 1];
  int first_qblock[DIT_MAX_REQUESTS + 1], first_kblock[DIT_MAX_REQUESTS + 1];
  int order[DIT_MAX_REQUESTS];
};

struct BlockAttnParams {
  void* out;
  long long ld_out;
  const int* index;          // [heads, query blocks, ld_index]
  const int* count;          // [heads, query blocks]
  long long ld_index;
  int n_heads;
  float scale_log2;          // scale * log2(e), positive
  int items;                 // (request, head, 256 query rows) triples
  int wide_out;              // rows of out start on 32-byte boundaries
  int clamp;                 // infinite results become the largest finite value (steps, whose activations all do)
  int* status;
};

// Results are packed with finite values clamped (rounded probabilities may add up to a little more than one, and a value at the
// format's limit must not leave it); an infinite result stays one.
template <bool BF16>
__device__ __forceinline__ uint32_t infinity_bits(float x) { return (BF16 ? 0x7F80u : 0x7C00u) | (x < 0.f ? 0x8000u : 0u); }
template <bool BF16>
__device__ __forceinline__ uint32_t put_infinities(uint32_t packed, float lo, float hi) {
  if (fabsf(lo) == INFINITY) packed = (packed & 0xFFFF0000u) | infinity_bits<BF16>(lo);
  if (fabsf(hi) == INFINITY) packed = (packed & 0x0000FFFFu) | infinity_bits<BF16>(hi) << 16;
  return packed;
}

constexpr int kWindowBlocks = 256;      // key blocks whose lists are laid out in shared memory at a time
constexpr int kMaxKeyBlocks = 16384;    // of one request

template <int D>
struct BlockAttnCfg {
  static constexpr int NP = D / 64, PANEL = 128 * 128, TILE_BYTES = NP * PANEL;
  static constexpr int K_STAGES = 3, V_STAGES = 2;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + K_STAGES * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_V + V_STAGES * TILE_BYTES;
  static constexpr int OFF_BITS = OFF_BAR + 256;                                  // uint32 [2][kWindowBlocks / 32]
  static constexpr int OFF_LIST = OFF_BITS + 2 * kWindowBlocks / 8;               // uint16 [2][kWindowBlocks]
  static constexpr int SMEM_USED = OFF_LIST + 2 * 2 * kWindowBlocks + 1024;
  // one CTA per SM: each takes all of tensor memory (see AttnCfg)
  static constexpr int SMEM_BYTES = SMEM_USED > 116 * 1024 ? SMEM_USED : 116 * 1024;
  static constexpr int THREADS = 384, Q_ROWS = 256;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};

// One warp marks the listed key blocks of window [w0, w0 + kWindowBlocks) in `bits`; entries outside [0, n_kv) are ignored, repeated
// ones meet.  The first entries are read together with the list's length (all ld entries of a list exist).
__device__ __forceinline__ void mark_blocks(uint32_t* bits, const int* list, const int* count, long long ld, int w0, int n_kv, int lane) {
  const int first = lane < ld ? __ldg(list + lane) : -1;
  const int n = static_cast<int>(min(static_cast<long long>(max(__ldg(count), 0)), ld));
  for (int e = lane; e < n; e += 32) {
    const int j = e < 32 ? first : __ldg(list + e);
    if (j >= w0 && j < min(n_kv, w0 + kWindowBlocks)) atomicOr(bits + ((j - w0) >> 5), 1u << (j & 31));
  }
}

// One warp turns the two query tiles' marks into the visiting order: entries (block << 2 | tiles), first the blocks both
// tiles take, then those of one tile only, alternating between the tiles as long as both have some (so that the two
// softmax warpgroups keep working in turn).  Returns the number of entries.
__device__ __forceinline__ int order_blocks(const uint32_t* bits, uint16_t* list, int lane) {
  constexpr int WORDS = kWindowBlocks / 32;
  const uint32_t a = lane < WORDS ? bits[lane] : 0u, b = lane < WORDS ? bits[WORDS + lane] : 0u;
  uint32_t cls[3] = {a & b, a & ~b, b & ~a};
  int before[3], total[3];
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    const int own = __popc(cls[c]);
    int sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    before[c] = sum - own;
    total[c] = __shfl_sync(0xffffffffu, sum, 31);
  }
  const int both = total[0], paired = min(total[1], total[2]);
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    const int mask = c == 0 ? 3 : c;
    int k = before[c];
    for (uint32_t m = cls[c]; m; m &= m - 1, ++k) {
      const int block = lane * 32 + __ffs(m) - 1;
      const int at = c == 0 ? k : both + (k < paired ? 2 * k + (c - 1) : paired + k);
      list[at] = static_cast<uint16_t>(block << 2 | mask);
    }
  }
  return both + total[1] + total[2];
}

// ------------------------------------------------------------------------------------------------
// The dense kernel's scheme (attention_tcgen05_kernel: two 128-row query tiles per CTA with a softmax warpgroup each, one
// S buffer handed between them, P in tensor memory, O rescaled rarely) over a list of key blocks instead of all of
// them.  The two tiles' lists are merged: a block in both is loaded once and used twice, as in the dense kernel; one
// in a single list is loaded for that tile alone.  The key ring is three tiles deep (the dense kernel needs two):
// without sharing every use of S needs a new K tile.
// Lists are short, so what a CTA does before its first and after its last product counts: with one item per CTA that was
// 7 us of 31 (14 blocks per list).  The grid is persistent instead, and all roles run on from item to item: a warp of its own
// lays out the next lists meanwhile (two buffers), the next item's Q, K and V are requested as soon as the last
// score product of the current one has been issued, and its first scores are computed under the current item's last softmax.
// 24 heads of 128, 16896 rows, 14 of 132 blocks: 362-397 us (940-1030 TFLOP/s) under the power cap, 308 us when neighbouring tiles list the
// same blocks and 384 us when they share none; marginal rate 1400 TFLOP/s shared, 1100 not, and about 4 us per item that the
// hand-over still costs.  (Separate barriers for the two tiles' Q, so that the first scores need only half of it, cost
// 8 %: the warpgroups then fall out of turn.)
// No barrier guards O between items: a warpgroup hands over an item's first P only after it has read the previous O.
// A key block may end inside the tile.  The scores behind the end are dropped before the row maximum, and the V rows there,
// which belong to somebody else and may hold anything, are cleared in shared memory before the product
// (a zero probability times an infinity or NaN would be NaN).
// ------------------------------------------------------------------------------------------------
struct BlockItem {
  int head, qb, req, q_begin, q_len, kv_begin, kv_len, n_kv, n_windows;
  bool tile1;                                  // the second query tile has rows
};
template <int Q_ROWS>
__device__ __forceinline__ BlockItem block_item(const BlockBatch& batch, int n_heads, int item) {
  // heads of a request one after the other, so that the CTAs at work at one time share the keys of a few heads
  BlockItem it{};
  for (int i = 0; i < batch.n; ++i) {
    it.req = batch.order[i];
    const int nb = (batch.cu_q[it.req + 1] - batch.cu_q[it.req] + Q_ROWS - 1) / Q_ROWS;
    if (item < nb * n_heads) { it.head = item / nb; it.qb = item - it.head * nb; break; }
    item -= nb * n_heads;
  }
  it.q_begin = batch.cu_q[it.req]; it.q_len = batch.cu_q[it.req + 1] - it.q_begin;
  it.kv_begin = batch.cu_kv[it.req]; it.kv_len = batch.cu_kv[it.req + 1] - it.kv_begin;
  it.n_kv = (it.kv_len + 127) >> 7; it.n_windows = (it.n_kv + kWindowBlocks - 1) / kWindowBlocks;
  it.tile1 = it.qb * Q_ROWS + 128 < it.q_len;
  return it;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(BlockAttnCfg<D>::THREADS, 1)
block_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const BlockAttnParams p, const __grid_constant__ BlockBatch batch) {
  using C = BlockAttnCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  const uint32_t q_full = bar0, q_empty = bar0 + 8u, s_free = bar0 + 16u;
  auto seg_full = [&](int b) { return bar0 + 8u * (3 + b); };                     // a window's entries lie in list b
  auto seg_empty = [&](int b) { return bar0 + 8u * (5 + b); };
  auto k_full = [&](int s) { return bar0 + 8u * (7 + s); };
  auto k_empty = [&](int s) { return bar0 + 8u * (10 + s); };
  auto v_full = [&](int s) { return bar0 + 8u * (13 + s); };
  auto v_empty = [&](int s) { return bar0 + 8u * (15 + s); };
  auto s_full = [&](int i) { return bar0 + 8u * (17 + i); };
  auto p_full = [&](int i) { return bar0 + 8u * (19 + i); };
  auto o_full = [&](int i) { return bar0 + 8u * (21 + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * 23);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* n_entries = reinterpret_cast<volatile int*>(tmem_slot + 2);       // [2]
  uint32_t* bits = reinterpret_cast<uint32_t*>(aligned + C::OFF_BITS);
  uint16_t* lists = reinterpret_cast<uint16_t*>(aligned + C::OFF_LIST);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(s_free, 4);
    for (int b = 0; b < 2; ++b) { mbar_init(seg_full(b), 1); mbar_init(seg_empty(b), 11); }   // producer, two issuers, eight softmax warps
    for (int s = 0; s < C::K_STAGES; ++s) { mbar_init(k_full(s), 1); mbar_init(k_empty(s), 1); }
    for (int s = 0; s < C::V_STAGES; ++s) { mbar_init(v_full(s), 1); mbar_init(v_empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(s_full(i), 1); mbar_init(p_full(i), 4); mbar_init(o_full(i), 1); }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV); }
  if (warp == 1) { tmem_alloc(smem_u32(tmem_slot), 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t tS = tmem_base, tP = tmem_base + 128, tO = tmem_base + 256;      // columns: S 128, P 2 x 64, O 2 x 128

  // Every role walks the same items and windows; `seg` counts the windows.  The entries of a window are read between these two.
  auto seg_begin = [&](uint32_t seg) { return mbar_wait(seg_full(seg & 1), (seg >> 1) & 1u, abort_flag); };
  auto seg_entries = [&](uint32_t seg) { return static_cast<volatile const uint16_t*>(lists + (seg & 1) * kWindowBlocks); };
  uint32_t seg = 0;

  if (warp < 4) {
    DIT_SETMAXNREG_DEC(96);
    if (warp == 0) {
      if (lane == 0) {
        // ---------------------------------------------------------------- TMA producer
        int ks = 0, vs = 0; uint32_t kph = 1, vph = 1, qph = 1;
        for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
          const BlockItem it = block_item<C::Q_ROWS>(batch, p.n_heads, item);
          if (!mbar_wait(q_empty, qph, abort_flag)) goto done;
          qph ^= 1u;
          mbar_arrive_expect_tx(q_full, 2 * C::TILE_BYTES);
          for (int i = 0; i < 2; ++i)
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + C::OFF_Q + i * C::TILE_BYTES + pn * C::PANEL, &tmQ, it.head * D + pn * 64, it.q_begin + it.qb * C::Q_ROWS + i * 128, q_full);
          for (int w = 0; w < it.n_windows; ++w, ++seg) {
            if (!seg_begin(seg)) goto done;
            volatile const uint16_t* entries = seg_entries(seg);
            const int n = n_entries[seg & 1];
            for (int e = 0; e < n; ++e) {
              const int y = it.kv_begin + (w * kWindowBlocks + (entries[e] >> 2)) * 128;
              if (!mbar_wait(k_empty(ks), kph, abort_flag)) goto done;
              mbar_arrive_expect_tx(k_full(ks), C::TILE_BYTES);
              for (int pn = 0; pn < C::NP; ++pn)
                tma_load_2d(base + C::OFF_K + ks * C::TILE_BYTES + pn * C::PANEL, &tmK, it.head * D + pn * 64, y, k_full(ks));
              if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
              if (!mbar_wait(v_empty(vs), vph, abort_flag)) goto done;
              mbar_arrive_expect_tx(v_full(vs), C::TILE_BYTES);
              for (int pn = 0; pn < C::NP; ++pn)
                tma_load_2d(base + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL, &tmV, it.head * D + pn * 64, y, v_full(vs));
              if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
            }
            mbar_arrive(seg_empty(seg & 1));
          }
        }
      }
    } else if (warp == 1) {
      if (lane == 0) {
        // ---------------------------------------------------------------- MMA issuer 1: scores
        constexpr uint32_t idesc_s = idesc_f16(128, 128, false, BF16);
        const uint64_t qdesc0 = smem_desc_sw128(base + C::OFF_Q, 16, 1024), kdesc0 = smem_desc_sw128(base + C::OFF_K, 16, 1024);
        constexpr uint32_t kTileStep = C::TILE_BYTES >> 4;
        int ks = 0; uint32_t kph = 0, qph = 0, u = 0;                             // u: uses of S so far
        for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
          const BlockItem it = block_item<C::Q_ROWS>(batch, p.n_heads, item);
          if (!mbar_wait(q_full, qph, abort_flag)) goto done;
          qph ^= 1u;
          for (int w = 0; w < it.n_windows; ++w, ++seg) {
            if (!seg_begin(seg)) goto done;
            volatile const uint16_t* entries = seg_entries(seg);
            const int n = n_entries[seg & 1];
            for (int e = 0; e < n; ++e) {
              const int tiles = entries[e] & 3;
              if (!mbar_wait(k_full(ks), kph, abort_flag)) goto done;
              for (int i = 0; i < 2; ++i) {
                if (!((tiles >> i) & 1)) continue;
                if (u > 0 && !mbar_wait(s_free, (u - 1) & 1u, abort_flag)) goto done;
                ++u;
                tc_fence_after();
                const uint64_t qd = qdesc0 + i * kTileStep, kd = kdesc0 + ks * kTileStep;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  const uint32_t off = ((kk >> 2) * C::PANEL + (kk & 3) * 32) >> 4;
                  umma_f16(tS, qd + off, kd + off, idesc_s, kk != 0);
                }
                if (i == 1 || tiles == 1) umma_commit(k_empty(ks));               // the entry's last use of its K tile
                umma_commit(s_full(i));
              }
              if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
            }
            mbar_arrive(seg_empty(seg & 1));
          }
          umma_commit(q_empty);                                                   // Q may be replaced once these products have read it
        }
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ MMA issuer 2: P V (the whole warp walks the lists: it also
      // clears the V rows behind a request's last key)
      constexpr uint32_t idesc_pv = idesc_f16(128, D, true, BF16);
      const uint64_t vdesc0 = smem_desc_sw128(base + C::OFF_V, C::PANEL, 1024);
      constexpr uint32_t kTileStep = C::TILE_BYTES >> 4;
      int vs = 0; uint32_t vph = 0, done_uses[2] = {0, 0};
      for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
        const BlockItem it = block_item<C::Q_ROWS>(batch, p.n_heads, item);
        bool more[2] = {false, false};                                            // O holds products of this item
        for (int w = 0; w < it.n_windows; ++w, ++seg) {
          if (!__all_sync(0xffffffffu, seg_begin(seg))) goto done;
          volatile const uint16_t* entries = seg_entries(seg);
          const int n = n_entries[seg & 1];
          for (int e = 0; e < n; ++e) {
            const int tiles = entries[e] & 3, j = w * kWindowBlocks + (entries[e] >> 2);
            if (!__all_sync(0xffffffffu, mbar_wait(v_full(vs), vph, abort_flag))) goto done;
            const int valid = it.kv_len - j * 128;
            if (valid < 128) {
              for (int r = valid * 8 + lane; r < 128 * 8; r += 32)                // 16-byte units of rows valid .. 127
                for (int pn = 0; pn < C::NP; ++pn)
                  *reinterpret_cast<uint4*>(aligned + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL + r * 16) = make_uint4(0, 0, 0, 0);
              fence_proxy_async_smem();
              __syncwarp();
            }
            const uint64_t vd = vdesc0 + vs * kTileStep;
            for (int i = 0; i < 2; ++i) {
              if (!((tiles >> i) & 1)) continue;
              if (!__all_sync(0xffffffffu, mbar_wait(p_full(i), done_uses[i] & 1u, abort_flag))) goto done;
              tc_fence_after();
              if (lane == 0) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                  umma_f16_ts(tO + i * 128, tP + i * 64 + kk * 8, vd + kk * (2048 >> 4), idesc_pv, more[i] || kk != 0);
                if (i == 1 || tiles == 1) umma_commit(v_empty(vs));
                umma_commit(o_full(i));
              }
              __syncwarp();
              ++done_uses[i];
              more[i] = true;
            }
            if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(seg_empty(seg & 1));
        }
      }
    } else {
      // ------------------------------------------------------------------ lists of the coming windows
      for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
        const BlockItem it = block_item<C::Q_ROWS>(batch, p.n_heads, item);
        const long long row = static_cast<long long>(it.head) * batch.first_qblock[batch.n] + batch.first_qblock[it.req] + 2 * it.qb;
        for (int w = 0; w < it.n_windows; ++w, ++seg) {
          if (lane < 2 * kWindowBlocks / 32) bits[lane] = 0;
          __syncwarp();
          mark_blocks(bits, p.index + row * p.ld_index, p.count + row, p.ld_index, w * kWindowBlocks, it.n_kv, lane);
          if (it.tile1)
            mark_blocks(bits + kWindowBlocks / 32, p.index + (row + 1) * p.ld_index, p.count + row + 1, p.ld_index, w * kWindowBlocks, it.n_kv, lane);
          __syncwarp();
          if (!__all_sync(0xffffffffu, mbar_wait(seg_empty(seg & 1), ((seg >> 1) & 1u) ^ 1u, abort_flag))) goto done;
          const int n = order_blocks(bits, lists + (seg & 1) * kWindowBlocks, lane);
          if (lane == 0) n_entries[seg & 1] = n;
          __syncwarp();
          if (lane == 0) mbar_arrive(seg_full(seg & 1));
        }
      }
    }
  } else {
    // -------------------------------------------------------------------- softmax + accumulate (2 warpgroups)
    DIT_SETMAXNREG_INC(200);
    const int tile = (warp >> 2) - 1, quarter = warp & 3;
    const uint32_t lane_sel = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tSi = tS + lane_sel, tPi = tP + tile * 64 + lane_sel, tOi = tO + tile * 128 + lane_sel;
    const float c = p.scale_log2;
    const float2 c2 = make_float2(c, c);
    constexpr float kRescaleLog2 = 8.0f;       // O is rescaled when a row's maximum has grown by more than 2^8: P stays <= 2^8
    constexpr float kFarLog2 = 1024.0f;        // scaled references beyond it are taken off before the scaling
    uint32_t use = 0;                          // key blocks of this warpgroup so far

    for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
      const BlockItem it = block_item<C::Q_ROWS>(batch, p.n_heads, item);
      float m_ref = -INFINITY, l = 0.f;
      const uint32_t first_use = use;
      for (int w = 0; w < it.n_windows; ++w, ++seg) {
        if (!__all_sync(0xffffffffu, seg_begin(seg))) goto done;
        volatile const uint16_t* entries = seg_entries(seg);
        const int n = n_entries[seg & 1];
        for (int e = 0; e < n; ++e) {
          const int entry = entries[e];
          if (!((entry >> tile) & 1)) continue;
          if (!__all_sync(0xffffffffu, mbar_wait(s_full(tile), use & 1u, abort_flag))) goto done;
          tc_fence_after();
          const int valid = it.kv_len - (w * kWindowBlocks + (entry >> 2)) * 128;
          uint32_t sv[128];
          __syncwarp();
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) tmem_ld32p(tSi + ch * 32, sv + ch * 32);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_free);
          if (valid < 128) {
#pragma unroll
            for (int i = 0; i < 128; ++i)
              if (i >= valid) sv[i] = 0xff800000u;
          }
          float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
          for (int i = 0; i < 128; i += 8) {
            mx0 = fmax3(mx0, __uint_as_float(sv[i]), __uint_as_float(sv[i + 1]));
            mx1 = fmax3(mx1, __uint_as_float(sv[i + 2]), __uint_as_float(sv[i + 3]));
            mx2 = fmax3(mx2, __uint_as_float(sv[i + 4]), __uint_as_float(sv[i + 5]));
            mx3 = fmax3(mx3, __uint_as_float(sv[i + 6]), __uint_as_float(sv[i + 7]));
          }
          const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
          // Two rare things, behind one vote.  A row's maximum has grown far beyond its reference: this warp's rows of O are rescaled.
          // Or its reference is large: the exponent s * c - round(m_ref * c) is off by that rounding, which is at most 2^-14 below the
          // limit and common to all that share the reference, but from 2^28 on would leave the 16-bit probabilities.  Beyond the
          // limit the reference is therefore taken off the scores before the scaling: (s - m_ref) * c is 0 for the largest
          // whatever c is.  Decided row by row, so that a row does not depend on its neighbours.
          if (use == first_use) m_ref = mx;
          const bool grow = (mx - m_ref) * c > kRescaleLog2;
          bool far = fabsf(m_ref * c) > kFarLog2;
          if (__any_sync(0xffffffffu, grow || far)) {
            if (__any_sync(0xffffffffu, grow)) {
              if (!__all_sync(0xffffffffu, mbar_wait(o_full(tile), (use - 1) & 1u, abort_flag))) goto done;
              tc_fence_after();
              const float alpha = grow ? exp2_approx((m_ref - mx) * c) : 1.0f;
              if (grow) { m_ref = mx; l *= alpha; }
#pragma unroll 1
              for (int ch = 0; ch < D / 32; ++ch) {
                uint32_t r[32];
                __syncwarp();
                tmem_ld32(tOi + ch * 32, r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
                tmem_st32(tOi + ch * 32, r);
              }
              tmem_st_wait();
            }
            far = fabsf(m_ref * c) > kFarLog2;
            // (a reference of -inf, every score so far -inf from infinite inputs, would make the exponents NaN: nothing is taken off)
            const float off = far && m_ref != -INFINITY ? m_ref : 0.f;
#pragma unroll
            for (int i = 0; i < 128; ++i) sv[i] = __float_as_uint(__uint_as_float(sv[i]) - off);
          }
          const float neg_mc = far ? 0.f : -m_ref * c;
          const float2 nm2 = make_float2(neg_mc, neg_mc);
          float2 rs0 = make_float2(0.f, 0.f), rs1 = make_float2(0.f, 0.f);
#pragma unroll
          for (int i = 0; i < 128; i += 2) {
            const float2 x = ffma2(make_float2(__uint_as_float(sv[i]), __uint_as_float(sv[i + 1])), c2, nm2);
            const float2 ex = make_float2(exp2_approx(x.x), exp2_approx(x.y));
            if (i & 2) rs1 = fadd2(rs1, ex); else rs0 = fadd2(rs0, ex);
            sv[i >> 1] = pack16x2<BF16>(ex.x, ex.y);
          }
          if (use != first_use) {              // P is still read by this tile's previous product until that has finished
            if (!__all_sync(0xffffffffu, mbar_wait(o_full(tile), (use - 1) & 1u, abort_flag))) goto done;
            tc_fence_after();
          }
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) tmem_st16(tPi + ch * 16, *reinterpret_cast<const uint32_t(*)[16]>(sv + ch * 16));
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(tile));
          l += (rs0.x + rs0.y) + (rs1.x + rs1.y);
          ++use;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(seg_empty(seg & 1));
      }
      if (tile == 1 && !it.tile1) continue;
      const int row = it.qb * C::Q_ROWS + tile * 128 + quarter * 32 + lane;       // in the request
      uint16_t* out = static_cast<uint16_t*>(p.out) + (static_cast<long long>(it.q_begin) + row) * p.ld_out + it.head * D;
      const bool any = use != first_use;       // without a key: zeros
      if (any) {
        if (!__all_sync(0xffffffffu, mbar_wait(o_full(tile), (use - 1) & 1u, abort_flag))) goto done;
        tc_fence_after();
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      // The results of 32 channels at a time; `kept` writes infinities as such and is a second pass over the rare rows that have one, so that
      // the ordinary one pays for the largest magnitude only.
      float largest[2] = {0.f, 0.f};
      auto write = [&](auto kept) {
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t r[32];
          __syncwarp();
          if (any) {
            tmem_ld32(tOi + ch * 32, r);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = 0u;
          }
          if (row < it.q_len) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {      // a lane writes its own row, a whole 32-byte sector per store
              uint32_t wd[8];
#pragma unroll
              for (int h = 0; h < 8; ++h) {
                const float lo = __uint_as_float(r[16 * v + 2 * h]), hi = __uint_as_float(r[16 * v + 2 * h + 1]);
                wd[h] = pack16x2<BF16>(lo * inv, hi * inv);
                if constexpr (decltype(kept)::value) wd[h] = put_infinities<BF16>(wd[h], lo * inv, hi * inv);
              }
              uint16_t* at = out + ch * 32 + v * 16;
              if (p.wide_out) {
                st_global_v8(at, wd);
              } else {
                reinterpret_cast<uint4*>(at)[0] = make_uint4(wd[0], wd[1], wd[2], wd[3]);
                reinterpret_cast<uint4*>(at)[1] = make_uint4(wd[4], wd[5], wd[6], wd[7]);
              }
            }
            if constexpr (!decltype(kept)::value) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                largest[0] = fmax3(largest[0], fabsf(__uint_as_float(r[i])), fabsf(__uint_as_float(r[i + 1])));
                largest[1] = fmax3(largest[1], fabsf(__uint_as_float(r[i + 2])), fabsf(__uint_as_float(r[i + 3])));
              }
            }
          }
        }
      };
      write(std::false_type{});
      if (!p.clamp && __any_sync(0xffffffffu, fmaxf(largest[0], largest[1]) == INFINITY)) write(std::true_type{});
    }
  }

done:
  tc_fence_before();
  __syncthreads();
  settle_if_aborted(abort_flag);
  __syncwarp();
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, 512); }
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusAttnTimeout);
}

// ------------------------------------------------------------------------------------------------
// Few query rows per request (a new token or two against a stored context).  Reading the selected K and V blocks once is the
// bound, and 16 rows or fewer do not fill a tensor-memory tile: the products are warp-level 16 x 8 x 16 ones, which
// cost the same for one row as for sixteen (on the FMA pipe one row took 550 instructions per 64 keys and warp and
// issue was the bound; this form takes about 150).  A cluster of CTAs shares a (request, head): rank r takes every splits-th selected
// block.  K and V arrive by TMA as tiles of 64 keys in swizzled panels through one ring (K, V, K, V, ...), five of
// six tiles in flight per CTA and two CTAs per SM.  Warp w works on keys 16 w .. 16 w + 15 of every tile on its
// own, with its own running maximum and sum per row: the accumulator layout of the scores is the operand layout of
// the second product, so probabilities stay in registers.  The warps' results meet in shared memory (the ring's,
// once everything has been read), the CTAs' through distributed shared memory, in rank and warp order.
// Four requests of one row, 24 heads of 128, 60 blocks in all (94 MB): 19 us when they are in L2, 24.8 us (3.8 TB/s) from DRAM; longer
// lists, beyond L2, 5.7-6.2 TB/s.
// ------------------------------------------------------------------------------------------------
constexpr int kRowsTile = 64;                  // keys per tile
constexpr int kRowsMax = 16;                   // query rows
template <int D>
struct BlockRowsCfg {
  static constexpr int NP = D / 64, PANEL = kRowsTile * 128, TILE_BYTES = NP * PANEL;
  static constexpr int STAGES = 96 * 1024 / TILE_BYTES;                          // 6 (d = 128), 12 (d = 64)
  static constexpr int OFF_BAR = STAGES * TILE_BYTES;
  static constexpr int OFF_BITS = OFF_BAR + 256;                                 // uint32 [kMaxKeyBlocks / 32]
  static constexpr int SMEM_BYTES = OFF_BITS + kMaxKeyBlocks / 8 + 1024;
  static constexpr int THREADS = 160;                                            // four key warps and a producer
  static constexpr int PART = D + 2;                                             // floats of a row's partial result: channels, maximum, sum
  static_assert(4 * kRowsMax * PART * 4 <= OFF_BAR, "the partial results take the ring's place");
  static_assert(2 * SMEM_BYTES <= 227 * 1024, "two CTAs per SM");
};

template <int D, bool BF16>
__global__ void __launch_bounds__(BlockRowsCfg<D>::THREADS, 2)
block_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const BlockAttnParams p, const uint16_t* q,
                  const long long ld_q, const __grid_constant__ BlockBatch batch, const int splits) {
  using C = BlockRowsCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(aligned + C::OFF_BAR + 16 * C::STAGES);
  uint32_t* bits = reinterpret_cast<uint32_t*>(aligned + C::OFF_BITS);
  float* part = reinterpret_cast<float*>(aligned);                      // [4 warps][kRowsMax][PART], after the main loop

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int item = blockIdx.x / splits, head = item % p.n_heads, req = item / p.n_heads;
  const int q_begin = batch.cu_q[req], rows = batch.cu_q[req + 1] - q_begin;      // 0 .. kRowsMax
  const int kv_begin = batch.cu_kv[req], kv_len = batch.cu_kv[req + 1] - kv_begin;
  const int n_kv = (kv_len + 127) >> 7, words = (n_kv + 31) >> 5;

  for (int i = threadIdx.x; i < words; i += C::THREADS) bits[i] = 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 4); }
    *abort_flag = 0;
    fence_mbar_init();
  }
  // Q as the first operand: k step t, rows lane / 4 and + 8, channels 16 t + 2 (lane % 4) and + 8; absent rows are zero
  uint32_t qa[D / 16][4];
  if (warp < 4) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = (lane >> 2) + (i & 1) * 8, c = t * 16 + (lane & 3) * 2 + (i >> 1) * 8;
        qa[t][i] = r < rows ? *reinterpret_cast<const uint32_t*>(q + (static_cast<long long>(q_begin) + r) * ld_q + head * D + c) : 0u;
      }
  }
  __syncthreads();
  if (rows > 0) {
    const long long at = static_cast<long long>(head) * batch.first_qblock[batch.n] + batch.first_qblock[req];
    const int n = static_cast<int>(min(static_cast<long long>(max(__ldg(p.count + at), 0)), p.ld_index));
    const int* list = p.index + at * p.ld_index;
    for (int e = threadIdx.x; e < n; e += C::THREADS) {
      const int j = __ldg(list + e);
      if (j >= 0 && j < n_kv) atomicOr(bits + (j >> 5), 1u << (j & 31));
    }
  }
  __syncthreads();

  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};               // rows lane / 4 and + 8; l: this lane's columns only
  float acc[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
  bool ok = true;
  if (warp == 4) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int stage = 0, turn = 0; uint32_t phase = 1;
      for (int w = 0; w < words && ok; ++w)
        for (uint32_t b = bits[w]; b && ok; b &= b - 1) {
          if (turn++ % splits != rank) continue;
          const int y = (w * 32 + __ffs(b) - 1) * 128;
          for (int t = 0; t < 4 && ok; ++t) {                           // K, V of the first 64 keys, K, V of the rest if there is one
            const int y0 = y + (t >> 1) * kRowsTile;
            if (y0 >= kv_len) break;
            if (!(ok = mbar_wait(empty(stage), phase, abort_flag))) break;
            mbar_arrive_expect_tx(full(stage), C::TILE_BYTES);
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + stage * C::TILE_BYTES + pn * C::PANEL, (t & 1) ? &tmV : &tmK, head * D + pn * 64, kv_begin + y0, full(stage));
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
          }
        }
    }
  } else {
    // ------------------------------------------------------------------ keys 16 * warp .. + 15 of every tile
    int stage = 0, turn = 0; uint32_t phase = 0;
    // row addresses of the ldmatrix loads: of K, matrices (keys 0-7 | 8-15) x (channels 0-7, 8-15 of a k step); of V, transposed,
    // (channels 0-7 | 8-15 of a pair of output tiles) x (keys 0-7, 8-15)
    const int k_row = 16 * warp + (lane >> 4) * 8 + (lane & 7), k_unit = (lane >> 3) & 1;
    const int v_row = 16 * warp + ((lane >> 3) & 1) * 8 + (lane & 7), v_unit = lane >> 4;
    for (int w = 0; w < words && ok; ++w)
      for (uint32_t b = bits[w]; b && ok; b &= b - 1) {
        if (turn++ % splits != rank) continue;
        for (int y0 = (w * 32 + __ffs(b) - 1) * 128, half = 0; half < 2 && y0 < kv_len; ++half, y0 += kRowsTile) {
          const int keys = kv_len - y0 - 16 * warp;                     // of this warp: 16 or more, or the rest (may be <= 0)
          if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(stage), phase, abort_flag)))) break;
          float s[2][4] = {};                                           // keys 0-7 and 8-15
          {
            const uint32_t kt = base + stage * C::TILE_BYTES + k_row * 128;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
              const int u = 2 * t + k_unit;
              uint32_t kb[4];
              ldmatrix_x4(kb, kt + (u >> 3) * C::PANEL + (((u & 7) ^ (k_row & 7)) << 4));
              mma_16816<BF16>(s[0], qa[t], kb[0], kb[1]);
              mma_16816<BF16>(s[1], qa[t], kb[2], kb[3]);
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(empty(stage));
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
          if (keys < 16) {                                              // drop the scores behind the request's last key
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (8 * i + 2 * (lane & 3) + (k & 1) >= keys) s[i][k] = -INFINITY;
          }
          uint32_t pa[4];
#pragma unroll
          for (int r = 0; r < 2; ++r) {                                 // rows lane / 4 + 8 r
            float mx = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            // the reference is taken off before the scaling: the largest score's exponent is 0 however large the factor is
            const float top = fmaxf(m[r], mx), at = top == -INFINITY ? 0.f : top;
            const float alpha = exp2_approx((m[r] - at) * p.scale_log2);                 // 0 while m is -inf
            m[r] = top;
            float e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = exp2_approx((s[k >> 1][2 * r + (k & 1)] - at) * p.scale_log2);
            l[r] = l[r] * alpha + (e[0] + e[1]) + (e[2] + e[3]);
            pa[r] = pack16x2<BF16>(e[0], e[1]);
            pa[2 + r] = pack16x2<BF16>(e[2], e[3]);
            if (__any_sync(0xffffffffu, alpha != 1.0f)) {
#pragma unroll
              for (int i = 0; i < D / 8; ++i) { acc[i][2 * r] *= alpha; acc[i][2 * r + 1] *= alpha; }
            }
          }
          if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(stage), phase, abort_flag)))) break;
          if (keys < 16) {                                              // clear the V rows behind it: they may hold anything
            for (int i = lane; i < 16 * 8; i += 32)
              if ((i >> 3) >= keys)
                for (int pn = 0; pn < C::NP; ++pn)
                  *reinterpret_cast<uint4*>(aligned + stage * C::TILE_BYTES + pn * C::PANEL + (16 * warp * 8 + i) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();                                   // the stage is refilled by TMA
            __syncwarp();
          }
          {
            const uint32_t vt = base + stage * C::TILE_BYTES + v_row * 128;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
              const int u = 2 * t + v_unit;
              uint32_t vb[4];
              ldmatrix_x4_trans(vb, vt + (u >> 3) * C::PANEL + (((u & 7) ^ (v_row & 7)) << 4));
              mma_16816<BF16>(acc[2 * t], pa, vb[0], vb[1]);
              mma_16816<BF16>(acc[2 * t + 1], pa, vb[2], vb[3]);
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(empty(stage));
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
      }
  }
  __syncthreads();                             // every tile has been read: the partial results take the ring's place
  settle_if_aborted(abort_flag);
  if (warp < 4) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      const int row = (lane >> 2) + 8 * r;
      if (row < rows) {
        float* dst = part + (warp * kRowsMax + row) * C::PART;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2*>(dst + i * 8 + (lane & 3) * 2) = make_float2(acc[i][2 * r], acc[i][2 * r + 1]);
        if ((lane & 3) == 0) { dst[D] = m[r]; dst[D + 1] = l[r]; }
      }
    }
  }
  __syncwarp();
  if (splits > 1) cluster_sync_all(); else __syncthreads();
  if (threadIdx.x < D) {
    // rank's share of the rows, channel per thread: the parts rescaled to their common maximum
    for (int row = rank; row < rows; row += splits) {
      auto read = [&](int s, int w, int i) {
        const float* at = part + (w * kRowsMax + row) * C::PART + i;
        return splits > 1 ? ld_cluster_f32(map_to_cta(smem_u32(at), s)) : *at;
      };
      float ref = -INFINITY, sum = 0.f, o = 0.f;
      for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float pm = read(s, w, D), pl = read(s, w, D + 1), po = read(s, w, threadIdx.x);
          const float top = fmaxf(ref, pm), at = top == -INFINITY ? 0.f : top;
          const float keep = exp2_approx((ref - at) * p.scale_log2), f = exp2_approx((pm - at) * p.scale_log2);
          sum = sum * keep + pl * f;
          o = o * keep + po * f;
          ref = top;
        }
      const float x = sum == 0.f ? 0.f : o / sum;
      static_cast<uint16_t*>(p.out)[(static_cast<long long>(q_begin) + row) * p.ld_out + head * D + threadIdx.x] =
          fabsf(x) == INFINITY && !p.clamp ? static_cast<uint16_t>(infinity_bits<BF16>(x)) : pack16<BF16>(x);
    }
  }
  __syncwarp();
  if (splits > 1) cluster_sync_all(); else __syncthreads();           // peers may be read until here
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusAttnTimeout);
}

// ------------------------------------------------------------------------------------------------
// Selector.  Means of the 128-row blocks of q and k in 64 bits (the sum of 128 fp16 values is exact there, and of bf16
// values too unless their magnitudes are more than 2^38 apart), then their products in 64 bits: the order of two scores is decided by
// their values and not by an order of summation, so lists do not change with the batch or the launch.
// ------------------------------------------------------------------------------------------------
struct BlockSelectParams {
  const uint16_t *q, *k;
  long long ld_q, ld_k;
  int width, n_heads, head_dim;
  double* q_mean;            // [query blocks, width]
  double* k_mean;            // [key blocks, width]
  int* index;
  int* count;
  long long ld_index;
  int widest;                // largest keep: entries of a list that are written
  int rows;                  // query blocks per CTA of the selecting kernel
  int keep[DIT_MAX_REQUESTS], tail[DIT_MAX_REQUESTS];
};

template <bool BF16>
__device__ __forceinline__ double widen_double(uint16_t h) {
  double d;
  if (BF16) return static_cast<double>(__uint_as_float(static_cast<uint32_t>(h) << 16));
  asm("cvt.f64.f16 %0, %1;" : "=d"(d) : "h"(h));
  return d;
}

// 42 us for 208 MB (4.9 TB/s): the conversions to 64 bits, 16 per clock and SM, take 24 us of issue beside the loads.
// One CTA per (block, 256 columns): eight warps take every eighth row, a lane 16 bytes of it.  Bound by reading q and k once.
template <bool BF16>
__global__ void __launch_bounds__(256, 3)
block_means_kernel(const BlockSelectParams p, const __grid_constant__ BlockBatch batch) {
  __shared__ double sums[8][256];
  const int q_blocks = batch.first_qblock[batch.n];
  const int chunks = (p.width + 255) / 256;
  int block = blockIdx.x / chunks;
  const int col0 = blockIdx.x % chunks * 256;
  const bool is_k = block >= q_blocks;
  if (is_k) block -= q_blocks;
  const int* first = is_k ? batch.first_kblock : batch.first_qblock;
  const int* cu = is_k ? batch.cu_kv : batch.cu_q;
  int lo = 0, hi = batch.n - 1;                // the block's request: the last one whose first block is not behind it
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= block) lo = mid; else hi = mid - 1;
  }
  const int row0 = cu[lo] + (block - first[lo]) * 128, n = min(128, cu[lo + 1] - row0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = col0 + lane * 8;
  const long long ld = is_k ? p.ld_k : p.ld_q;
  const uint16_t* src = (is_k ? p.k : p.q) + row0 * ld + col;
  double acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.0;
  if (col < p.width) {
    {
      uint4 v[16];                             // all sixteen rows of the lane are requested before the first is used
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = warp + 8 * i;
        v[i] = r < n ? load_once(src + r * ld) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          acc[2 * c] += widen_double<BF16>(static_cast<uint16_t>(u[c])); acc[2 * c + 1] += widen_double<BF16>(static_cast<uint16_t>(u[c] >> 16));
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[warp][lane * 8 + i] = acc[i];
  __syncthreads();
  const int mine = col0 + threadIdx.x;
  if (mine < p.width) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += sums[w][threadIdx.x];
    s /= static_cast<double>(n);
    (is_k ? p.k_mean : p.q_mean)[static_cast<long long>(block) * p.width + mine] = s;
  }
}

// Order-preserving map of a score to an unsigned number: NaN lowest, the two zeros alike.
__device__ __forceinline__ unsigned long long score_key(double s) {
  if (s != s) return 0ull;
  const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(s + 0.0));
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// One CTA per (head, up to eight query blocks of a request).  Scores: 8 x 8 x 4 products in 64 bits, a warp per eight key
// blocks (a thread per key block on the FMA pipe took three times as long, most of it in operand reads).  Lists: a
// warp per row finds the keep-th largest score by deciding its bits from the top (counting the scores that reach the
// candidate), starting at the first bit in which the row's scores differ and ending as soon as exactly `keep` reach it.
constexpr int kSelectRows = 8, kSelectThreads = 256, kSelectPitch = 130;   // pitch: rows four banks apart

__global__ void __launch_bounds__(kSelectThreads, 4)
block_select_kernel(const BlockSelectParams p, const __grid_constant__ BlockBatch batch) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  double* qm = reinterpret_cast<double*>(smem_raw);                              // [kSelectRows][kSelectPitch]
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(qm + kSelectRows * kSelectPitch);   // [rows][n_kv]
  const int q_blocks = batch.first_qblock[batch.n];
  int head = 0, group = blockIdx.x, req = 0;
  for (req = 0; req < batch.n; ++req) {
    const int groups = (batch.first_qblock[req + 1] - batch.first_qblock[req] + p.rows - 1) / p.rows;
    if (group < groups * p.n_heads) { head = group / groups; group -= head * groups; break; }
    group -= groups * p.n_heads;
  }
  const int qb0 = batch.first_qblock[req] + group * p.rows, n_rows = min(p.rows, batch.first_qblock[req + 1] - qb0);
  const int kb0 = batch.first_kblock[req], n_kv = batch.first_kblock[req + 1] - kb0;
  const int kv_len = batch.cu_kv[req + 1] - batch.cu_kv[req];
  const int d = p.head_dim;
  for (int i = threadIdx.x; i < d * kSelectRows; i += kSelectThreads) {
    const int r = i / d, c = i % d;
    qm[r * kSelectPitch + c] = r < n_rows ? p.q_mean[static_cast<long long>(qb0 + r) * p.width + head * d + c] : 0.0;
  }
  __syncthreads();
  {
    const int lane = threadIdx.x & 31, row = lane >> 2, col = lane & 3;
    const double* qa = qm + row * kSelectPitch + col;
    for (int j0 = (threadIdx.x >> 5) * 8; j0 < n_kv; j0 += kSelectThreads / 32 * 8) {
      const bool there = j0 + row < n_kv;                                        // this lane's key block as an operand
      const double* km = p.k_mean + static_cast<long long>(kb0 + (there ? j0 + row : 0)) * p.width + head * d + col;
      double s[2][2] = {};
      for (int c0 = 0; c0 < d; c0 += 64) {
        double k[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) k[i] = __ldg(km + c0 + 4 * i);
#pragma unroll
        for (int i = 0; i < 16; ++i) mma_884_f64(s[i & 1], qa[c0 + 4 * i], k[i]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {                                              // score of (row, key block j)
        const int j = j0 + 2 * col + i;
        if (j < n_kv && row < n_rows) {
          const bool forced = p.tail[req] > 0 && static_cast<long long>(j + 1) * 128 > static_cast<long long>(kv_len) - p.tail[req];
          keys[static_cast<long long>(row) * n_kv + j] = forced ? ~0ull : score_key(s[0][i] + s[1][i]);
        }
      }
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp >= n_rows) return;
  const unsigned long long* mine = keys + static_cast<long long>(warp) * n_kv;
  const int want = min(p.keep[req], n_kv);
  unsigned long long high = 0, low = ~0ull;
  for (int j = lane; j < n_kv; j += 32) { high = max(high, mine[j]); low = min(low, mine[j]); }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    high = max(high, __shfl_xor_sync(0xffffffffu, high, o));
    low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
  }
  const int first_bit = n_kv > 0 ? 63 - __clzll(static_cast<long long>(high ^ low)) : -1;   // -1: all alike
  unsigned long long least = first_bit < 63 ? (high >> (first_bit + 1)) << (first_bit + 1) : 0ull;   // keys >= least: at least `want`
  int reach = n_kv, bit = first_bit;           // how many they are; the next bit to decide
  constexpr int kHeld = 8;
  if (n_kv <= 32 * kHeld) {
    // the upper 32 bits nearly always decide: they are held in registers for that part
    uint32_t top[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top[i] = i * 32 + lane < n_kv ? static_cast<uint32_t>(mine[i * 32 + lane] >> 32) : 0u;
    for (; bit >= 32 && reach != want; --bit) {
      const uint32_t candidate = static_cast<uint32_t>(least >> 32) | (1u << (bit - 32));
      int n = 0;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i * 32 < n_kv) n += __popc(__ballot_sync(0xffffffffu, top[i] >= candidate));
      if (n >= want) { least = static_cast<unsigned long long>(candidate) << 32; reach = n; }
    }
  }
  for (; bit >= 0 && reach != want; --bit) {
    const unsigned long long candidate = least | (1ull << bit);
    int n = 0;
    for (int j = lane; j < n_kv; j += 32) n += mine[j] >= candidate ? 1 : 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (n >= want) { least = candidate; reach = n; }
  }
  // more than `want` reach it only if several equal it: the lowest of those are taken
  int ties = INT32_MAX;
  if (reach != want) {
    int above = 0;
    for (int j = lane; j < n_kv; j += 32) above += mine[j] > least ? 1 : 0;
    ties = want - __reduce_add_sync(0xffffffffu, above);
  }
  const long long at = static_cast<long long>(head) * q_blocks + qb0 + warp;
  int* list = p.index + at * p.ld_index;
  int written = 0;
  for (int j0 = 0; j0 < n_kv; j0 += 32) {
    const int j = j0 + lane;
    const unsigned long long key = j < n_kv ? mine[j] : 0ull;
    const unsigned equal = __ballot_sync(0xffffffffu, j < n_kv && key == least);
    const bool take = j < n_kv && (key > least || (key == least && __popc(equal & ((1u << lane) - 1u)) < ties));
    const unsigned taken = __ballot_sync(0xffffffffu, take);
    if (take) list[written + __popc(taken & ((1u << lane) - 1u))] = j;
    written += __popc(taken);
    if (ties != INT32_MAX) ties = max(0, ties - __popc(equal));
  }
  for (long long e = want + lane; e < p.widest; e += 32) list[e] = -1;           // (widest may be the largest int: `all of them`)
  if (lane == 0) p.count[at] = want;
}

}  // namespace dit
