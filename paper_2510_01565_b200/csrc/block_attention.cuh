// Attention over selected key blocks (128 rows each), and the selection by the product of block means.
//
// block_attention_kernel   256 query rows of a head per CTA on the tensor cores, for query blocks of many rows
// block_rows_kernel        up to 4 query rows of a head per cluster on the FMA pipe, for a few rows that read a long context
// block_means_kernel, block_select_kernel   the selector
#pragma once
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
  int* status;
};

constexpr int kWindowBlocks = 512;      // key blocks whose lists are laid out in shared memory at a time
constexpr int kMaxKeyBlocks = 16384;    // of one request

template <int D>
struct BlockAttnCfg {
  static constexpr int NP = D / 64, PANEL = 128 * 128, TILE_BYTES = NP * PANEL;
  static constexpr int K_STAGES = 3, V_STAGES = 2;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + K_STAGES * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_V + V_STAGES * TILE_BYTES;
  static constexpr int OFF_BITS = OFF_BAR + 256;                                  // uint32 [2][kWindowBlocks / 32]
  static constexpr int OFF_LIST = OFF_BITS + 2 * kWindowBlocks / 8;               // uint16 [kWindowBlocks]
  static constexpr int SMEM_USED = OFF_LIST + 2 * kWindowBlocks + 1024;
  // one CTA per SM: each takes all of tensor memory (see AttnCfg)
  static constexpr int SMEM_BYTES = SMEM_USED > 116 * 1024 ? SMEM_USED : 116 * 1024;
  static constexpr int THREADS = 384, Q_ROWS = 256;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};

// Marks the listed key blocks of window [w0, w0 + kWindowBlocks) in `bits`; entries outside [0, n_kv) are ignored, repeated ones meet.
__device__ __forceinline__ void mark_blocks(uint32_t* bits, const int* list, int n, int w0, int n_kv, int tid, int threads) {
  for (int e = tid; e < n; e += threads) {
    const int j = __ldg(list + e);
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
// A key block may end inside the tile.  The scores behind the end are dropped before the row maximum, and the V rows there,
// which belong to somebody else and may hold anything, are cleared in shared memory before the product
// (a zero probability times an infinity or NaN would be NaN).
// ------------------------------------------------------------------------------------------------
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
  const uint32_t q_full = bar0, s_free = bar0 + 8u, win_full = bar0 + 16u, win_empty = bar0 + 24u;
  auto k_full = [&](int s) { return bar0 + 8u * (4 + s); };
  auto k_empty = [&](int s) { return bar0 + 8u * (7 + s); };
  auto v_full = [&](int s) { return bar0 + 8u * (10 + s); };
  auto v_empty = [&](int s) { return bar0 + 8u * (12 + s); };
  auto s_full = [&](int i) { return bar0 + 8u * (14 + i); };
  auto p_full = [&](int i) { return bar0 + 8u * (16 + i); };
  auto o_full = [&](int i) { return bar0 + 8u * (18 + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * 20);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* n_entries = reinterpret_cast<volatile int*>(tmem_slot + 2);
  uint32_t* bits = reinterpret_cast<uint32_t*>(aligned + C::OFF_BITS);
  uint16_t* list = reinterpret_cast<uint16_t*>(aligned + C::OFF_LIST);
  volatile const uint16_t* entries = list;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // ---- (request, head, 256 query rows) of this CTA; heads of a request one after the other, so that the CTAs resident at
  // one time share the keys of a few heads
  int head = 0, qb = blockIdx.x, req = 0;
  for (int i = 0; i < batch.n; ++i) {
    req = batch.order[i];
    const int nb = (batch.cu_q[req + 1] - batch.cu_q[req] + C::Q_ROWS - 1) / C::Q_ROWS;
    if (qb < nb * p.n_heads) { head = qb / nb; qb -= head * nb; break; }
    qb -= nb * p.n_heads;
  }
  const int q_begin = batch.cu_q[req], q_len = batch.cu_q[req + 1] - q_begin;
  const int kv_begin = batch.cu_kv[req], kv_len = batch.cu_kv[req + 1] - kv_begin;
  const int n_kv = (kv_len + 127) >> 7, n_windows = (n_kv + kWindowBlocks - 1) / kWindowBlocks;
  const bool tile1_valid = qb * C::Q_ROWS + 128 < q_len;
  const long long row_of_lists = static_cast<long long>(head) * batch.first_qblock[batch.n] + batch.first_qblock[req] + 2 * qb;
  const int* lists[2] = {p.index + row_of_lists * p.ld_index, p.index + (row_of_lists + 1) * p.ld_index};
  auto list_length = [&](int i) {
    if (i == 1 && !tile1_valid) return 0;
    return static_cast<int>(min(static_cast<long long>(max(__ldg(p.count + row_of_lists + i), 0)), p.ld_index));
  };

  if (threadIdx.x < 2 * kWindowBlocks / 32) bits[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    mbar_init(s_free, 4);
    mbar_init(win_full, 1);
    mbar_init(win_empty, tile1_valid ? 11 : 7);          // producer, two issuers, four warps per query tile
    for (int s = 0; s < C::K_STAGES; ++s) { mbar_init(k_full(s), 1); mbar_init(k_empty(s), 1); }
    for (int s = 0; s < C::V_STAGES; ++s) { mbar_init(v_full(s), 1); mbar_init(v_empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(s_full(i), 1); mbar_init(p_full(i), 4); mbar_init(o_full(i), 1); }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV); }
  if (warp == 1) { tmem_alloc(smem_u32(tmem_slot), 512); tmem_relinquish(); }
  __syncthreads();
  for (int i = 0; i < 2; ++i) mark_blocks(bits + i * (kWindowBlocks / 32), lists[i], list_length(i), 0, n_kv, threadIdx.x, C::THREADS);
  __syncthreads();
  if (warp == 3) {
    const int n = order_blocks(bits, list, lane);
    if (lane == 0) *n_entries = n;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t tS = tmem_base, tP = tmem_base + 128, tO = tmem_base + 256;      // columns: S 128, P 2 x 64, O 2 x 128
  // Every role walks all windows: waits until the window's entries are laid out, and says when it has read them.
  auto window_begin = [&](int w) { return w == 0 || mbar_wait(win_full, (w - 1) & 1u, abort_flag); };

  if (warp < 4) {
    DIT_SETMAXNREG_DEC(96);
    if (warp == 0) {
      if (lane == 0) {
        // ---------------------------------------------------------------- TMA producer
        mbar_arrive_expect_tx(q_full, 2 * C::TILE_BYTES);
        for (int i = 0; i < 2; ++i)
          for (int pn = 0; pn < C::NP; ++pn)
            tma_load_2d(base + C::OFF_Q + i * C::TILE_BYTES + pn * C::PANEL, &tmQ, head * D + pn * 64, q_begin + qb * C::Q_ROWS + i * 128, q_full);
        int ks = 0, vs = 0; uint32_t kph = 1, vph = 1;
        for (int w = 0; w < n_windows; ++w) {
          if (!window_begin(w)) goto done;
          const int n = *n_entries;
          for (int e = 0; e < n; ++e) {
            const int y = kv_begin + (w * kWindowBlocks + (entries[e] >> 2)) * 128;
            if (!mbar_wait(k_empty(ks), kph, abort_flag)) goto done;
            mbar_arrive_expect_tx(k_full(ks), C::TILE_BYTES);
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + C::OFF_K + ks * C::TILE_BYTES + pn * C::PANEL, &tmK, head * D + pn * 64, y, k_full(ks));
            if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
            if (!mbar_wait(v_empty(vs), vph, abort_flag)) goto done;
            mbar_arrive_expect_tx(v_full(vs), C::TILE_BYTES);
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL, &tmV, head * D + pn * 64, y, v_full(vs));
            if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
          }
          if (w + 1 < n_windows) mbar_arrive(win_empty);
        }
      }
    } else if (warp == 1) {
      if (lane == 0) {
        // ---------------------------------------------------------------- MMA issuer 1: scores
        constexpr uint32_t idesc_s = idesc_f16(128, 128, false, BF16);
        const uint64_t qdesc0 = smem_desc_sw128(base + C::OFF_Q, 16, 1024), kdesc0 = smem_desc_sw128(base + C::OFF_K, 16, 1024);
        constexpr uint32_t kTileStep = C::TILE_BYTES >> 4;
        int ks = 0; uint32_t kph = 0, u = 0;                                      // u: uses of S so far
        if (!mbar_wait(q_full, 0, abort_flag)) goto done;
        for (int w = 0; w < n_windows; ++w) {
          if (!window_begin(w)) goto done;
          const int n = *n_entries;
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
              if (i == 1 || tiles == 1) umma_commit(k_empty(ks));                 // the entry's last use of its K tile
              umma_commit(s_full(i));
            }
            if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
          }
          if (w + 1 < n_windows) mbar_arrive(win_empty);
        }
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ MMA issuer 2: P V (the whole warp walks the list: it also
      // clears the V rows behind the request's last key)
      constexpr uint32_t idesc_pv = idesc_f16(128, D, true, BF16);
      const uint64_t vdesc0 = smem_desc_sw128(base + C::OFF_V, C::PANEL, 1024);
      constexpr uint32_t kTileStep = C::TILE_BYTES >> 4;
      int vs = 0; uint32_t vph = 0, uses[2] = {0, 0};
      for (int w = 0; w < n_windows; ++w) {
        if (!__all_sync(0xffffffffu, window_begin(w))) goto done;
        const int n = *n_entries;
        for (int e = 0; e < n; ++e) {
          const int tiles = entries[e] & 3, j = w * kWindowBlocks + (entries[e] >> 2);
          if (!__all_sync(0xffffffffu, mbar_wait(v_full(vs), vph, abort_flag))) goto done;
          const int valid = kv_len - j * 128;
          if (valid < 128) {
            for (int r = valid * 8 + lane; r < 128 * 8; r += 32)                  // 16-byte units of rows valid .. 127
              for (int pn = 0; pn < C::NP; ++pn)
                *reinterpret_cast<uint4*>(aligned + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL + r * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
          }
          const uint64_t vd = vdesc0 + vs * kTileStep;
          for (int i = 0; i < 2; ++i) {
            if (!((tiles >> i) & 1)) continue;
            if (!__all_sync(0xffffffffu, mbar_wait(p_full(i), uses[i] & 1u, abort_flag))) goto done;
            tc_fence_after();
            if (lane == 0) {
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                umma_f16_ts(tO + i * 128, tP + i * 64 + kk * 8, vd + kk * (2048 >> 4), idesc_pv, (uses[i] | kk) != 0);
              if (i == 1 || tiles == 1) umma_commit(v_empty(vs));
              umma_commit(o_full(i));
            }
            __syncwarp();
            ++uses[i];
          }
          if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
        }
        __syncwarp();
        if (w + 1 < n_windows && lane == 0) mbar_arrive(win_empty);
      }
    } else {
      // ------------------------------------------------------------------ further windows' lists
      for (int w = 1; w < n_windows; ++w) {
        if (!__all_sync(0xffffffffu, mbar_wait(win_empty, (w - 1) & 1u, abort_flag))) goto done;
        bits[lane] = 0;
        __syncwarp();
        for (int i = 0; i < 2; ++i) mark_blocks(bits + i * (kWindowBlocks / 32), lists[i], list_length(i), w * kWindowBlocks, n_kv, lane, 32);
        __syncwarp();
        const int n = order_blocks(bits, list, lane);
        if (lane == 0) *n_entries = n;
        __syncwarp();
        if (lane == 0) mbar_arrive(win_full);
      }
    }
  } else {
    // -------------------------------------------------------------------- softmax + accumulate (2 warpgroups)
    DIT_SETMAXNREG_INC(200);
    const int tile = (warp >> 2) - 1, quarter = warp & 3;
    if (tile == 1 && !tile1_valid) goto done;
    const uint32_t lane_sel = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tSi = tS + lane_sel, tPi = tP + tile * 64 + lane_sel, tOi = tO + tile * 128 + lane_sel;
    const float c = p.scale_log2;
    const float2 c2 = make_float2(c, c);
    constexpr float kRescaleLog2 = 8.0f;       // O is rescaled when a row's maximum has grown by more than 2^8: P stays <= 2^8
    float m_ref = -INFINITY, l = 0.f;
    uint32_t use = 0;                          // key blocks of this tile so far

    for (int w = 0; w < n_windows; ++w) {
      if (!__all_sync(0xffffffffu, window_begin(w))) goto done;
      const int n = *n_entries;
      for (int e = 0; e < n; ++e) {
        const int entry = entries[e];
        if (!((entry >> tile) & 1)) continue;
        if (!__all_sync(0xffffffffu, mbar_wait(s_full(tile), use & 1u, abort_flag))) goto done;
        tc_fence_after();
        const int valid = kv_len - (w * kWindowBlocks + (entry >> 2)) * 128;
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
        if (use == 0) {
          m_ref = mx;
        } else {
          const bool grow = (mx - m_ref) * c > kRescaleLog2;
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
        }
        // a reference of -inf (every score so far -inf, from infinite inputs) would make the exponents NaN
        const float neg_mc = m_ref == -INFINITY ? 0.f : -m_ref * c;
        const float2 nm2 = make_float2(neg_mc, neg_mc);
        float2 rs0 = make_float2(0.f, 0.f), rs1 = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 128; i += 2) {
          const float2 x = ffma2(make_float2(__uint_as_float(sv[i]), __uint_as_float(sv[i + 1])), c2, nm2);
          const float2 ex = make_float2(exp2_approx(x.x), exp2_approx(x.y));
          if (i & 2) rs1 = fadd2(rs1, ex); else rs0 = fadd2(rs0, ex);
          sv[i >> 1] = pack16x2<BF16>(ex.x, ex.y);
        }
        if (use > 0) {                         // P is still read by this tile's previous product until that has finished
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
      if (w + 1 < n_windows && lane == 0) mbar_arrive(win_empty);
    }
    {
      constexpr int ROW_BYTES = D * 2, UNITS = ROW_BYTES / 16, ROWS_PER_STORE = 32 / UNITS;
      const int row0 = qb * C::Q_ROWS + tile * 128 + quarter * 32;               // in the request
      uint16_t* out0 = static_cast<uint16_t*>(p.out) + (static_cast<long long>(q_begin) + row0) * p.ld_out + head * D;
      const int unit = lane % UNITS, sub = lane / UNITS;
      if (use == 0) {                          // no key at all: zeros (Q may still be arriving: nothing is staged)
        for (int rr = sub; rr < 32 && row0 + rr < q_len; rr += ROWS_PER_STORE)
          *(reinterpret_cast<uint4*>(out0 + rr * p.ld_out) + unit) = make_uint4(0, 0, 0, 0);
        goto done;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(o_full(tile), (use - 1) & 1u, abort_flag))) goto done;
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      // rows leave through the shared memory of the tile's Q (its last score product has finished), 16-byte units
      // XOR-swizzled by the row, so that stores cover whole rows
      uint8_t* stage = aligned + C::OFF_Q + tile * C::TILE_BYTES + quarter * 32 * ROW_BYTES;
#pragma unroll 1
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t r[32];
        __syncwarp();
        tmem_ld32(tOi + ch * 32, r);
        tmem_ld_wait();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          uint32_t wd[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) wd[h] = pack16x2<BF16>(__uint_as_float(r[8 * v + 2 * h]) * inv, __uint_as_float(r[8 * v + 2 * h + 1]) * inv);
          *reinterpret_cast<uint4*>(stage + lane * ROW_BYTES + (((ch * 4 + v) ^ (lane & (UNITS - 1))) << 4)) = make_uint4(wd[0], wd[1], wd[2], wd[3]);
        }
      }
      __syncwarp();
#pragma unroll 4
      for (int it = 0; it < 32 / ROWS_PER_STORE; ++it) {
        const int rr = it * ROWS_PER_STORE + sub;
        if (row0 + rr < q_len) {
          const uint4 val = *reinterpret_cast<const uint4*>(stage + rr * ROW_BYTES + ((unit ^ (rr & (UNITS - 1))) << 4));
          *(reinterpret_cast<uint4*>(out0 + rr * p.ld_out) + unit) = val;
        }
      }
    }
  }

done:
  tc_fence_before();
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, 512); }
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusAttnTimeout);
}

// ------------------------------------------------------------------------------------------------
// Few query rows per request (a new token or two against a stored context).  Reading the selected K and V blocks once is the
// bound; one row per key does not fill a tensor-core tile.  A cluster of CTAs shares a (request, head): rank r takes
// every splits-th selected block.  K and V tiles arrive by TMA in swizzled panels; warp w works on keys 32 w .. 32 w + 31 of
// every tile on its own: lane = key for the scores (16-byte reads of 32 different rows, free of bank conflicts thanks
// to the swizzle), lane = four (two) channels for P V, running maximum and sum per warp.  The warps' results
// meet in shared memory, the CTAs' through distributed shared memory, in rank and warp order.
// ------------------------------------------------------------------------------------------------
template <int D>
struct BlockRowsCfg {
  static constexpr int NP = D / 64, PANEL = 128 * 128, TILE_BYTES = NP * PANEL;
  static constexpr int K_STAGES = 2, V_STAGES = 1 * (128 / D);                   // 96 KB (d = 128), 64 KB (d = 64)
  static constexpr int OFF_K = 0, OFF_V = K_STAGES * TILE_BYTES, OFF_BAR = OFF_V + V_STAGES * TILE_BYTES;
  static constexpr int OFF_BITS = OFF_BAR + 128;                                 // uint32 [kMaxKeyBlocks / 32]
  static constexpr int OFF_Q = OFF_BITS + kMaxKeyBlocks / 8;                     // float [4][D]
  static constexpr int OFF_PART = OFF_Q + 4 * D * 4;                             // float [4 warps][4 rows][D + 2]
  static constexpr int SMEM_BYTES = OFF_PART + 16 * (D + 2) * 4 + 1024;
  static constexpr int THREADS = 160;                                            // four key warps and a producer
  static_assert(2 * SMEM_BYTES <= 227 * 1024, "two CTAs per SM");
};

template <bool BF16>
__device__ __forceinline__ float2 widen2(uint32_t w) {
  if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

template <int D, bool BF16, int R>
__global__ void __launch_bounds__(BlockRowsCfg<D>::THREADS)
block_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const BlockAttnParams p, const uint16_t* q,
                  const long long ld_q, const __grid_constant__ BlockBatch batch, const int splits) {
  using C = BlockRowsCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto k_full = [&](int s) { return bar0 + 8u * s; };
  auto k_empty = [&](int s) { return bar0 + 8u * (2 + s); };
  auto v_full = [&](int s) { return bar0 + 8u * (4 + s); };
  auto v_empty = [&](int s) { return bar0 + 8u * (6 + s); };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(aligned + C::OFF_BAR + 64);
  uint32_t* bits = reinterpret_cast<uint32_t*>(aligned + C::OFF_BITS);
  float* qs = reinterpret_cast<float*>(aligned + C::OFF_Q);
  float* part = reinterpret_cast<float*>(aligned + C::OFF_PART);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int item = blockIdx.x / splits, head = item % p.n_heads, req = item / p.n_heads;
  const int q_begin = batch.cu_q[req], rows = batch.cu_q[req + 1] - q_begin;      // 0 .. R
  const int kv_begin = batch.cu_kv[req], kv_len = batch.cu_kv[req + 1] - kv_begin;
  const int n_kv = (kv_len + 127) >> 7, words = (n_kv + 31) >> 5;

  for (int i = threadIdx.x; i < words; i += C::THREADS) bits[i] = 0;
  for (int i = threadIdx.x; i < R * D; i += C::THREADS) {
    const int r = i / D;
    uint32_t v = 0;
    if (r < rows) v = q[(static_cast<long long>(q_begin) + r) * ld_q + head * D + i % D];
    qs[i] = widen2<BF16>(v).x;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) { mbar_init(k_full(s), 1); mbar_init(k_empty(s), 4); mbar_init(v_full(s), 1); mbar_init(v_empty(s), 4); }
    *abort_flag = 0;
    fence_mbar_init();
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

  float m[R], l[R];                            // per warp: running maximum (of score * scale * log2 e), per-lane sum
  constexpr int CPL = D / 32;                  // channels per lane: 4 or 2
  float acc[R][CPL];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) acc[r][i] = 0.f;
  }
  bool ok = true;
  if (warp == 4) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int ks = 0, vs = 0, turn = 0; uint32_t kph = 1, vph = 1;
      for (int w = 0; w < words && ok; ++w)
        for (uint32_t b = bits[w]; b && ok; b &= b - 1) {
          if (turn++ % splits != rank) continue;
          const int y = kv_begin + (w * 32 + __ffs(b) - 1) * 128;
          if (!(ok = mbar_wait(k_empty(ks), kph, abort_flag))) break;
          mbar_arrive_expect_tx(k_full(ks), C::TILE_BYTES);
          for (int pn = 0; pn < C::NP; ++pn) tma_load_2d(base + C::OFF_K + ks * C::TILE_BYTES + pn * C::PANEL, &tmK, head * D + pn * 64, y, k_full(ks));
          if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
          if (!(ok = mbar_wait(v_empty(vs), vph, abort_flag))) break;
          mbar_arrive_expect_tx(v_full(vs), C::TILE_BYTES);
          for (int pn = 0; pn < C::NP; ++pn) tma_load_2d(base + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL, &tmV, head * D + pn * 64, y, v_full(vs));
          if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
        }
    }
  } else {
    // ------------------------------------------------------------------ keys 32 * warp .. + 31 of every tile
    int ks = 0, vs = 0, turn = 0; uint32_t kph = 0, vph = 0;
    for (int w = 0; w < words && ok; ++w)
      for (uint32_t b = bits[w]; b && ok; b &= b - 1) {
        if (turn++ % splits != rank) continue;
        const int keys = min(32, kv_len - (w * 32 + __ffs(b) - 1) * 128 - 32 * warp);    // of this warp (may be <= 0)
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(k_full(ks), kph, abort_flag)))) break;
        float s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = 0.f;
        {
          const int row = 32 * warp + lane;
          const uint8_t* kt = aligned + C::OFF_K + ks * C::TILE_BYTES + row * 128;
#pragma unroll 4
          for (int u = 0; u < D / 8; ++u) {
            const uint4 k4 = *reinterpret_cast<const uint4*>(kt + (u >> 3) * C::PANEL + (((u & 7) ^ (row & 7)) << 4));
            const float2 k0 = widen2<BF16>(k4.x), k1 = widen2<BF16>(k4.y), k2 = widen2<BF16>(k4.z), k3 = widen2<BF16>(k4.w);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 qa = *reinterpret_cast<const float4*>(qs + r * D + u * 8), qb = *reinterpret_cast<const float4*>(qs + r * D + u * 8 + 4);
              s[r] = fmaf(qa.x, k0.x, s[r]); s[r] = fmaf(qa.y, k0.y, s[r]); s[r] = fmaf(qa.z, k1.x, s[r]); s[r] = fmaf(qa.w, k1.y, s[r]);
              s[r] = fmaf(qb.x, k2.x, s[r]); s[r] = fmaf(qb.y, k2.y, s[r]); s[r] = fmaf(qb.z, k3.x, s[r]); s[r] = fmaf(qb.w, k3.y, s[r]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(k_empty(ks));
        if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
        float pr[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float x = lane < keys ? s[r] * p.scale_log2 : -INFINITY;
          float mx = x;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const float top = fmaxf(m[r], mx), at = top == -INFINITY ? 0.f : top;
          const float alpha = exp2_approx(m[r] - at);                  // 0 while m is -inf
          pr[r] = lane < keys ? exp2_approx(x - at) : 0.f;
          l[r] = l[r] * alpha + pr[r];
          m[r] = top;
#pragma unroll
          for (int i = 0; i < CPL; ++i) acc[r][i] *= alpha;
        }
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(v_full(vs), vph, abort_flag)))) break;
        {
          // channels CPL * lane ..: 16-byte unit (lane * CPL) / 8 of the row, swizzled by the row
          const int ch = lane * CPL, panel = ch / 64, unit = (ch % 64) / 8, in = (ch % 8) * 2;
          const uint8_t* vt = aligned + C::OFF_V + vs * C::TILE_BYTES + panel * C::PANEL + in;
#pragma unroll 8
          for (int k = 0; k < keys; ++k) {
            const int row = 32 * warp + k;
            const uint8_t* at = vt + row * 128 + ((unit ^ (row & 7)) << 4);
            float v[CPL];
            if constexpr (CPL == 4) {
              const uint2 t = *reinterpret_cast<const uint2*>(at);
              const float2 a = widen2<BF16>(t.x), c = widen2<BF16>(t.y);
              v[0] = a.x; v[1] = a.y; v[2] = c.x; v[3] = c.y;
            } else {
              const float2 a = widen2<BF16>(*reinterpret_cast<const uint32_t*>(at));
              v[0] = a.x; v[1] = a.y;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float pk = __shfl_sync(0xffffffffu, pr[r], k);
#pragma unroll
              for (int i = 0; i < CPL; ++i) acc[r][i] = fmaf(pk, v[i], acc[r][i]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(v_empty(vs));
        if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
      }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
      float* dst = part + (warp * R + r) * (D + 2);
#pragma unroll
      for (int i = 0; i < CPL; ++i) dst[lane * CPL + i] = acc[r][i];
      if (lane == 0) { dst[D] = m[r]; dst[D + 1] = l[r]; }
    }
  }
  __syncwarp();
  if (splits > 1) cluster_sync_all(); else __syncthreads();
  if (rank == 0 && threadIdx.x < 128) {
    // row after row, channel per thread: the parts rescaled to their common maximum
    for (int r = 0; r < rows; ++r) {
      auto read = [&](int s, int w, int i) {
        const float* at = part + (w * R + r) * (D + 2) + i;
        return splits > 1 ? ld_cluster_f32(map_to_cta(smem_u32(at), s)) : *at;
      };
      float top = -INFINITY;
      for (int s = 0; s < splits; ++s)
        for (int w = 0; w < 4; ++w) top = fmaxf(top, read(s, w, D));
      const float ref = top == -INFINITY ? 0.f : top;
      for (int ch = threadIdx.x; ch < D; ch += 128) {
        float sum = 0.f, o = 0.f;
        for (int s = 0; s < splits; ++s)
          for (int w = 0; w < 4; ++w) {
            const float f = exp2_approx(read(s, w, D) - ref);
            sum = fmaf(f, read(s, w, D + 1), sum);
            o = fmaf(f, read(s, w, ch), o);
          }
        static_cast<uint16_t*>(p.out)[(static_cast<long long>(q_begin) + r) * p.ld_out + head * D + ch] = pack16<BF16>(sum == 0.f ? 0.f : o / sum);
      }
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
// The means of k are stored transposed, [column][key block], as the products read them.
// ------------------------------------------------------------------------------------------------
struct BlockSelectParams {
  const uint16_t *q, *k;
  long long ld_q, ld_k;
  int width, n_heads, head_dim;
  double* q_mean;            // [query blocks, width]
  double* k_mean;            // [width, key blocks]
  int* index;
  int* count;
  long long ld_index;
  int widest;                // largest keep: entries of a list that are written
  int rows;                  // query blocks per CTA of the selecting kernel
  int keep[DIT_MAX_REQUESTS], tail[DIT_MAX_REQUESTS];
};

// One CTA per (block, 256 columns): eight warps take every eighth row, a lane 16 bytes of it.  Bound by reading q and k once.
template <bool BF16>
__global__ void __launch_bounds__(256)
block_means_kernel(const BlockSelectParams p, const __grid_constant__ BlockBatch batch) {
  __shared__ double sums[8][256];
  const int q_blocks = batch.first_qblock[batch.n], k_blocks = batch.first_kblock[batch.n];
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = warp + 8 * (8 * h + i);
        v[i] = r < n ? __ldg(reinterpret_cast<const uint4*>(src + r * ld)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float2 f = widen2<BF16>(u[c]);
          acc[2 * c] += static_cast<double>(f.x); acc[2 * c + 1] += static_cast<double>(f.y);
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
    if (is_k) p.k_mean[static_cast<long long>(mine) * k_blocks + block] = s;
    else p.q_mean[static_cast<long long>(block) * p.width + mine] = s;
  }
}

// Order-preserving map of a score to an unsigned number: NaN lowest, the two zeros alike.
__device__ __forceinline__ unsigned long long score_key(double s) {
  if (s != s) return 0ull;
  const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(s + 0.0));
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// One CTA per (head, up to four query blocks of a request): every thread scores key blocks against the four rows, then a
// warp per row finds the keep-th largest score by deciding its bits from the top (counting the scores that reach
// the candidate; most rows are decided after a few bits, when exactly `keep` do) and writes the list in order.
constexpr int kSelectRows = 4;

__global__ void __launch_bounds__(256)
block_select_kernel(const BlockSelectParams p, const __grid_constant__ BlockBatch batch) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  double* qm = reinterpret_cast<double*>(smem_raw);                              // [head_dim][kSelectRows]
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(smem_raw + 128 * kSelectRows * 8);   // [rows][n_kv]
  const int q_blocks = batch.first_qblock[batch.n], k_blocks = batch.first_kblock[batch.n];
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
  for (int i = threadIdx.x; i < d * kSelectRows; i += 256) {
    const int r = i % kSelectRows, c = i / kSelectRows;
    qm[i] = r < n_rows ? p.q_mean[static_cast<long long>(qb0 + r) * p.width + head * d + c] : 0.0;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < n_kv; j += 256) {
    double s[kSelectRows];
#pragma unroll
    for (int r = 0; r < kSelectRows; ++r) s[r] = 0.0;
    const double* km = p.k_mean + static_cast<long long>(head * d) * k_blocks + kb0 + j;
#pragma unroll 8
    for (int c = 0; c < d; ++c) {
      const double k = __ldg(km + static_cast<long long>(c) * k_blocks);
#pragma unroll
      for (int r = 0; r < kSelectRows; ++r) s[r] = fma(qm[c * kSelectRows + r], k, s[r]);
    }
    const bool forced = p.tail[req] > 0 && static_cast<long long>(j + 1) * 128 > static_cast<long long>(kv_len) - p.tail[req];
#pragma unroll
    for (int r = 0; r < kSelectRows; ++r)
      if (r < n_rows) keys[static_cast<long long>(r) * n_kv + j] = forced ? ~0ull : score_key(s[r]);
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp >= n_rows) return;
  const unsigned long long* mine = keys + static_cast<long long>(warp) * n_kv;
  const int want = min(p.keep[req], n_kv);
  unsigned long long least = 0;                // keys >= least: at least `want`
  int reach = n_kv;                            // how many they are
  for (int bit = 63; bit >= 0 && reach != want; --bit) {
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
  for (int e = want + lane; e < p.widest; e += 32) list[e] = -1;
  if (lane == 0) p.count[at] = want;
}

}  // namespace dit
