// Attention over packed requests with grouped heads: every query row over the keys of its request up to its own place (causal) or over all.
//
// prompt_attention_kernel   two tiles of 128 query rows that share a key head per CTA, on the tensor cores, for many rows
// prompt_rows_kernel        up to 16 rows (query rows x heads of a group) per CTA over a part of the keys, for a few rows against a long
//                           context; prompt_join_kernel joins the parts
#pragma once
#include <type_traits>

#include "attention.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace dit {

// Packed batch, passed by value.  `order`: the requests that a launch takes.
struct PromptBatch {
  int n;                     // entries of order
  int cu_q[DIT_MAX_REQUESTS + 1], cu_kv[DIT_MAX_REQUESTS + 1];
  int order[DIT_MAX_REQUESTS];
};

struct PromptAttnParams {
  void* out;
  long long ld_out;
  const uint16_t* q;
  const uint16_t* v;         // for values that are no finite numbers in places that only some rows see
  long long ld_q, ld_v;
  int n_heads, kv_heads, group;
  int causal;
  float scale_log2;          // scale * log2(e), positive
  int items;                 // tiled kernel: pairs, or their parts
  int most_blocks;           // key blocks of the longest of its requests
  int pairs;                 // (request, key head, pair of query tiles)
  int part_blocks;           // key blocks of an item at most (0: a pair is one item)
  float* tile_parts;         // [items][2][head_dim + 4][128]
  int wide_out;              // rows of out start on 32-byte boundaries
  int* status;
  // few rows
  int chunk;                 // keys per CTA, a multiple of 64
  int beside;                // the tiled kernel of the same call is in front
  float* parts;              // [CTAs][16][head_dim + 4]
};

// The 16-bit value's exponent is all ones: an infinity or NaN.
template <bool BF16>
__device__ __forceinline__ bool odd_bits(uint32_t h) { return (h & (BF16 ? 0x7F80u : 0x7C00u)) == (BF16 ? 0x7F80u : 0x7C00u); }
template <bool BF16>
__device__ __forceinline__ float widen16bit(uint32_t h) {
  return BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
}
// A pair of 16-bit values with infinities and NaN replaced by zero; *odd becomes true where one was.
template <bool BF16>
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool* odd) {
  const bool lo = odd_bits<BF16>(w & 0xFFFFu), hi = odd_bits<BF16>(w >> 16);
  *odd |= lo || hi;
  return (lo ? 0u : w & 0xFFFFu) | (hi ? 0u : w & 0xFFFF0000u);
}

template <int D>
struct PromptAttnCfg {
  static constexpr int NP = D / 64, PANEL = 128 * 128, TILE_BYTES = NP * PANEL;
  static constexpr int K_STAGES = 3, V_STAGES = 2;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + K_STAGES * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_V + V_STAGES * TILE_BYTES;
  static constexpr int OFF_ITEM = OFF_BAR + 256;                                  // PromptItem [2]
  static constexpr int SMEM_USED = OFF_ITEM + 2 * 64 + 1024;
  // one CTA per SM: each takes all of tensor memory
  static constexpr int SMEM_BYTES = SMEM_USED > 116 * 1024 ? SMEM_USED : 116 * 1024;
  static constexpr int THREADS = 384;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};

// Two query tiles: consecutive ones of the list (last 128-row block first, the heads of the group one after the other) of a request and a key
// head.  With an even group they are two heads' tiles of the same rows; otherwise also neighbouring row blocks.  An item is a pair, or, where
// there are few pairs and long ones, up to part_blocks of its key blocks.
struct PromptItem {
  int kv_head, q_begin, q_len, kv_begin, kv_len;
  int before;                // keys before the first query row's own (may be negative)
  int head[2], qb[2];
  int first, end[2];         // key blocks of the item, per tile (end[1] <= end[0]; none where end <= first)
  int ragged;                // first key block of which some row of a tile sees only a part
  int tile1;
  int slot;                  // place of its partial results, or -1: it is the whole pair
  __device__ __forceinline__ int limit(int row, int causal) const { return causal ? min(kv_len, before + row + 1) : kv_len; }   // keys of a row
};
// Pairs of tiles of a request whose first tile sees `blocks` key blocks or more (they are the request's first ones).
__host__ __device__ inline int pairs_of(int q_len, int kv_len, int group, int causal, int blocks) {
  const int nb = (q_len + 127) >> 7;
  int from = 0;                                // first row block that qualifies
  if (blocks > 0) {
    if (blocks > (kv_len + 127) >> 7) return 0;
    if (causal) {
      from = ((128 * (blocks - 1) + 1 - (kv_len - q_len) + 127) >> 7) - 1;
      if (from < 0) from = 0;
    }
  }
  return ((nb - from) * group + 1) >> 1;
}
__device__ __forceinline__ int pairs_with(const PromptBatch& batch, int group, int causal, int i, int blocks) {
  if (i >= batch.n) return 0;
  const int r = batch.order[i];
  return pairs_of(batch.cu_q[r + 1] - batch.cu_q[r], batch.cu_kv[r + 1] - batch.cu_kv[r], group, causal, blocks);
}
// Pairs of the batch that see `blocks` key blocks or more; the whole warp counts.
__device__ __forceinline__ int all_pairs_with(const PromptBatch& batch, const PromptAttnParams& p, int blocks, int lane) {
  const unsigned mine = static_cast<unsigned>(pairs_with(batch, p.group, p.causal, lane, blocks) + (batch.n > 32 ? pairs_with(batch, p.group, p.causal, lane + 32, blocks) : 0));
  return static_cast<int>(__reduce_add_sync(0xffffffffu, mine)) * p.kv_heads;
}
// The item-th item: the first parts of all pairs, most key blocks first, whatever request they belong to, then the second parts of those that
// have one, and so on.  (The pairs with a t-th part are the first ones of that order.)  The whole warp looks for it.
template <bool kParts>
__device__ __forceinline__ PromptItem prompt_item(const PromptBatch& batch, const PromptAttnParams& p, int item, int lane) {
  int layer = 0, rank = item;
  if constexpr (kParts)
    for (int n = p.pairs; rank >= n;) {
      rank -= n;
      ++layer;
      n = all_pairs_with(batch, p, layer * p.part_blocks + 1, lane);
      if (n == 0) break;                       // (no such item)
    }
  int low = 0, high = p.most_blocks + 1, behind = 0;              // more than `rank` pairs have `low` blocks or more; `behind` of them `high`
  while (high - low > 1) {
    const int mid = (low + high) >> 1, n = all_pairs_with(batch, p, mid, lane);
    if (n > rank) low = mid; else { high = mid; behind = n; }
  }
  rank -= behind;                                                 // among the pairs with exactly `low` blocks
  int i = 0, pair = 0, kv_head = 0;
  for (int half = 0; half < 2; ++half) {
    const int first = pairs_with(batch, p.group, p.causal, lane + 32 * half, high);
    const int mine = (pairs_with(batch, p.group, p.causal, lane + 32 * half, low) - first) * p.kv_heads;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    const unsigned past = __ballot_sync(0xffffffffu, sum > rank);
    if (past) {
      const int at = __ffs(past) - 1, within = rank - __shfl_sync(0xffffffffu, sum - mine, at);
      i = at + 32 * half;
      pair = __shfl_sync(0xffffffffu, first, at) + within / p.kv_heads;
      kv_head = within % p.kv_heads;
      break;
    }
    rank -= __shfl_sync(0xffffffffu, sum, 31);
  }
  PromptItem it{};
  const int r = batch.order[i];
  it.kv_head = kv_head;
  it.q_begin = batch.cu_q[r]; it.q_len = batch.cu_q[r + 1] - it.q_begin;
  it.kv_begin = batch.cu_kv[r]; it.kv_len = batch.cu_kv[r + 1] - it.kv_begin;
  it.before = it.kv_len - it.q_len;
  const int row_blocks = (it.q_len + 127) >> 7, tiles = row_blocks * p.group;
  it.tile1 = 2 * pair + 1 < tiles;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int tile = min(2 * pair + t, tiles - 1), back = tile / p.group;
    it.qb[t] = row_blocks - 1 - back;
    it.head[t] = kv_head * p.group + tile - back * p.group;
    it.end[t] = (max(0, it.limit(min(it.q_len, it.qb[t] * 128 + 128) - 1, p.causal)) + 127) >> 7;
  }
  if (!it.tile1) it.end[1] = 0;
  it.ragged = p.causal ? max(0, it.limit((it.tile1 ? it.qb[1] : it.qb[0]) * 128, 1)) >> 7 : it.end[0];
  it.first = layer * p.part_blocks;
  it.slot = -1;
  if (kParts && it.end[0] > p.part_blocks) {
    it.slot = item;
    it.end[0] = min(it.end[0], it.first + p.part_blocks);
    it.end[1] = min(it.end[1], it.first + p.part_blocks);
  }
  return it;
}

// The scheme of the list kernel (block_attention_kernel: two 128-row query tiles with a softmax warpgroup each, one S buffer handed between
// them, P in tensor memory, O rescaled rarely, persistent grid whose roles run on from item to item) over the key blocks 0 .. n - 1 of a
// request.  Sharing a key head is what makes a pair: a key block is loaded once and used by both tiles.
// Items are ordered by their cost over the whole batch and dealt out forwards and backwards in turn, so that CTAs come out even (four requests of
// 2048 rows one after the other: 159 us, ordered: 131).  A warp of its own finds them ahead and hands them to the others through shared memory.
// A causal tile masks its last block or two.  Scores that a row does not see are dropped before its maximum.  Values that it does not
// see meet a probability of zero, which an infinity or NaN would turn into NaN: in the blocks that some rows see only in part such values are
// replaced by zeros in shared memory, and if there was one, the rows that do see it add it to their results at the end.
// Probabilities are rounded to the inputs' type, in which the tensor cores take both operands of the second product; their sum is of the unrounded ones.
// It moves a result of many keys by 1.5e-3 of itself in bf16 and 1.5e-4 in fp16 (2-norms), where the rounding of the result alone moves it by 1.65e-3 and
// 2.1e-4.  Keeping what is rounded off would take a third product of the same size beside the two.
// What bounds it: the softmax chain of two tiles against the products of one S buffer, 1.7 us per key block and pair of tiles, 2.6 us more per pair.
// 8192 rows, 32 heads of 128 over 8 key heads, causal: 396-430 us (1.28-1.39 PFLOP/s) under the power cap.
// kParts: items may be parts of pairs.  (A kernel of its own: with it the ordinary one took 4 to 8 % longer, 8192 rows of 32 heads 452 us for 419.)
template <int D, bool BF16, bool kParts>
__global__ void __launch_bounds__(PromptAttnCfg<D>::THREADS, 1)
prompt_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                        const PromptAttnParams p, const __grid_constant__ PromptBatch batch) {
  using C = PromptAttnCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  const uint32_t q_full = bar0, q_empty = bar0 + 8u, s_free = bar0 + 16u;
  auto k_full = [&](int s) { return bar0 + 8u * (3 + s); };
  auto k_empty = [&](int s) { return bar0 + 8u * (6 + s); };
  auto v_full = [&](int s) { return bar0 + 8u * (9 + s); };
  auto v_empty = [&](int s) { return bar0 + 8u * (11 + s); };
  auto s_full = [&](int i) { return bar0 + 8u * (13 + i); };
  auto p_full = [&](int i) { return bar0 + 8u * (15 + i); };
  auto o_full = [&](int i) { return bar0 + 8u * (17 + i); };
  auto item_full = [&](int b) { return bar0 + 8u * (19 + b); };
  auto item_empty = [&](int b) { return bar0 + 8u * (21 + b); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aligned + C::OFF_BAR + 8 * 23);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* odd_values = reinterpret_cast<volatile int*>(tmem_slot + 2);      // [2]: a tile's item met values that were replaced

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(s_free, 4);
    for (int s = 0; s < C::K_STAGES; ++s) { mbar_init(k_full(s), 1); mbar_init(k_empty(s), 1); }
    for (int s = 0; s < C::V_STAGES; ++s) { mbar_init(v_full(s), 1); mbar_init(v_empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(s_full(i), 1); mbar_init(p_full(i), 4); mbar_init(o_full(i), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(item_full(b), 1); mbar_init(item_empty(b), 11); }     // producer, two issuers, eight softmax warps
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV); }
  if (warp == 1) { tmem_alloc(smem_u32(tmem_slot), 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // What is in front is complete before anything of this call begins: the few-row kernel beside this one does not wait itself.
  await_predecessor();
  dependents_may_start();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t tS = tmem_base, tP = tmem_base + 128, tO = tmem_base + 256;      // columns: S 128, P 2 x 64, O 2 x 128

  // this CTA's k-th item: forwards and backwards in turn
  auto item_at = [&](int k) { return k * static_cast<int>(gridDim.x) + ((k & 1) ? static_cast<int>(gridDim.x - 1 - blockIdx.x) : static_cast<int>(blockIdx.x)); };
  static_assert(sizeof(PromptItem) <= 64, "room of an item");
  auto item_slot = [&](int k) { return reinterpret_cast<PromptItem*>(aligned + C::OFF_ITEM + (k & 1) * 64); };
  // its description, copied; `one`: called by a single thread
  auto take_item = [&](int k, PromptItem& it, bool one) {
    if (one) {
      if (!mbar_wait(item_full(k & 1), (k >> 1) & 1u, abort_flag)) return false;
      it = *item_slot(k);
      mbar_arrive(item_empty(k & 1));
    } else {
      if (!__all_sync(0xffffffffu, mbar_wait(item_full(k & 1), (k >> 1) & 1u, abort_flag))) return false;
      it = *item_slot(k);
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty(k & 1));
    }
    return true;
  };

  if (warp < 4) {
    DIT_SETMAXNREG_DEC(96);
    if (warp == 0) {
      if (lane == 0) {
        // ---------------------------------------------------------------- TMA producer
        int ks = 0, vs = 0; uint32_t kph = 1, vph = 1, qph = 1;
        PromptItem it;
        for (int k = 0; item_at(k) < p.items; ++k) {
          if (!take_item(k, it, true)) goto done;
          if (!mbar_wait(q_empty, qph, abort_flag)) goto done;
          qph ^= 1u;
          mbar_arrive_expect_tx(q_full, (it.tile1 ? 2 : 1) * C::TILE_BYTES);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            for (int pn = 0; pn < (i == 0 || it.tile1 ? C::NP : 0); ++pn)
              tma_load_2d(base + C::OFF_Q + i * C::TILE_BYTES + pn * C::PANEL, &tmQ, it.head[i] * D + pn * 64, it.q_begin + it.qb[i] * 128, q_full);
          for (int j = kParts ? it.first : 0; j < it.end[0]; ++j) {
            const int y = it.kv_begin + j * 128;
            if (!mbar_wait(k_empty(ks), kph, abort_flag)) goto done;
            mbar_arrive_expect_tx(k_full(ks), C::TILE_BYTES);
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + C::OFF_K + ks * C::TILE_BYTES + pn * C::PANEL, &tmK, it.kv_head * D + pn * 64, y, k_full(ks));
            if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
            if (!mbar_wait(v_empty(vs), vph, abort_flag)) goto done;
            mbar_arrive_expect_tx(v_full(vs), C::TILE_BYTES);
            for (int pn = 0; pn < C::NP; ++pn)
              tma_load_2d(base + C::OFF_V + vs * C::TILE_BYTES + pn * C::PANEL, &tmV, it.kv_head * D + pn * 64, y, v_full(vs));
            if (++vs == C::V_STAGES) { vs = 0; vph ^= 1u; }
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
        PromptItem it;
        for (int k = 0; item_at(k) < p.items; ++k) {
          if (!take_item(k, it, true)) goto done;
          if (!mbar_wait(q_full, qph, abort_flag)) goto done;
          qph ^= 1u;
          for (int j = kParts ? it.first : 0; j < it.end[0]; ++j) {
            const int tiles = j < it.end[1] ? 2 : 1;
            if (!mbar_wait(k_full(ks), kph, abort_flag)) goto done;
            for (int i = 0; i < tiles; ++i) {
              if (u > 0 && !mbar_wait(s_free, (u - 1) & 1u, abort_flag)) goto done;
              ++u;
              tc_fence_after();
              const uint64_t qd = qdesc0 + i * kTileStep, kd = kdesc0 + ks * kTileStep;
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * C::PANEL + (kk & 3) * 32) >> 4;
                umma_f16(tS, qd + off, kd + off, idesc_s, kk != 0);
              }
              if (i == tiles - 1) umma_commit(k_empty(ks));
              umma_commit(s_full(i));
            }
            if (++ks == C::K_STAGES) { ks = 0; kph ^= 1u; }
          }
          umma_commit(q_empty);                                                   // Q may be replaced once these products have read it
        }
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ MMA issuer 2: P V; the whole warp clears the V rows behind a
      // request's last key and replaces what is no finite number in blocks that some rows see in part
      constexpr uint32_t idesc_pv = idesc_f16(128, D, true, BF16);
      const uint64_t vdesc0 = smem_desc_sw128(base + C::OFF_V, C::PANEL, 1024);
      constexpr uint32_t kTileStep = C::TILE_BYTES >> 4;
      int vs = 0; uint32_t vph = 0, done_uses[2] = {0, 0};
      PromptItem it;
      for (int k = 0; item_at(k) < p.items; ++k) {
        if (!take_item(k, it, false)) goto done;
        bool odd = false;                                                         // values replaced in this item (warp-uniform)
        int checked = -1;                                                         // last key block that has been looked through
        // Looks through the V tile of key block j in `stage`, which has arrived.
        auto look_through = [&](int j, int stage) {
          checked = j;
          const int valid = it.kv_len - j * 128;
          if (valid >= 128 && j < it.ragged) return;
          uint8_t* tile = aligned + C::OFF_V + stage * C::TILE_BYTES;
          bool wrote = false;
          if (valid < 128) {
            wrote = true;
            for (int r = valid * 8 + lane; r < 128 * 8; r += 32)                  // 16-byte units of rows valid .. 127
              for (int pn = 0; pn < C::NP; ++pn) *reinterpret_cast<uint4*>(tile + pn * C::PANEL + r * 16) = make_uint4(0, 0, 0, 0);
          }
          if (j >= it.ragged) {
            constexpr uint32_t kExp = BF16 ? 0x7F80u : 0x7C00u;
            const int units = min(128, valid) * 8;
            uint32_t most = 0;                                                    // largest magnitudes of the odd and the even columns
            for (int pn = 0; pn < C::NP; ++pn)
#pragma unroll 4
              for (int r = lane; r < units; r += 32) {
                const uint4 w = *reinterpret_cast<const uint4*>(tile + pn * C::PANEL + r * 16);
                most = __vmaxu2(__vmaxu2(__vmaxu2(most, w.x & 0x7FFF7FFFu), __vmaxu2(w.y & 0x7FFF7FFFu, w.z & 0x7FFF7FFFu)), w.w & 0x7FFF7FFFu);
              }
            if (__any_sync(0xffffffffu, (most & 0xFFFFu) >= kExp || (most >> 16) >= kExp)) {
              odd = wrote = true;
              bool unused = false;
              for (int pn = 0; pn < C::NP; ++pn)
                for (int r = lane; r < units; r += 32) {
                  uint4* at = reinterpret_cast<uint4*>(tile + pn * C::PANEL + r * 16);
                  const uint4 w = *at;
                  *at = make_uint4(finite_pair<BF16>(w.x, &unused), finite_pair<BF16>(w.y, &unused), finite_pair<BF16>(w.z, &unused), finite_pair<BF16>(w.w, &unused));
                }
            }
          }
          if (wrote) {
            fence_proxy_async_smem();
            __syncwarp();
          }
        };
        for (int j = kParts ? it.first : 0; j < it.end[0]; ++j) {
          const int tiles = j < it.end[1] ? 2 : 1;
          const int next = vs + 1 == C::V_STAGES ? 0 : vs + 1;
          if (checked != j) {
            if (!__all_sync(0xffffffffu, mbar_wait(v_full(vs), vph, abort_flag))) goto done;
            look_through(j, vs);
          }
          const uint64_t vd = vdesc0 + vs * kTileStep;
          for (int i = 0; i < tiles; ++i) {
            if (!__all_sync(0xffffffffu, mbar_wait(p_full(i), done_uses[i] & 1u, abort_flag))) goto done;
            tc_fence_after();
            if (lane == 0) {
              // (the tile's warps are in this item, since they have handed over a P of it: they no longer read the last item's word)
              odd_values[i] = odd;
              __threadfence_block();
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                umma_f16_ts(tO + i * 128, tP + i * 64 + kk * 8, vd + kk * (2048 >> 4), idesc_pv, j != (kParts ? it.first : 0) || kk != 0);
              if (i == tiles - 1) umma_commit(v_empty(vs));
              umma_commit(o_full(i));
            }
            __syncwarp();
            ++done_uses[i];
            // the next block, while the other tile's P is still being made (looking through it in its own turn cost 3 % of long prompts)
            if (i == 0 && tiles == 2 && j + 1 < it.end[0] && __all_sync(0xffffffffu, mbar_test_wait(v_full(next), vph ^ (next == 0 ? 1u : 0u)))) look_through(j + 1, next);
          }
          vs = next;
          if (vs == 0) vph ^= 1u;
        }
      }
    } else {
      // ------------------------------------------------------------------ the coming items
      for (int k = 0; item_at(k) < p.items; ++k) {
        const PromptItem it = prompt_item<kParts>(batch, p, item_at(k), lane);
        if (!__all_sync(0xffffffffu, mbar_wait(item_empty(k & 1), ((k >> 1) & 1u) ^ 1u, abort_flag))) goto done;
        if (lane == 0) {
          *item_slot(k) = it;
          mbar_arrive(item_full(k & 1));
        }
        __syncwarp();
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

    PromptItem it;
    for (int k = 0; item_at(k) < p.items; ++k) {
      if (!take_item(k, it, false)) goto done;
      const int qb = tile == 0 ? it.qb[0] : it.qb[1], head = tile == 0 ? it.head[0] : it.head[1], end = tile == 0 ? it.end[0] : it.end[1];
      const int row = qb * 128 + quarter * 32 + lane;                             // in the request
      const int limit = it.limit(row, p.causal);
      float m_ref = -INFINITY, l = 0.f;
      const uint32_t first_use = use;
      for (int j = kParts ? it.first : 0; j < end; ++j) {
        if (!__all_sync(0xffffffffu, mbar_wait(s_full(tile), use & 1u, abort_flag))) goto done;
        tc_fence_after();
        const int valid = limit - j * 128;   // keys of the block that the row sees (may be <= 0)
        uint32_t sv[128];
        __syncwarp();
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) tmem_ld32p(tSi + ch * 32, sv + ch * 32);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_free);
        if (__any_sync(0xffffffffu, valid < 128)) {
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
      if (tile == 1 && !it.tile1) continue;
      uint16_t* out = static_cast<uint16_t*>(p.out) + (static_cast<long long>(it.q_begin) + row) * p.ld_out + head * D;
      const bool any = use != first_use;       // without a key: zeros
      bool odd = false;
      if (any) {
        if (!__all_sync(0xffffffffu, mbar_wait(o_full(tile), (use - 1) & 1u, abort_flag))) goto done;
        tc_fence_after();
        odd = odd_values[tile] != 0;
      }
      if (kParts && it.slot >= 0) {            // a part: sums as they are, reference and sum of probabilities (nothing where the tile has no block in it)
        if (any) {
          // channel by channel, so that a warp's rows lie side by side
          float* to = p.tile_parts + (static_cast<long long>(it.slot) * 2 + tile) * (D + 4) * 128 + quarter * 32 + lane;
#pragma unroll 1
          for (int ch = 0; ch < D / 32; ++ch) {
            uint32_t r[32];
            __syncwarp();
            tmem_ld32(tOi + ch * 32, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) to[(ch * 32 + i) * 128] = __uint_as_float(r[i]);
          }
          to[D * 128] = m_ref; to[(D + 1) * 128] = l; to[(D + 2) * 128] = odd ? 1.f : 0.f;
        }
        continue;
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      // The results of 32 channels at a time; `kept` writes infinities as such, with the replaced values that the row sees, and is a second
      // pass over the rare rows that have one, so that the ordinary one pays for the largest magnitude only.
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
            if constexpr (decltype(kept)::value) {
              if (odd) {                       // (a factor of 1 / l is positive: it leaves infinities and NaN as they are)
                const uint16_t* v = p.v + (static_cast<long long>(it.kv_begin) + it.ragged * 128) * p.ld_v + it.kv_head * D + ch * 32;
                for (int key = it.ragged * 128; key < limit; ++key, v += p.ld_v) {
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (odd_bits<BF16>(v[i])) r[i] = __float_as_uint(__uint_as_float(r[i]) + widen16bit<BF16>(v[i]));
                }
              }
            }
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
      if (__any_sync(0xffffffffu, odd || fmaxf(largest[0], largest[1]) == INFINITY)) write(std::true_type{});
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
// Few rows.  The query rows of a request and the heads of a group make rows of one product with the group's keys (row i * group + h), 16 to
// a CTA, so that a new token's heads read the keys once.  Reading the stored keys and values is the bound: a CTA takes p.chunk of them,
// chosen so that one CTA per SM covers the batch, however uneven its requests are.  Inside it is block_rows_kernel: K and V by TMA in
// tiles of 64 keys through one ring, four warps with 16 keys of every tile each, warp-level products (probabilities rounded as above), the warps' results joined in
// shared memory.  A request with one chunk writes its rows; the parts of the others go to memory as (sums, maximum, sum of
// probabilities) and prompt_join_kernel joins them in their order.
// 32 heads of 128 over 8 key heads, us: one row against 32768 keys (134 MB) 28, of which 3 are the joining kernel; 64 rows of 64 requests against 4096 keys
// each (1.07 GB) 153 = 7.0 TB/s, part of it from L2.  Heads of 64 take half the bytes and nearly the same time per key (23 us): a tile's waits and
// dependent steps, not its bytes, are the bound there.
// ------------------------------------------------------------------------------------------------
template <int D>
struct PromptRowsCfg {
  static constexpr int NP = D / 64, PANEL = kRowsTile * 128, TILE_BYTES = NP * PANEL;
  static constexpr int STAGES = 96 * 1024 / TILE_BYTES;                          // 6 (d = 128), 12 (d = 64)
  static constexpr int OFF_BAR = STAGES * TILE_BYTES;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  static constexpr int THREADS = 160;                                            // four key warps and a producer
  static constexpr int PART = D + 4;                                             // floats of a row's partial result: channels, maximum, sum, values replaced
  static_assert(4 * kRowsMax * PART * 4 <= OFF_BAR, "the partial results take the ring's place");
  static_assert(2 * SMEM_BYTES <= 227 * 1024, "two CTAs per SM");
};

// Where a CTA of the few-row kernels works: CTAs are counted request by request, key head by key head, row tile by row tile, chunk by chunk.
struct PromptPart {
  int req, kv_head, row0, part, parts;         // parts of the request
  int q_begin, q_len, kv_begin, kv_len, before;
};
__host__ __device__ inline int prompt_row_tiles(int q_len, int group) { return (q_len * group + kRowsMax - 1) / kRowsMax; }
__host__ __device__ inline int prompt_parts(int kv_len, int chunk) { return kv_len > chunk ? (kv_len + chunk - 1) / chunk : 1; }
__device__ __forceinline__ PromptPart prompt_part(const PromptBatch& batch, const PromptAttnParams& p, int cta) {
  PromptPart w{};
  for (int i = 0; i < batch.n; ++i) {
    w.req = batch.order[i];
    w.q_begin = batch.cu_q[w.req]; w.q_len = batch.cu_q[w.req + 1] - w.q_begin;
    w.kv_begin = batch.cu_kv[w.req]; w.kv_len = batch.cu_kv[w.req + 1] - w.kv_begin;
    w.parts = prompt_parts(w.kv_len, p.chunk);
    const int tiles = prompt_row_tiles(w.q_len, p.group), here = tiles * w.parts * p.kv_heads;
    if (cta < here) {
      w.part = cta % w.parts;
      const int rest = cta / w.parts;
      w.row0 = rest % tiles * kRowsMax;
      w.kv_head = rest / tiles;
      break;
    }
    cta -= here;
  }
  w.before = w.kv_len - w.q_len;
  return w;
}
// Keys that row i of the request sees.
__device__ __forceinline__ int prompt_limit(const PromptPart& w, const PromptAttnParams& p, int i) {
  return p.causal ? max(0, min(w.kv_len, w.before + i + 1)) : w.kv_len;
}
// Four finished channels of a row; odd: some values were replaced, and those that the row sees (keys first .. limit - 1) are added.
template <bool BF16>
__device__ __forceinline__ void prompt_store(const PromptAttnParams& p, const PromptPart& w, int row, int channel, int d, float4 o, int first, bool odd) {
  const int i = row / p.group, head = w.kv_head * p.group + row - i * p.group;
  float x[4] = {o.x, o.y, o.z, o.w};
  if (odd) {
    const int limit = prompt_limit(w, p, i);
    const uint16_t* v = p.v + (static_cast<long long>(w.kv_begin) + first) * p.ld_v + w.kv_head * d + channel;
    for (int key = first; key < limit; ++key, v += p.ld_v)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (odd_bits<BF16>(v[c])) x[c] += widen16bit<BF16>(v[c]);
  }
  uint2 r = make_uint2(pack16x2<BF16>(x[0], x[1]), pack16x2<BF16>(x[2], x[3]));
  r.x = put_infinities<BF16>(r.x, x[0], x[1]);
  r.y = put_infinities<BF16>(r.y, x[2], x[3]);
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + (static_cast<long long>(w.q_begin) + i) * p.ld_out + head * d + channel) = r;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(PromptRowsCfg<D>::THREADS, 2)
prompt_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const PromptAttnParams p,
                   const __grid_constant__ PromptBatch batch) {
  using C = PromptRowsCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - raw);
  const uint32_t bar0 = base + C::OFF_BAR;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(aligned + C::OFF_BAR + 16 * C::STAGES);
  volatile int* odd_values = abort_flag + 1;                            // a value was replaced
  float* part = reinterpret_cast<float*>(aligned);                      // [4 warps][kRowsMax][PART], after the main loop

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PromptPart w = prompt_part(batch, p, blockIdx.x);
  const int rows = min(kRowsMax, w.q_len * p.group - w.row0);           // of this CTA, 1 .. kRowsMax
  const int first = prompt_limit(w, p, w.row0 / p.group);               // keys that all of its rows see
  const int most = prompt_limit(w, p, (w.row0 + rows - 1) / p.group);   // keys that the last one sees
  const int begin = w.part * p.chunk, end = min(most, begin + p.chunk); // of this CTA (begin may be >= end)

  // Beside the tiled kernel, which has waited for what is in front of both, this one waits at its end only.  (Then too what follows the call
  // is behind both.)
  if (!p.beside) await_predecessor();
  dependents_may_start();                      // (the joining kernel waits for this one's end)
  // The producer's thread sets the barriers up and requests the first tiles before the CTA meets.
  auto load = [&](int n, int stage) {          // tile n: K, V, K, V, ... of the keys from `begin` on
    mbar_arrive_expect_tx(full(stage), C::TILE_BYTES);
    for (int pn = 0; pn < C::NP; ++pn)
      tma_load_2d(base + stage * C::TILE_BYTES + pn * C::PANEL, (n & 1) ? &tmV : &tmK, w.kv_head * D + pn * 64, w.kv_begin + begin + (n >> 1) * kRowsTile, full(stage));
  };
  const int tiles = end > begin ? 2 * ((end - begin + kRowsTile - 1) / kRowsTile) : 0;
  if (threadIdx.x == 128) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 4); }
    *abort_flag = 0; *odd_values = 0;
    fence_mbar_init();
    for (int n = 0; n < min(tiles, C::STAGES); ++n) load(n, n);
  }
  // Q as the first operand: k step t, rows lane / 4 and + 8, channels 16 t + 2 (lane % 4) and + 8; absent rows are zero
  uint32_t qa[D / 16][4];
  int limit[2] = {0, 0};                                                // keys of the lane's two rows
  if (warp < 4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (lane >> 2) + 8 * h, row = w.row0 + r, i = row / p.group;
      const uint16_t* q = p.q + (static_cast<long long>(w.q_begin) + i) * p.ld_q + (w.kv_head * p.group + row - i * p.group) * D;
      if (r < rows) limit[h] = prompt_limit(w, p, i);
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        const int c = t * 16 + (lane & 3) * 2;
        qa[t][h] = r < rows ? *reinterpret_cast<const uint32_t*>(q + c) : 0u;
        qa[t][2 + h] = r < rows ? *reinterpret_cast<const uint32_t*>(q + c + 8) : 0u;
      }
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
      int stage = 0; uint32_t phase = 0;
      for (int n = C::STAGES; n < tiles && ok; ++n) {
        if (!(ok = mbar_wait(empty(stage), phase, abort_flag))) break;
        load(n, stage);
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------------ keys 16 * warp .. + 15 of every tile
    int stage = 0; uint32_t phase = 0;
    // row addresses of the ldmatrix loads: of K, matrices (keys 0-7 | 8-15) x (channels 0-7, 8-15 of a k step); of V, transposed,
    // (channels 0-7 | 8-15 of a pair of output tiles) x (keys 0-7, 8-15)
    const int k_row = 16 * warp + (lane >> 4) * 8 + (lane & 7), k_unit = (lane >> 3) & 1;
    const int v_row = 16 * warp + ((lane >> 3) & 1) * 8 + (lane & 7), v_unit = lane >> 4;
    for (int y = begin; y < end && ok; y += kRowsTile) {
      const int key0 = y + 16 * warp;                                   // this warp's first key
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(stage), phase, abort_flag)))) break;
      float s[2][4] = {};                                               // keys 0-7 and 8-15
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
      const bool ragged = key0 + 16 > first;                            // some row does not see all of the warp's keys
      if (ragged) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (key0 + 8 * i + 2 * (lane & 3) + (k & 1) >= limit[k >> 1]) s[i][k] = -INFINITY;
      }
      uint32_t pa[4];
#pragma unroll
      for (int r = 0; r < 2; ++r) {                                     // rows lane / 4 + 8 r
        float mx = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // the reference is taken off before the scaling: the largest score's exponent is 0 however large the factor is
        const float top = fmaxf(m[r], mx), at = top == -INFINITY ? 0.f : top;
        const float alpha = exp2_approx((m[r] - at) * p.scale_log2);    // 0 while m is -inf
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
      if (ragged) {                            // V rows that no row sees are cleared, of the others what is no finite number
        bool odd = false;
        for (int i = lane; i < 16 * 8; i += 32) {
          const int key = key0 + (i >> 3);
          if (key < first) continue;
          for (int pn = 0; pn < C::NP; ++pn) {
            uint4* at = reinterpret_cast<uint4*>(aligned + stage * C::TILE_BYTES + pn * C::PANEL + (16 * warp * 8 + i) * 16);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (key < most) {
              v = *at;
              v = make_uint4(finite_pair<BF16>(v.x, &odd), finite_pair<BF16>(v.y, &odd), finite_pair<BF16>(v.z, &odd), finite_pair<BF16>(v.w, &odd));
            }
            *at = v;
          }
        }
        if (odd) *odd_values = 1;
        fence_proxy_async_smem();              // the stage is refilled by TMA
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
  __syncthreads();
  // The warps' parts rescaled to their common maximum: a thread per row finds the factors, which take the places of the maxima, then four
  // channels per thread and turn.
  if (threadIdx.x < rows) {
    float top = -INFINITY, sum = 0.f;
    float* at = part + threadIdx.x * C::PART + D;
    constexpr int kWarp = kRowsMax * C::PART;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, at[k * kWarp]);
    const float ref = top == -INFINITY ? 0.f : top;
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[k] = exp2_approx((at[k * kWarp] - ref) * p.scale_log2);
      sum += at[k * kWarp + 1] * f[k];
    }
    if (w.parts > 1) {
      float* to = p.parts + (static_cast<long long>(blockIdx.x) * kRowsMax + threadIdx.x) * C::PART + D;
      *reinterpret_cast<float4*>(to) = make_float4(top, sum, static_cast<float>(*odd_values), 0.f);
      sum = 1.f;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k * kWarp] = f[k] * inv;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * (D / 4); i += C::THREADS) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    const float* from = part + row * C::PART;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(from + k * kRowsMax * C::PART + c);
      const float f = from[k * kRowsMax * C::PART + D];
      o = make_float4(fmaf(x.x, f, o.x), fmaf(x.y, f, o.y), fmaf(x.z, f, o.z), fmaf(x.w, f, o.w));
    }
    if (w.parts > 1) *reinterpret_cast<float4*>(p.parts + (static_cast<long long>(blockIdx.x) * kRowsMax + row) * C::PART + c) = o;
    else prompt_store<BF16>(p, w, w.row0 + row, c, D, o, first, *odd_values != 0);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicMax(p.status, kStatusAttnTimeout);
  await_predecessor();
}

// A warp per row of a row tile with several parts (grid: row tiles x 4, four rows each): the parts rescaled to their common maximum, in order.  Lanes hold
// the parts' factors, 32 at a time, and four (d = 128) or two channels each.
constexpr int kJoinRows = 4;
template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinRows * 32)
prompt_join_kernel(const PromptAttnParams p, const __grid_constant__ PromptBatch batch) {
  constexpr int PART = PromptRowsCfg<D>::PART;
  // row tiles are counted request by request, key head by key head
  int tile = blockIdx.x, cta = 0;
  PromptPart w{};
  for (int i = 0; i < batch.n; ++i) {
    w.req = batch.order[i];
    w.q_begin = batch.cu_q[w.req]; w.q_len = batch.cu_q[w.req + 1] - w.q_begin;
    w.kv_begin = batch.cu_kv[w.req]; w.kv_len = batch.cu_kv[w.req + 1] - w.kv_begin;
    w.parts = prompt_parts(w.kv_len, p.chunk);
    const int tiles = prompt_row_tiles(w.q_len, p.group), here = tiles * p.kv_heads;
    if (tile < here) {
      w.row0 = tile % tiles * kRowsMax;
      w.kv_head = tile / tiles;
      cta += tile * w.parts;
      break;
    }
    tile -= here;
    cta += here * w.parts;
  }
  w.before = w.kv_len - w.q_len;
  const int row = blockIdx.y * kJoinRows + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (w.parts == 1 || row >= w.q_len * p.group - w.row0) return;
  await_predecessor();                    // the parts are complete
  const float* from = p.parts + (static_cast<long long>(cta) * kRowsMax + row) * PART;
  constexpr long long kStep = static_cast<long long>(kRowsMax) * PART;
  const int c = lane * 4;                                               // (d = 64: half of the lanes hold channels)
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float ref = -INFINITY, sum = 0.f, odd = 0.f;
  for (int k0 = 0; k0 < w.parts; k0 += 32) {
    const int n = min(32, w.parts - k0);
    const float4 mine = lane < n ? *reinterpret_cast<const float4*>(from + (k0 + lane) * kStep + D) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    float top = fmaxf(ref, mine.x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    const float at = top == -INFINITY ? 0.f : top;
    const float keep = exp2_approx((ref - at) * p.scale_log2), f = exp2_approx((mine.x - at) * p.scale_log2);
    float part = mine.y * f;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) part += __shfl_xor_sync(0xffffffffu, part, s);
    sum = sum * keep + part;
    odd = __any_sync(0xffffffffu, mine.z != 0.f) ? 1.f : odd;
    o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
    ref = top;
#pragma unroll 8
    for (int k = 0; k < n; ++k) {
      const float fk = __shfl_sync(0xffffffffu, f, k);
      const float4 x = c < D ? *reinterpret_cast<const float4*>(from + (k0 + k) * kStep + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      o = make_float4(fmaf(x.x, fk, o.x), fmaf(x.y, fk, o.y), fmaf(x.z, fk, o.z), fmaf(x.w, fk, o.w));
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  if (c < D)
    prompt_store<BF16>(p, w, w.row0 + row, c, D, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), prompt_limit(w, p, w.row0 / p.group), odd != 0.f);
}

// For a tile of a pair with several parts and 32 of its channels: a thread per row and 16 channels.  grid: (pairs, 2 tiles x head_dim / 32).
constexpr int kTileParts = 32;                 // parts of a pair at most
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
prompt_tile_join_kernel(const PromptAttnParams p, const __grid_constant__ PromptBatch batch) {
  __shared__ PromptItem item;
  __shared__ int slot_of[kTileParts];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tile = blockIdx.y / (D / 32);
  if (warp == 0) {
    const PromptItem it = prompt_item<true>(batch, p, blockIdx.x, lane);          // the pair's first part
    if (lane == 0) item = it;
    int n = p.pairs, base = 0;
    for (int t = 0; t < kTileParts && n > static_cast<int>(blockIdx.x); ++t) {    // (the pairs with a t-th part: the first n)
      if (lane == 0) slot_of[t] = base + blockIdx.x;
      base += n;
      n = all_pairs_with(batch, p, (t + 1) * p.part_blocks + 1, lane);
    }
  }
  __syncthreads();
  const PromptItem it = item;
  const int qb = tile == 0 ? it.qb[0] : it.qb[1], head = tile == 0 ? it.head[0] : it.head[1];
  const int blocks = (max(0, it.limit(min(it.q_len, qb * 128 + 128) - 1, p.causal)) + 127) >> 7;
  const int parts = (blocks + p.part_blocks - 1) / p.part_blocks;
  const int in = threadIdx.x & 127, row = qb * 128 + in, c = blockIdx.y % (D / 32) * 32 + (threadIdx.x >> 7) * 16;
  if ((tile == 1 && !it.tile1) || row >= it.q_len) return;
  await_predecessor();                    // the parts are complete
  auto part = [&](int t) { return p.tile_parts + (static_cast<long long>(slot_of[t]) * 2 + tile) * (D + 4) * 128 + in; };
  float top = -INFINITY, odd = 0.f;
#pragma unroll 4
  for (int t = 0; t < parts; ++t) {
    top = fmaxf(top, part(t)[D * 128]);
    odd = fmaxf(odd, part(t)[(D + 2) * 128]);
  }
  const float at = top == -INFINITY ? 0.f : top;
  float sum = 0.f, o[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll 2
  for (int t = 0; t < parts; ++t) {
    const float* from = part(t);
    const float f = exp2_approx((from[D * 128] - at) * p.scale_log2);
    sum += from[(D + 1) * 128] * f;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = fmaf(from[(c + i) * 128], f, o[i]);
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] *= inv;
  if (odd != 0.f) {                            // values were replaced in the blocks that rows see in part: those that this row sees are added
    const int limit = it.limit(row, p.causal);
    const uint16_t* v = p.v + (static_cast<long long>(it.kv_begin) + it.ragged * 128) * p.ld_v + it.kv_head * D + c;
    for (int key = it.ragged * 128; key < limit; ++key, v += p.ld_v)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (odd_bits<BF16>(v[i])) o[i] += widen16bit<BF16>(v[i]);
  }
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = put_infinities<BF16>(pack16x2<BF16>(o[2 * i], o[2 * i + 1]), o[2 * i], o[2 * i + 1]);
  uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (static_cast<long long>(it.q_begin) + row) * p.ld_out + head * D + c);
  out[0] = make_uint4(w[0], w[1], w[2], w[3]);
  out[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

}  // namespace dit
