// Rotary positions and attention over packed prompts (include/dit_ops.h): argument checks, tensor maps, launch rules.
#include <algorithm>
#include <cmath>
#include <functional>
#include <mutex>

#include "common.cuh"
#include "ops_launch.h"
#include "prompt_attention.cuh"
#include "prompt_call.h"
#include "rotary.cuh"

using namespace dit;

namespace {

constexpr int64_t kMaxSize = INT32_MAX - 1024;

int type_bytes(dit_type t) { return t == DIT_TYPE_F32 ? 4 : 2; }
bool type_ok(dit_type t) { return t == DIT_TYPE_F16 || t == DIT_TYPE_BF16 || t == DIT_TYPE_F32; }
bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// units: pieces of a head that lanes take, 0 for the form that takes any alignment.
template <int kType, int kBytes, bool kInterleaved>
cudaError_t launch_rotary(const RotaryParams& p, int units, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>((p.rows + p.rows_per_cta - 1) / p.rows_per_cta);
  switch (units) {
    case 4: return launch_overlapping(&rotary_kernel<kType, 4, kBytes, kInterleaved>, dim3(grid), kRotaryThreads, 0, st, p);
    case 8: return launch_overlapping(&rotary_kernel<kType, 8, kBytes, kInterleaved>, dim3(grid), kRotaryThreads, 0, st, p);
    case 16: return launch_overlapping(&rotary_kernel<kType, 16, kBytes, kInterleaved>, dim3(grid), kRotaryThreads, 0, st, p);
    case 32: return launch_overlapping(&rotary_kernel<kType, 32, kBytes, kInterleaved>, dim3(grid), kRotaryThreads, 0, st, p);
    default: return launch_overlapping(&rotary_kernel<kType, 0, 16, kInterleaved>, dim3(grid), kRotaryThreads, 0, st, p);
  }
}
template <int kType>
cudaError_t launch_rotary(RotaryParams p, const dit_rotary_args& a, cudaStream_t st) {
  // pieces of 16 bytes, of 8 where rows, heads or halves start off 16-byte boundaries; the pieces of a head are rounded up to a power of two,
  // whose last lanes idle (heads of 80: 5 of 8)
  constexpr int kElem = kType == 2 ? 4 : 2;
  for (int bytes = 16; bytes >= 8; bytes /= 2) {
    const int per = bytes / kElem;
    if (!aligned(a.x, bytes) || !aligned(a.out, bytes) || a.ld_x % per || a.ld_out % per || a.head_dim % per || a.rotary_dim % per ||
        (!a.interleaved && p.pairs % per))
      continue;
    p.pieces = (a.interleaved ? a.rotary_dim : p.pairs) / per + (a.head_dim - a.rotary_dim) / per;
    if (p.pieces > 32) break;
    const int units = p.pieces <= 4 ? 4 : (p.pieces <= 8 ? 8 : (p.pieces <= 16 ? 16 : 32));
    if (bytes == 16) return a.interleaved ? launch_rotary<kType, 16, true>(p, units, st) : launch_rotary<kType, 16, false>(p, units, st);
    return a.interleaved ? launch_rotary<kType, 8, true>(p, units, st) : launch_rotary<kType, 8, false>(p, units, st);
  }
  return a.interleaved ? launch_rotary<kType, 16, true>(p, 0, st) : launch_rotary<kType, 16, false>(p, 0, st);
}

// ------------------------------------------------------------------------------------------------ attention
std::mutex g_mutex;
bool g_ready[kOpsMaxDevices];

template <class Kernel>
cudaError_t allow_smem(Kernel kernel, int bytes) {
  return cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int D, bool BF16>
cudaError_t allow_attention() {
  cudaError_t e = allow_smem(&prompt_attention_kernel<D, BF16, false>, PromptAttnCfg<D>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&prompt_attention_kernel<D, BF16, true>, PromptAttnCfg<D>::SMEM_BYTES);
  return e == cudaSuccess ? allow_smem(&prompt_rows_kernel<D, BF16>, PromptRowsCfg<D>::SMEM_BYTES) : e;
}
cudaError_t prepare(const OpsDevice& d) {
  std::lock_guard<std::mutex> lock(g_mutex);
  if (g_ready[d.index]) return cudaSuccess;
  cudaError_t e;
  if ((e = allow_attention<64, false>()) != cudaSuccess || (e = allow_attention<64, true>()) != cudaSuccess ||
      (e = allow_attention<128, false>()) != cudaSuccess || (e = allow_attention<128, true>()) != cudaSuccess)
    return e;
  g_ready[d.index] = true;
  return cudaSuccess;
}

// 16-bit matrix [rows, cols] with row stride ld: boxes of 64 columns x box_rows rows, 128-byte swizzle, zeros outside.
bool half_map(const OpsDevice& d, CUtensorMap* m, const void* ptr, uint64_t cols, uint64_t rows, uint64_t ld, uint32_t box_rows) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {ld * 2};
  const cuuint32_t box[2] = {64, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return d.encode(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a batch is worked on: which requests go to which kernel, and into how many parts their keys are cut.
struct PromptPlan {
  PromptBatch tiled, few;
  int64_t pairs, items;      // of the tiled kernel
  int most_blocks, part_blocks;
  int64_t cut;               // pairs with several parts
  int64_t row_tiles, ctas;   // of the few-row kernel
  int chunk;
  bool join;                 // some request of it has several parts
};
constexpr int kSms = 148;                        // (plans, and with them workspaces, depend on the sizes of a call alone)

// Estimates in us, from measurements.  The tiled kernel takes 7 us for anything, 1.7 for a key block of a pair of tiles (pairs side by side on the
// SMs) and 2.6 per pair; the few-row kernel 4 us, 0.45 for 64 keys of a part, and altogether the time to read the keys once for every 16
// rows, from L2 behind the first time, at 7 TB/s.
constexpr double kPairBlock = 1.7, kPair = 2.6;
struct RequestCost { double few, few_chain, blocks, most, pairs; int64_t rows; int r; };

// Which requests go to the few-row kernel: those of up to some number of rows, which is chosen so that the slower of the longest chain of
// dependent work in either kernel and the work of both spread over the device is least (3 us more where both run).  A lone short prompt of few heads has rows to spread over
// more CTAs than it has pairs (612 rows of 3 heads: 9 pairs, 18.5 us tiled, 10.7 by rows), a batch of many is better off in tiles.
int few_of(const dit_prompt_attention_args& a, RequestCost* c, int n) {
  std::sort(c, c + n, [](const RequestCost& x, const RequestCost& y) { return x.rows != y.rows ? x.rows < y.rows : x.r < y.r; });
  double blocks = 0, pairs = 0, few = 0, chain = 0, most[DIT_MAX_REQUESTS + 1] = {};
  for (int i = n - 1; i >= 0; --i) {             // most[i]: longest pair of the requests i ..
    most[i] = std::max(most[i + 1], c[i].most);
    blocks += c[i].blocks; pairs += c[i].pairs;
  }
  int best = 0;
  double least = 0;
  for (int i = 0; i <= n; ++i) {                 // requests 0 .. i - 1 by rows
    const double work = few + (kPairBlock * blocks + kPair * pairs) / kSms;
    const double time = std::max({work, i > 0 ? 4 + std::max(few, chain) : 0.0, i < n ? 7 + kPairBlock * most[i] : 0.0}) + (i > 0 && i < n ? 3 : 0);
    if (i == 0 || time <= least) { best = i; least = time; }
    if (i == n || c[i].rows > 2048) break;
    few += c[i].few; chain = std::max(chain, c[i].few_chain); blocks -= c[i].blocks; pairs -= c[i].pairs;
  }
  return best;
}

// Key blocks of the pairs of the tiled kernel, most first; returns their number.
int pair_lengths(const PromptPlan& p, const dit_prompt_attention_args& a, int* length) {
  const int group = a.n_heads / a.n_kv_heads;
  int n = 0;
  for (int i = 0; i < p.tiled.n; ++i) {
    const int r = p.tiled.order[i], q_len = a.q_lens[r], kv_len = a.kv_lens[r], row_blocks = (q_len + 127) / 128;
    const int pairs = static_cast<int>((static_cast<int64_t>(row_blocks) * group + 1) / 2);
    for (int pair = 0; pair < pairs; ++pair) {     // (a request's own come most first)
      const int64_t rows = static_cast<int64_t>(row_blocks - 2 * pair / group) * 128;      // up to the end of the pair's first row block
      const int64_t keys = a.causal ? std::max<int64_t>(0, kv_len - q_len + std::min<int64_t>(q_len, rows)) : kv_len;
      length[n++] = static_cast<int>((keys + 127) / 128);
    }
  }
  if (p.tiled.n > 1) std::sort(length, length + n, std::greater<int>());
  for (int i = n - 1; i >= 0; --i)                 // every key head's
    for (int h = 0; h < a.n_kv_heads; ++h) length[i * a.n_kv_heads + h] = length[i];
  return n * a.n_kv_heads;
}
// Time of the fullest CTA when items of up to `part` key blocks are dealt out, first parts, second parts ..., forwards and backwards in turn; *items counts
// them.  Whole parts cost the same, so they are added round by round.
double deal_out(const int* length, int n, int part, int* items) {
  double load[kSms] = {};
  int at = 0, round = 0, count = 0;              // CTAs of the round that have their item
  const double whole = kPairBlock * part + kPair;
  for (int t = 0, m = n; m > 0; ++t) {
    int next = m;                                // pairs with a further part: their t-th is a whole one
    while (next > 0 && length[next - 1] <= (t + 1) * part) --next;
    for (int left = next; left > 0;) {
      const int here = std::min(left, kSms - at), low = (round & 1) ? kSms - at - here : at;
      for (int i = low; i < low + here; ++i) load[i] += whole;
      left -= here; at += here;
      if (at == kSms) { at = 0; ++round; }
    }
    for (int i = next; i < m; ++i) {
      load[(round & 1) ? kSms - 1 - at : at] += kPairBlock * std::min(part, length[i] - t * part) + kPair;
      if (++at == kSms) { at = 0; ++round; }
    }
    count += m;
    m = next;
  }
  *items = count;
  return *std::max_element(load, load + kSms);
}

// Key blocks of an item at most, into p->part_blocks, 0 for whole pairs: cut where the longest pair would outlast the work of all by far, so that few pairs
// are dealt out to many SMs.  The time of a cut is that of the fullest CTA, as the items will be dealt out, and what the parts cost: their results through
// memory and a joining kernel.  us whole, and for the cut that is chosen: 8 heads of 64, 3240 rows 45, 33; 4 heads of 128, 8192 rows
// 101, 77; one head, 16384 rows 190, 78; 128 rows of 32 heads over 8 key heads against 32768 keys 369, 79.
// The host's time is part of a call's: cuts are tried in the order of a bound below their time, until no bound promises less than the best found.
void choose_parts(PromptPlan* p, const dit_prompt_attention_args& a, double blocks) {
  constexpr int kMost = 512, kTries = 64;
  const double chain = kPairBlock * p->most_blocks + kPair, work = (kPairBlock * blocks + kPair * p->pairs) / kSms;
  if (p->pairs > kMost || chain < 1.3 * work + 8.0) return;
  int length[kMost];
  const int n = pair_lengths(*p, a, length);
  double total = 0;
  for (int i = 0; i < n; ++i) total += length[i];
  struct Try { double bound; int part; } tries[kTries];
  int count = 0, longer = n;                     // pairs with more than `part` key blocks, `blocks_of` in all
  double blocks_of = total;
  for (int part = std::max(4, (p->most_blocks + kTileParts - 1) / kTileParts); 3 * part <= 2 * p->most_blocks && count < kTries; part += std::max(1, part / 4)) {
    while (longer > 0 && length[longer - 1] <= part) blocks_of -= length[--longer];
    const double items = n - longer + std::max(2.0 * longer, blocks_of / part);
    const double most = std::max(kPairBlock * part + kPair, (kPairBlock * total + kPair * items) / kSms);
    tries[count++] = Try{most + 6.0 + 0.06 * items, part};
  }
  std::sort(tries, tries + count, [](const Try& x, const Try& y) { return x.bound != y.bound ? x.bound < y.bound : x.part < y.part; });
  double least = 0.95 * chain;
  int best = 0, best_items = 0;
  for (int i = 0; i < count && tries[i].bound * (1.0 - 1e-9) <= least; ++i) {
    int items = 0;
    const double time = deal_out(length, n, tries[i].part, &items) + 6.0 + 0.06 * items;
    if (time < least || (time == least && best > 0 && tries[i].part < best)) { least = time; best = tries[i].part; best_items = items; }
  }
  if (best == 0) return;
  p->part_blocks = best;
  p->items = best_items;
  for (p->cut = 0; p->cut < n && length[p->cut] > best; ++p->cut) {}
}

// Checks sizes and lays the batch out.
dit_status plan_prompts(const dit_prompt_attention_args& a, PromptPlan* p) {
  if (a.n_requests < 0 || a.n_heads < 1 || a.n_kv_heads < 1 || a.n_heads % a.n_kv_heads || (a.type != DIT_TYPE_F16 && a.type != DIT_TYPE_BF16)) return DIT_ERR_INVALID_ARG;
  if (a.head_dim != 64 && a.head_dim != 128) return DIT_ERR_SHAPE;
  if (a.n_requests > DIT_MAX_REQUESTS) return DIT_ERR_CAPACITY;
  if (a.n_requests > 0 && (!a.q_lens || !a.kv_lens)) return DIT_ERR_INVALID_ARG;
  if (static_cast<int64_t>(a.n_heads) * a.head_dim > (1 << 20)) return DIT_ERR_SHAPE;
  *p = PromptPlan{};
  const int64_t group = a.n_heads / a.n_kv_heads;
  const bool causal = a.causal != 0;
  int64_t q = 0, kv = 0;
  RequestCost cost[DIT_MAX_REQUESTS];
  int n = 0;
  for (int r = 0; r <= a.n_requests; ++r) {
    p->tiled.cu_q[r] = p->few.cu_q[r] = static_cast<int>(q);
    p->tiled.cu_kv[r] = p->few.cu_kv[r] = static_cast<int>(kv);
    if (r == a.n_requests) break;
    const int64_t q_len = a.q_lens[r], kv_len = a.kv_lens[r];
    if (q_len < 0 || kv_len < 0) return DIT_ERR_INVALID_ARG;
    q += q_len; kv += kv_len;
    if (q > kMaxSize || kv > kMaxSize) return DIT_ERR_SHAPE;
    if (q_len == 0) continue;
    RequestCost& c = cost[n++];
    c.r = r; c.rows = q_len * group;
    c.few = static_cast<double>((c.rows + kRowsMax - 1) / kRowsMax) * a.n_kv_heads * kv_len * a.head_dim * 4 * 1e-6 / 7.0;
    const double tiles = static_cast<double>((c.rows + kRowsMax - 1) / kRowsMax) * a.n_kv_heads;
    c.few_chain = 0.45 / 64 * std::max(std::min<double>(kv_len, 256.0), std::min<double>(kv_len, tiles * kv_len / kSms)) + (kv_len > 256 ? 3.0 : 0.0);
    c.pairs = static_cast<double>(((q_len + 127) / 128 * group + 1) / 2 * a.n_kv_heads);
    c.most = static_cast<double>((kv_len + 127) / 128);
    // keys that the row blocks' last rows see: evenly from the first block's to the last one's
    const double first = causal ? std::max<double>(0.0, std::min<double>(kv_len, kv_len - q_len + std::min<int64_t>(q_len, 128))) : static_cast<double>(kv_len);
    c.blocks = c.pairs * (0.5 * (first + kv_len) / 128 + 0.5);
  }
  const int few = few_of(a, cost, n);
  double blocks = 0, keys = 0;
  for (int i = 0; i < n; ++i) {
    const int r = cost[i].r;
    PromptBatch& b = i < few ? p->few : p->tiled;
    int at = b.n++;
    for (; at > 0 && a.kv_lens[b.order[at - 1]] < a.kv_lens[r]; --at) b.order[at] = b.order[at - 1];      // most keys first
    b.order[at] = r;
    if (i < few) {
      const int64_t tiles = static_cast<int64_t>(a.n_kv_heads) * prompt_row_tiles(a.q_lens[r], static_cast<int>(group));
      p->row_tiles += tiles;
      keys += static_cast<double>(tiles) * a.kv_lens[r];
    } else {
      p->most_blocks = std::max(p->most_blocks, static_cast<int>((static_cast<int64_t>(a.kv_lens[r]) + 127) / 128));
      blocks += cost[i].blocks;
      p->pairs += ((((static_cast<int64_t>(a.q_lens[r]) + 127) / 128) * group + 1) / 2) * a.n_kv_heads;
    }
  }
  if (p->pairs > INT32_MAX / 16) return DIT_ERR_SHAPE;
  p->items = p->pairs;
  if (p->pairs > 0) choose_parts(p, a, blocks);
  if (p->few.n > 0) {
    // Parts of equal length, one for each SM: what a CTA costs before its first product and after its last one is several us, and one per SM
    // keeps enough loads in flight (one row of 32 heads against 32768 keys, parts of 256, 896, 1792 keys: 60, 34, 29 us).  Beyond 4096 keys
    // a part is only cut off: more CTAs than SMs are resident at once, and share the memory's bandwidth evenly.
    const int least = static_cast<int>(std::min(4096.0, std::max(256.0, std::ceil(keys / kSms / 64) * 64)));
    int64_t tiles[DIT_MAX_REQUESTS], ctas;
    int keys_of[DIT_MAX_REQUESTS];
    for (int i = 0; i < p->few.n; ++i) {
      const int r = p->few.order[i];
      tiles[i] = static_cast<int64_t>(a.n_kv_heads) * prompt_row_tiles(a.q_lens[r], static_cast<int>(group));
      keys_of[i] = a.kv_lens[r];
    }
    auto ctas_with = [&](int chunk) {
      int64_t n = 0;
      for (int i = 0; i < p->few.n; ++i) n += tiles[i] * prompt_parts(keys_of[i], chunk);
      return n;
    };
    int chunk = least;
    while ((ctas = ctas_with(chunk)) > kSms && chunk < 2 * least) chunk += std::max(64, least / 16 / 64 * 64);
    p->chunk = std::min(chunk, 4096);
    p->ctas = p->chunk == chunk ? ctas : ctas_with(p->chunk);
    if (p->ctas > INT32_MAX / 16) return DIT_ERR_SHAPE;
    p->join = p->ctas > p->row_tiles;
  }
  return DIT_OK;
}
// Room for the parts of the few-row kernel, then for those of the tiled one.
size_t few_bytes(const PromptPlan& p, int head_dim) { return p.join ? static_cast<size_t>(p.ctas) * kRowsMax * (head_dim + 4) * sizeof(float) : 0; }
size_t part_bytes(const PromptPlan& p, int head_dim) { return few_bytes(p, head_dim) + (p.part_blocks > 0 ? static_cast<size_t>(p.items) * 2 * 128 * (head_dim + 4) * sizeof(float) : 0); }

template <int D, bool BF16>
cudaError_t launch_attention(const OpsDevice& d, const dit_prompt_attention_args& a, const PromptPlan& plan, PromptAttnParams p, void* workspace, cudaStream_t st) {
  const uint64_t width = static_cast<uint64_t>(a.n_heads) * D, kv_width = static_cast<uint64_t>(a.n_kv_heads) * D;
  const int q_rows = plan.tiled.cu_q[a.n_requests], kv_rows = plan.tiled.cu_kv[a.n_requests];
  // without keys nothing is loaded; the maps still have to describe some memory
  const void* k = kv_rows > 0 ? a.k : a.q;
  const void* v = kv_rows > 0 ? a.v : a.q;
  const uint64_t ld_k = kv_rows > 0 ? a.ld_k : a.ld_q, ld_v = kv_rows > 0 ? a.ld_v : a.ld_q;
  CUtensorMap tmQ, tmK, tmV;
  cudaError_t e;
  if (plan.items > 0) {
    if (!half_map(d, &tmQ, a.q, width, q_rows, a.ld_q, 128) || !half_map(d, &tmK, k, kv_width, std::max(kv_rows, 1), ld_k, 128) ||
        !half_map(d, &tmV, v, kv_width, std::max(kv_rows, 1), ld_v, 128))
      return cudaErrorInvalidValue;
    p.items = static_cast<int>(plan.items); p.pairs = static_cast<int>(plan.pairs);
    p.most_blocks = plan.most_blocks; p.part_blocks = plan.part_blocks;
    p.tile_parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + few_bytes(plan, D));
    const int grid = std::min(p.items, d.num_sms);
    auto kernel = p.part_blocks > 0 ? &prompt_attention_kernel<D, BF16, true> : &prompt_attention_kernel<D, BF16, false>;
    // (beside the few-row kernel, which starts under this one and does not wait for what is in front of both, the ordinary launch)
    if (plan.few.n > 0) kernel<<<grid, PromptAttnCfg<D>::THREADS, PromptAttnCfg<D>::SMEM_BYTES, st>>>(tmQ, tmK, tmV, p, plan.tiled);
    else if ((e = launch_overlapping(kernel, dim3(grid), PromptAttnCfg<D>::THREADS, PromptAttnCfg<D>::SMEM_BYTES, st, tmQ, tmK, tmV, p, plan.tiled)) != cudaSuccess) return e;
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  if (plan.few.n > 0) {
    if (!half_map(d, &tmK, k, kv_width, std::max(kv_rows, 1), ld_k, kRowsTile) || !half_map(d, &tmV, v, kv_width, std::max(kv_rows, 1), ld_v, kRowsTile))
      return cudaErrorInvalidValue;
    p.chunk = plan.chunk;
    p.parts = static_cast<float*>(workspace);
    p.beside = plan.items > 0;
    if ((e = launch_overlapping(&prompt_rows_kernel<D, BF16>, dim3(static_cast<unsigned>(plan.ctas)), PromptRowsCfg<D>::THREADS, PromptRowsCfg<D>::SMEM_BYTES, st, tmK, tmV, p, plan.few)) != cudaSuccess)
      return e;
    if (plan.join &&
        (e = launch_overlapping(&prompt_join_kernel<D, BF16>, dim3(static_cast<unsigned>(plan.row_tiles), kRowsMax / kJoinRows), kJoinRows * 32, 0, st, p, plan.few)) != cudaSuccess)
      return e;
  }
  if (plan.part_blocks > 0)
    return launch_overlapping(&prompt_tile_join_kernel<D, BF16>, dim3(static_cast<unsigned>(plan.cut), 2 * D / 32), 256, 0, st, p, plan.tiled);
  return cudaSuccess;
}

// Checks what the plan did not look at and launches.  give(bytes, &workspace) is asked for memory where the plan needs some.
template <class Give>
dit_status attend(const dit_prompt_attention_args& a, const PromptPlan& plan, Give&& give, void* stream) {
  const int64_t width = static_cast<int64_t>(a.n_heads) * a.head_dim, kv_width = static_cast<int64_t>(a.n_kv_heads) * a.head_dim;
  auto matrix = [&](const void* p, int64_t ld, int64_t rows, int64_t cols) { return rows == 0 || (p && aligned(p, 16) && ld >= cols && ld % 8 == 0); };
  const int q_rows = plan.tiled.cu_q[a.n_requests], kv_rows = plan.tiled.cu_kv[a.n_requests];
  if (!matrix(a.q, a.ld_q, q_rows, width) || !matrix(a.out, a.ld_out, q_rows, width) || !matrix(a.k, a.ld_k, kv_rows, kv_width) ||
      !matrix(a.v, a.ld_v, kv_rows, kv_width))
    return DIT_ERR_INVALID_ARG;
  if (!(a.scale >= 0.f) || !(a.scale <= 2.0e38f)) return DIT_ERR_INVALID_ARG;        // scale * log2(e) has to be finite
  if (q_rows == 0) return DIT_OK;
  void* workspace = nullptr;
  dit_status s;
  if (const size_t need = part_bytes(plan, a.head_dim); need > 0 && (s = give(need, &workspace)) != DIT_OK) return s;
  OpsDevice d;
  s = ops_device(&d);
  if (s != DIT_OK) return s;
  if (prepare(d) != cudaSuccess) return DIT_ERR_CUDA;
  PromptAttnParams p{};
  p.out = a.out; p.ld_out = a.ld_out; p.q = static_cast<const uint16_t*>(a.q); p.v = static_cast<const uint16_t*>(a.v);
  p.ld_q = a.ld_q; p.ld_v = a.ld_v; p.n_heads = a.n_heads; p.kv_heads = a.n_kv_heads; p.group = a.n_heads / a.n_kv_heads;
  p.causal = a.causal != 0;
  p.scale_log2 = 1.4426950408889634f * (a.scale > 0.f ? a.scale : 1.0f / sqrtf(static_cast<float>(a.head_dim)));
  p.wide_out = aligned(a.out, 32) && a.ld_out % 16 == 0;
  p.status = d.status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (a.head_dim == 128) e = a.type == DIT_TYPE_BF16 ? launch_attention<128, true>(d, a, plan, p, workspace, st) : launch_attention<128, false>(d, a, plan, p, workspace, st);
  else e = a.type == DIT_TYPE_BF16 ? launch_attention<64, true>(d, a, plan, p, workspace, st) : launch_attention<64, false>(d, a, plan, p, workspace, st);
  return e == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

}  // namespace

// =============================================================================================== C ABI
extern "C" {

dit_status dit_rotary(const dit_rotary_args* a, void* stream) {
  if (!a || !type_ok(a->type) || a->rows < 0 || a->n_heads < 1) return DIT_ERR_INVALID_ARG;
  if (a->rows > kMaxSize || a->head_dim < 2 || a->head_dim > 4096 || a->rotary_dim < 2 || a->rotary_dim % 2 || a->rotary_dim > a->head_dim ||
      a->rotary_dim > 2 * kRotaryMaxPairs || static_cast<int64_t>(a->n_heads) * a->head_dim > (1 << 20))
    return DIT_ERR_SHAPE;
  if (!(a->base > 0.0) || !std::isfinite(a->base) || !(a->factor >= 1.0) || !std::isfinite(a->factor) || !(a->trained_len >= 0.0) ||
      !std::isfinite(a->trained_len) || !std::isfinite(a->magnitude))
    return DIT_ERR_INVALID_ARG;
  if (a->trained_len > 0.0 && (!std::isfinite(a->low) || !std::isfinite(a->high) || !(a->high > a->low))) return DIT_ERR_INVALID_ARG;
  RotaryParams p{};
  p.pairs = a->rotary_dim / 2;
  constexpr double kTurn = 6.283185307179586476925287;
  for (int i = 0; i < p.pairs; ++i) {
    double f = std::pow(a->base, -2.0 * i / a->rotary_dim);
    if (a->trained_len > 0.0) {
      const double keep = std::min(1.0, std::max(0.0, (a->trained_len * f / kTurn - a->low) / (a->high - a->low)));
      f *= keep + (1.0 - keep) / a->factor;
    } else {
      f /= a->factor;
    }
    p.turns[i] = f / kTurn;
    if (!std::isfinite(p.turns[i] * 2147483648.0)) return DIT_ERR_INVALID_ARG;       // (a base next to zero)
  }
  if (!a->positions) {
    if (a->n_requests < 0 || (a->n_requests > 0 && !a->lens)) return DIT_ERR_INVALID_ARG;
    if (a->n_requests > DIT_MAX_REQUESTS) return DIT_ERR_CAPACITY;
    int64_t rows = 0;
    for (int r = 0; r < a->n_requests; ++r) {
      const int64_t first = a->first ? a->first[r] : 0;
      if (a->lens[r] < 0 || first < 0) return DIT_ERR_INVALID_ARG;
      if (first + a->lens[r] > INT32_MAX) return DIT_ERR_SHAPE;
      p.cu[r] = static_cast<int>(rows); p.first[r] = static_cast<int>(first);
      rows += a->lens[r];
      if (rows > kMaxSize) return DIT_ERR_SHAPE;
    }
    p.cu[a->n_requests] = static_cast<int>(rows);
    p.n = a->n_requests;
    if (rows != a->rows) return DIT_ERR_INVALID_ARG;
  }
  if (a->rows == 0) return DIT_OK;
  const int64_t width = static_cast<int64_t>(a->n_heads) * a->head_dim;
  if (!a->x || !a->out || a->ld_x < width || a->ld_out < width || !aligned(a->x, type_bytes(a->type)) || !aligned(a->out, type_bytes(a->type)) ||
      !aligned(a->positions, 4) || (a->x == a->out && a->rows > 1 && a->ld_x != a->ld_out))
    return DIT_ERR_INVALID_ARG;
  OpsDevice d;
  const dit_status s = ops_device(&d);
  if (s != DIT_OK) return s;
  p.x = a->x; p.out = a->out; p.ld_x = a->ld_x; p.ld_out = a->ld_out; p.rows = a->rows; p.positions = a->positions;
  p.n_heads = a->n_heads; p.head_dim = a->head_dim; p.inverse = a->inverse != 0;
  p.magnitude = a->magnitude;
  // four rows per CTA once that leaves every SM one
  p.rows_per_cta = a->rows >= static_cast<int64_t>(kRotaryRows) * d.num_sms ? kRotaryRows : 1;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (a->type == DIT_TYPE_F16) e = launch_rotary<0>(p, *a, st);
  else if (a->type == DIT_TYPE_BF16) e = launch_rotary<1>(p, *a, st);
  else e = launch_rotary<2>(p, *a, st);
  return e == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

size_t dit_prompt_attention_workspace(const dit_prompt_attention_args* a) {
  PromptPlan plan;
  if (!a || plan_prompts(*a, &plan) != DIT_OK) return 0;
  return part_bytes(plan, a->head_dim);
}

dit_status dit_prompt_attention(const dit_prompt_attention_args* a, void* stream) {
  if (!a) return DIT_ERR_INVALID_ARG;
  PromptPlan plan;
  const dit_status s = plan_prompts(*a, &plan);
  if (s != DIT_OK) return s;
  return attend(*a, plan, [&](size_t need, void** workspace) {
    if (!a->workspace || !aligned(a->workspace, 16)) return DIT_ERR_INVALID_ARG;
    *workspace = a->workspace;
    return a->workspace_bytes < need ? DIT_ERR_CAPACITY : DIT_OK;
  }, stream);
}

}  // extern "C"

dit_status dit::prompt_attention_in(const dit_prompt_attention_args& a, void* (*room)(void*, size_t), void* context, void* stream) {
  PromptPlan plan;
  const dit_status s = plan_prompts(a, &plan);
  if (s != DIT_OK) return s;
  return attend(a, plan, [&](size_t need, void** workspace) {
    *workspace = room(context, need);
    return *workspace ? DIT_OK : DIT_ERR_CAPACITY;
  }, stream);
}
