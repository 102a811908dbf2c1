// Rotary positions of include/dit_ops.h: argument checks and launches.
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "ops_launch.h"
#include "rotary.cuh"

using namespace dit;

namespace {

constexpr int64_t kMaxSize = INT32_MAX - 1024;

int type_bytes(dit_type t) { return t == DIT_TYPE_F32 ? 4 : 2; }
bool type_ok(dit_type t) { return t == DIT_TYPE_F16 || t == DIT_TYPE_BF16 || t == DIT_TYPE_F32; }
bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

template <int kType>
cudaError_t launch_rotary(const RotaryParams& p, bool vec, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>((p.rows + p.rows_per_cta - 1) / p.rows_per_cta);
  if (vec) rotary_kernel<kType, true><<<grid, kRotaryThreads, 0, st>>>(p);
  else rotary_kernel<kType, false><<<grid, kRotaryThreads, 0, st>>>(p);
  return cudaGetLastError();
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
  p.n_heads = a->n_heads; p.head_dim = a->head_dim; p.pairs = a->rotary_dim / 2; p.interleaved = a->interleaved != 0; p.inverse = a->inverse != 0;
  p.magnitude = a->magnitude;
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
  }
  // four rows per CTA once that leaves every SM a few CTAs
  p.rows_per_cta = a->rows >= 8ll * kRotaryRows * d.num_sms ? kRotaryRows : 1;
  const int per = 16 / type_bytes(a->type);
  const bool vec = aligned(a->x, 16) && aligned(a->out, 16) && a->ld_x % per == 0 && a->ld_out % per == 0 && a->head_dim % per == 0 &&
                   (p.interleaved ? a->rotary_dim : p.pairs) % per == 0 && a->rotary_dim % per == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (a->type == DIT_TYPE_F16) e = launch_rotary<0>(p, vec, st);
  else if (a->type == DIT_TYPE_BF16) e = launch_rotary<1>(p, vec, st);
  else e = launch_rotary<2>(p, vec, st);
  return e == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

}  // extern "C"
