// The experts' rows back to their tokens, with the router's weights:
//
//   y[t] = sum over j of w[t][j] * rows[pos[t][j]]      (slots with a row)
//
// summed in fp32 in the order of j and rounded once; without weights (w = 1)
// it is the gradient of the dispatch.  And its gradient:
//
//   grad_rows[pos[t][j]] = w[t][j] * dy[t]
//   grad_w[t][j]         = <dy[t], rows[pos[t][j]]>     (0 without a row)
//
// pos comes from the dispatch: different slots have different rows, so the
// gradient's rows are written once each, without atomics.  Positions outside
// 0 .. n_rows - 1 count as slots without a row.
//
// Everything is one pass over the rows, bound by memory: a wave takes a token
// (or, for few tokens, a span of its row), 16 bytes per lane and access, with
// the loads of up to four slots in flight together.
#include <tuple>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kThreads = 256, kBlockWaves = kThreads / kWave;
constexpr int kMaxK = 64;

struct CombineParams {
  const void *rows, *dy;
  const int32_t *pos;
  const float *weights;
  void *out;                     // y, or grad_rows
  float *grad_weights;
  int64_t n_tokens, n_rows, width, rows_stride, dy_stride, out_stride;
  int32_t k, spans;
};

// Lane j's slot of token t: its row (-1 without one) and weight.
__device__ __forceinline__ void load_slot(const CombineParams &P, int64_t t, int lane, int &row, float &w) {
  row = -1;
  w = 1.0f;
  if (lane < P.k) {
    const int p = P.pos[t * P.k + lane];
    row = p >= 0 && p < P.n_rows ? p : -1;
    if (P.weights) w = P.weights[t * P.k + lane];
  }
}

__device__ __forceinline__ float readlane(float x, int j) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), j));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) combine_kernel(CombineParams P) {
  constexpr int E = Chunk<T>::kElems;
  const int64_t u = (int64_t)blockIdx.x * kBlockWaves + wave_index();
  const int64_t t = u / P.spans;
  if (t >= P.n_tokens) return;
  const int64_t chunks = (P.width + E - 1) / E, step = (int64_t)P.spans * kWave;
  const T *rows = static_cast<const T *>(P.rows);
  T *y = static_cast<T *>(P.out) + t * P.out_stride;
  int slot;
  float weight;
  load_slot(P, t, lane_index(), slot, weight);
  for (int64_t c = (u - t * P.spans) * kWave + lane_index(); c < chunks; c += step) {
    float acc[E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.0f;
    for (int j = 0; j < P.k; ++j) {
      const int64_t p = __builtin_amdgcn_readlane(slot, j);
      if (p < 0) continue;
      const float w = readlane(weight, j);
      const auto v = load_chunk<T>(rows + p * P.rows_stride, c, P.width);
#pragma unroll
      for (int i = 0; i < E; ++i) acc[i] += w * (float)v[i];
    }
    typename Chunk<T>::vec o;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = (T)acc[i];
    store_chunk<T>(y, c, P.width, o);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) combine_grad_kernel(CombineParams P) {
  constexpr int E = Chunk<T>::kElems;
  const int64_t t = (int64_t)blockIdx.x * kBlockWaves + wave_index();
  if (t >= P.n_tokens) return;
  const int lane = lane_index();
  const int64_t chunks = (P.width + E - 1) / E;
  const T *rows = static_cast<const T *>(P.rows), *dy = static_cast<const T *>(P.dy) + t * P.dy_stride;
  T *out = static_cast<T *>(P.out);
  int slot;
  float weight;
  load_slot(P, t, lane, slot, weight);
  for (int j = 0; j < P.k; ++j) {
    const int64_t p = __builtin_amdgcn_readlane(slot, j);
    float dot = 0.0f;
    if (p >= 0) {
      const float w = readlane(weight, j);
      for (int64_t c = lane; c < chunks; c += kWave) {
        const auto g = load_chunk<T>(dy, c, P.width);
        const auto v = load_chunk<T>(rows + p * P.rows_stride, c, P.width);
        typename Chunk<T>::vec o;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          dot += (float)g[i] * (float)v[i];
          o[i] = (T)(w * (float)g[i]);
        }
        store_chunk<T>(out + p * P.out_stride, c, P.width, o);
      }
    }
    dot = group_sum<64>(dot);
    if (lane == 0) P.grad_weights[t * P.k + j] = dot;
  }
}

bfs_status check_rows(const char *what, int64_t n_rows, int64_t width, int64_t n_tokens, int32_t k) {
  if (n_rows < 0 || width < 0 || n_tokens < 0 || k < 1)
    return fail(BFS_E_INVALID, std::string(what) + ": a negative or zero size");
  if (k > kMaxK || n_tokens > ((int64_t)1 << 31) / k - 1 || n_rows >= (int64_t)1 << 31)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 64 experts per token and 2^31 - 1 slots and rows");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_moe_combine(const void *rows, int32_t dtype, int64_t n_rows, int64_t width, int64_t rows_stride,
                           const int32_t *pos, const float *weights, int64_t n_tokens, int32_t k, void *y,
                           int64_t y_stride, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_rows("moe_combine", n_rows, width, n_tokens, k);
    if (st != BFS_OK) return st;
    if (rows_stride < 0 || y_stride < width)
      return fail(BFS_E_INVALID, "moe_combine: negative stride, or rows of y that overlap");
    return with_type(dtype, [&](auto t) -> bfs_status {
      using T = decltype(t);
      if (n_tokens == 0 || width == 0) return BFS_OK;
      if (!pos || !y || (n_rows > 0 && !rows)) return fail(BFS_E_INVALID, "moe_combine: null buffer");
      CombineParams P{};
      P.rows = rows;
      P.pos = pos;
      P.weights = weights;
      P.out = y;
      P.n_tokens = n_tokens;
      P.n_rows = n_rows;
      P.width = width;
      P.rows_stride = rows_stride;
      P.out_stride = y_stride;
      P.k = k;
      const int64_t chunks = (width + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
      const int64_t most = (chunks + kWave - 1) / kWave, wanted = (4096 + n_tokens - 1) / n_tokens;
      P.spans = (int32_t)(most < wanted ? most : wanted);
      return launch("moe_combine", combine_kernel<T>, (n_tokens * P.spans + kBlockWaves - 1) / kBlockWaves, kThreads, 0,
                    stream, P);
    });
  });
}

bfs_status bfs_moe_combine_grad(const void *grad_y, int32_t dtype, int64_t n_tokens, int64_t width, int64_t grad_y_stride,
                                const void *rows, int64_t n_rows, int64_t rows_stride, const int32_t *pos,
                                const float *weights, int32_t k, void *grad_rows, int64_t grad_rows_stride,
                                float *grad_weights, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_rows("moe_combine_grad", n_rows, width, n_tokens, k);
    if (st != BFS_OK) return st;
    if (rows_stride < 0 || grad_y_stride < 0 || grad_rows_stride < width)
      return fail(BFS_E_INVALID, "moe_combine_grad: negative stride, or rows of the gradient that overlap");
    return with_type(dtype, [&](auto t) -> bfs_status {
      using T = decltype(t);
      if (n_tokens == 0) return BFS_OK;
      if (!pos || !weights || !grad_weights || (width > 0 && !grad_y) || (width > 0 && n_rows > 0 && (!rows || !grad_rows)))
        return fail(BFS_E_INVALID, "moe_combine_grad: null buffer");
      CombineParams P{};
      P.rows = rows;
      P.dy = grad_y;
      P.pos = pos;
      P.weights = weights;
      P.out = grad_rows;
      P.grad_weights = grad_weights;
      P.n_tokens = n_tokens;
      P.n_rows = n_rows;
      P.width = width;
      P.rows_stride = rows_stride;
      P.dy_stride = grad_y_stride;
      P.out_stride = grad_rows_stride;
      P.k = k;
      return launch("moe_combine_grad", combine_grad_kernel<T>, (n_tokens + kBlockWaves - 1) / kBlockWaves, kThreads, 0,
                    stream, P);
    });
  });
}

}  // extern "C"
