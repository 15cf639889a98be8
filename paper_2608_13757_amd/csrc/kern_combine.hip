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
// Everything is one pass over the rows, bound by memory: 16 bytes per lane and
// access, up to 16 loads of a lane in flight (four slots, four steps of the
// row; the gradient two, with dy's).  In the combination a wave takes a token's
// row or a part of it (op_common.h: spans_of); in the gradient, whose dot
// products join the whole row, a workgroup takes a token where its four waves
// have two steps each, and with four rows and more one step, else a wave does
// (16000 tokens of 4096 bf16, two rows: 120 us with a workgroup and 125 with a
// wave for each, of 2048 57 and 53; seven rows of 2048: 183 and 191; of 2248,
// which begin anywhere in a line: 306 and 210), as it does for up to 512 tokens
// (64, eight rows of 2048: 4.1 and 6.3; 2400: 33 and 38, of 700: 17 and 14).
// 16384 tokens of eight rows of 2048 bf16, 605 MB: 100 us (6.0 TB/s; a large
// copy runs at 5.3), its gradient, 1.14 GB, 203 us (5.6).
#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kThreads = 256, kBlockWaves = kThreads / kWave;
constexpr int kMaxK = 64;
// Bytes of a row from which the gradient's rows that begin anywhere in a line
// are written by lines (32768 tokens, eight rows of 1409 bf16: 383 -> 332 us,
// two of 5003: 353 -> 316; 16000 tokens, four rows of 1201: 88 and 88, of 1001:
// 65 and 74, as the lines' ends are a larger part).
constexpr int64_t kLinesFrom = 2304;

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

// f(N, slots) for the slots whose bits are set, four at once, then two, one;
// in their order.
template <typename F>
__device__ __forceinline__ void each_slots(uint64_t set, F f) {
  auto take = [&](auto n) {
    constexpr int N = decltype(n)::value;
    int j[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      j[i] = __builtin_ctzll(set);
      set &= set - 1;
    }
    f(n, j);
  };
  while (__builtin_popcountll(set) >= 4) take(Int<4>{});
  if (__builtin_popcountll(set) >= 2) take(Int<2>{});
  if (set) take(Int<1>{});
}

// A wave takes a token, or one of `spans` interleaved parts of its row.
template <typename T, int kSteps, bool kStream>
__global__ void __launch_bounds__(kThreads) combine_kernel(CombineParams P) {
  constexpr int E = Chunk<T>::kElems;
  typedef typename Chunk<T>::vec vec;
  const int64_t u = (int64_t)blockIdx.x * kBlockWaves + wave_index();
  const int64_t t = u / P.spans;
  if (t >= P.n_tokens) return;
  const int lane = lane_index();
  const int64_t span = u - t * P.spans, chunks = P.width / E, step = (int64_t)P.spans * kWave;
  const T *rows = static_cast<const T *>(P.rows);
  T *y = static_cast<T *>(P.out) + t * P.out_stride;
  int slot;
  float weight;
  load_slot(P, t, lane, slot, weight);
  const uint64_t set = __ballot(slot >= 0);
  each_chunk<kSteps>(span * kWave + lane, chunks, step, [&](auto us, int64_t c) {
    constexpr int U = decltype(us)::value;
    float acc[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < E; ++i) acc[u][i] = 0.0f;
    each_slots(set, [&](auto ns, const int *j) {
      constexpr int N = decltype(ns)::value;
      vec v[N][U];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const T *row = rows + __builtin_amdgcn_readlane(slot, j[n]) * P.rows_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) v[n][u] = load<kStream>(row + (c + u * step) * E);
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float w = readlane(weight, j[n]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < E; ++i) acc[u][i] += w * (float)v[n][u][i];
      }
    });
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vec o;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] = (T)acc[u][i];
      store<kStream>(y + (c + u * step) * E, o);
    }
  });
  const int64_t i = chunks * E + lane;             // the elements behind the last whole chunk
  if (span == 0 && i < P.width) {
    float acc = 0.0f;
    each_slots(set, [&](auto ns, const int *j) {
      constexpr int N = decltype(ns)::value;
#pragma unroll
      for (int n = 0; n < N; ++n)
        acc += readlane(weight, j[n]) * (float)rows[__builtin_amdgcn_readlane(slot, j[n]) * P.rows_stride + i];
    });
    y[i] = (T)acc;
  }
}

// Slots j .. j + 3 of token t, for any lane: rows (-1 without one) and weights.
__device__ __forceinline__ void load_slots(const CombineParams &P, int64_t t, int j, int (&p)[4], float (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = -1;
    w[i] = 1.0f;
    if (j + i < P.k) {
      const int row = P.pos[t * P.k + j + i];
      p[i] = row >= 0 && row < P.n_rows ? row : -1;
      if (P.weights) w[i] = P.weights[t * P.k + j + i];
    }
  }
}

// Narrow rows: G lanes take a token, a chunk each.
template <typename T, int G>
__global__ void __launch_bounds__(kThreads) combine_narrow_kernel(CombineParams P) {
  constexpr int E = Chunk<T>::kElems;
  const int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / G;
  const int c = (int)threadIdx.x % G;
  if (t >= P.n_tokens || c * E >= P.width) return;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  for (int j = 0; j < P.k; j += 4) {
    int p[4];
    float w[4];
    typename Chunk<T>::vec v[4];
    load_slots(P, t, j, p, w);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p[i] >= 0) v[i] = load_chunk(static_cast<const T *>(P.rows) + p[i] * P.rows_stride, c, P.width);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p[i] < 0) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += w[i] * (float)v[i][e];
    }
  }
  typename Chunk<T>::vec o;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = (T)acc[e];
  store_chunk(static_cast<T *>(P.out) + t * P.out_stride, c, P.width, o);
}

template <typename T, int G>
__global__ void __launch_bounds__(kThreads) combine_grad_narrow_kernel(CombineParams P) {
  constexpr int E = Chunk<T>::kElems;
  typedef typename Chunk<T>::vec vec;
  const int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / G;
  const int c = (int)threadIdx.x % G;
  if (t >= P.n_tokens) return;
  const bool has = c * E < P.width;
  vec g;
  if (has) g = load_chunk(static_cast<const T *>(P.dy) + t * P.dy_stride, c, P.width);
  for (int j = 0; j < P.k; j += 4) {
    int p[4];
    float w[4];
    vec v[4];
    load_slots(P, t, j, p, w);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (has && p[i] >= 0) v[i] = load_chunk(static_cast<const T *>(P.rows) + p[i] * P.rows_stride, c, P.width);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (j + i >= P.k) break;
      float dot = 0.0f;
      if (has && p[i] >= 0) {
        vec o;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          dot += (float)g[e] * (float)v[i][e];
          o[e] = (T)(w[i] * (float)g[e]);
        }
        store_chunk(static_cast<T *>(P.out) + p[i] * P.out_stride, c, P.width, o);
      }
#pragma unroll
      for (int d = G / 2; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
      if (c == 0) P.grad_weights[t * P.k + j + i] = dot;
    }
  }
}

// <dy, rows[p_n]> over this lane's part of the rows, and rows of w_n * dy; for
// N slots.
template <typename T, int N, bool kStream>
__device__ __forceinline__ void grad_slots(const CombineParams &P, const T *dy, const int64_t *p, const float *w, int64_t at,
                                           int64_t step, float (&dot)[N]) {
  constexpr int E = Chunk<T>::kElems, kMost = N == 4 ? 2 : 4;
  typedef typename Chunk<T>::vec vec;
  const int64_t chunks = P.width / E;
  const T *rows = static_cast<const T *>(P.rows);
  T *out = static_cast<T *>(P.out);
#pragma unroll
  for (int n = 0; n < N; ++n) dot[n] = 0.0f;
  each_chunk<kMost>(at, chunks, step, [&](auto us, int64_t c) {
    constexpr int U = decltype(us)::value;
    vec g[U], v[N][U];
#pragma unroll
    for (int u = 0; u < U; ++u) g[u] = *reinterpret_cast<const vec *>(dy + (c + u * step) * E);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[n][u] = load<kStream>(rows + p[n] * P.rows_stride + (c + u * step) * E);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        vec o;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          dot[n] += (float)g[u][i] * (float)v[n][u][i];
          o[i] = (T)(w[n] * (float)g[u][i]);
        }
        store<kStream>(out + p[n] * P.out_stride + (c + u * step) * E, o);
      }
  });
  const int64_t i = chunks * E + at;
  if (at < E && i < P.width) {
    const float g = (float)dy[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      dot[n] += g * (float)rows[p[n] * P.rows_stride + i];
      out[p[n] * P.out_stride + i] = (T)(w[n] * g);
    }
  }
}

// The same where the gradient's rows begin anywhere in a line: its whole lines,
// and the elements before and behind them one by one.
template <typename T, int N>
__device__ __forceinline__ void grad_slots_lines(const CombineParams &P, const T *dy, const int64_t *p, const float *w, int64_t at,
                                                 int64_t step, float (&dot)[N]) {
  constexpr int E = Chunk<T>::kElems, kMost = N == 4 ? 2 : 4;
  typedef typename Chunk<T>::vec vec;
  const T *row[N];
  T *out[N];
  int64_t head[N], chunks[N], least = P.width;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    row[n] = static_cast<const T *>(P.rows) + p[n] * P.rows_stride;
    out[n] = static_cast<T *>(P.out) + p[n] * P.out_stride;
    head[n] = head_of(out[n], P.width);
    chunks[n] = (P.width - head[n]) * (int64_t)sizeof(T) / kLine * (kLine / 16);
    least = chunks[n] < least ? chunks[n] : least;
    dot[n] = 0.0f;
  }
  auto take = [&](int n, int64_t i, vec g, vec v) {
    vec o;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dot[n] += (float)g[e] * (float)v[e];
      o[e] = (T)(w[n] * (float)g[e]);
    }
    store<true>(out[n] + i, o);
  };
  each_chunk<kMost>(at, least, step, [&](auto us, int64_t c) {
    constexpr int U = decltype(us)::value;
    vec g[N][U], v[N][U];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = head[n] + (c + u * step) * E;
        g[n][u] = *reinterpret_cast<const vec *>(dy + i);
        v[n][u] = load<true>(row[n] + i);
      }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u) take(n, head[n] + (c + u * step) * E, g[n][u], v[n][u]);
  });
#pragma unroll
  for (int n = 0; n < N; ++n) {
    // one line's difference between the rows, then the ends
    const int64_t c = least + at;
    if (c < chunks[n]) {
      const int64_t i = head[n] + c * E;
      take(n, i, *reinterpret_cast<const vec *>(dy + i), load<true>(row[n] + i));
    }
    auto one = [&](int64_t i) {
      const float g = (float)dy[i];
      dot[n] += g * (float)row[n][i];
      out[n][i] = (T)(w[n] * g);
    };
    if (at < head[n]) one(at);
    const int64_t i = head[n] + chunks[n] * E + at;
    if (at < kWave && i < P.width) one(i);
  }
}

// W waves take a token: all of a workgroup, or one.
template <typename T, int W, bool kStream, bool kLines>
__global__ void __launch_bounds__(W > 1 ? W * kWave : kThreads) combine_grad_kernel(CombineParams P) {
  __shared__ float part[W][kMaxK];
  const int64_t t = W > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kBlockWaves + wave_index();
  if (t >= P.n_tokens) return;
  const int lane = lane_index(), wave = wave_index() % W;
  int slot;
  float weight, grad = 0.0f;                       // lane j: of slot j
  load_slot(P, t, lane, slot, weight);
  each_slots(__ballot(slot >= 0), [&](auto ns, const int *j) {
    constexpr int N = decltype(ns)::value;
    int64_t p[N];
    float w[N], dot[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      p[n] = __builtin_amdgcn_readlane(slot, j[n]);
      w[n] = readlane(weight, j[n]);
    }
    const T *dy = static_cast<const T *>(P.dy) + t * P.dy_stride;
    if (kLines) grad_slots_lines<T, N>(P, dy, p, w, wave * kWave + lane, W * kWave, dot);
    else grad_slots<T, N, kStream>(P, dy, p, w, wave * kWave + lane, W * kWave, dot);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float d = group_sum<64>(dot[n]);
      if (lane == j[n]) grad = d;
    }
  });
  if (W > 1) {                                     // the workgroup's only token
    part[wave][lane] = grad;
    __syncthreads();
    if (wave != 0) return;
    grad = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) grad += part[i][lane];
  }
  if (lane < P.k) P.grad_weights[t * P.k + lane] = grad;
}

bfs_status check_rows(const char *what, int64_t n_rows, int64_t width, int64_t n_tokens, int32_t k) {
  if (n_rows < 0 || width < 0 || n_tokens < 0 || k < 1)
    return fail(BFS_E_INVALID, std::string(what) + ": a negative or zero size");
  if (k > kMaxK || n_tokens > kMaxTokens || n_rows >= (int64_t)1 << 31 || width > kMaxWidth)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 64 experts per token, 2^24 - 1 tokens, 2^31 - 1 rows and 2^28 columns");
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
      const int64_t most = (chunks + kWave - 1) / kWave;
      if (narrow_rows(chunks, n_tokens, k))
        return with_group(chunks, [&](auto g) {
          constexpr int G = decltype(g)::value;
          return launch("moe_combine", combine_narrow_kernel<T, G>, (n_tokens + kThreads / G - 1) / (kThreads / G), kThreads, 0,
                        stream, P);
        });
      P.spans = (int32_t)spans_of(most, n_tokens);
      // chunks of a lane at once: four where a wave's part of the row has them
      auto kernel = most >= 4 * P.spans ? combine_kernel<T, 4, false> : combine_kernel<T, 2, false>;
      if ((k + 1) * n_tokens * width * (int64_t)sizeof(T) >= kStreamFrom)
        kernel = most >= 4 * P.spans ? combine_kernel<T, 4, true> : combine_kernel<T, 2, true>;
      return launch("moe_combine", kernel, (n_tokens * P.spans + kBlockWaves - 1) / kBlockWaves, kThreads, 0,
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
      const int64_t chunks = (width + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
      if (narrow_rows(chunks, n_tokens, k))
        return with_group(chunks, [&](auto g) {
          constexpr int G = decltype(g)::value;
          return launch("moe_combine_grad", combine_grad_narrow_kernel<T, G>, (n_tokens + kThreads / G - 1) / (kThreads / G),
                        kThreads, 0, stream, P);
        });
      const bool stream_rows = (2 * k + 1) * n_tokens * width * (int64_t)sizeof(T) >= kStreamFrom;
      const bool lines = stream_rows && width * (int64_t)sizeof(T) >= kLinesFrom &&
                         ((uintptr_t)grad_rows % kLine || grad_rows_stride * sizeof(T) % kLine);
      auto run = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        return launch("moe_combine_grad", !stream_rows ? combine_grad_kernel<T, W, false, false>
                                          : lines ? combine_grad_kernel<T, W, true, true> : combine_grad_kernel<T, W, true, false>,
                      W > 1 ? n_tokens : (n_tokens + kBlockWaves - 1) / kBlockWaves, W > 1 ? W * kWave : kThreads, 0, stream, P);
      };
      const int64_t whole = width / Chunk<T>::kElems;
      const bool workgroup = whole >= 2 * kThreads || (whole >= kThreads && k >= 4 && !lines) || (whole >= kWave && n_tokens <= 512);
      return workgroup ? run(Int<kBlockWaves>{}) : run(Int<1>{});
    });
  });
}

}  // extern "C"
