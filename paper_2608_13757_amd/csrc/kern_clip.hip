// Global gradient norm over many tensors, and clipping:
//
//   norm = sqrt(sum of g^2 over all elements of all tensors)
//   out  = g * min(1, max_norm / (norm + 1e-6))
//
// Squares are summed in 64 bits (an fp32 or bf16 gradient's square passes
// fp32's range from 2^64 on, and the sum is as long as the model), each
// workgroup over its own chunks in their order, the workgroups' sums in the
// order of the workgroups: the same bits in every run.  A norm that is not
// finite leaves in-place gradients as they are and copies them (cast) to a
// separate output, so that the caller sees them next to the norm that says so.
//
// Two passes over the gradients, since the scale depends on all of them;
// bound by memory.  The second goes over the chunks in the opposite order, so
// that it begins with what the 256 MiB last-level cache still holds.  Pointers
// and sizes travel in the launch's arguments, kTensors per launch: no table
// to upload, nothing kept between calls.
#include <cmath>
#include <tuple>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kTensors = 128;
constexpr int kThreads = 256;
constexpr int64_t kChunk = 8192;                  // elements a workgroup takes at once
constexpr int kBlocks = 2048;                     // workgroups of all launches of a call
constexpr double kEps = 1e-6;

struct TensorList {
  const void *in[kTensors];
  void *out[kTensors];
  int64_t n[kTensors];
  int32_t first[kTensors];       // the tensor's first chunk
  uint8_t type[kTensors];        // bfs_dtype of in | of out << 4
  int32_t n_tensors, n_chunks;
};
static_assert(sizeof(TensorList) <= 4000, "launch arguments");

// The tensor that holds chunk c.
__device__ __forceinline__ int tensor_of(const TensorList &L, int c) {
  int lo = 0, hi = L.n_tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (L.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Sum of s over the workgroup, in a fixed order, in thread 0.
__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[kThreads / kWave];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_down(s, d);
  if (lane_index() == 0) part[wave_index()] = s;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) t += part[w];
  __syncthreads();
  return t;
}

template <typename T>
__device__ __forceinline__ double square_sum(const T *g, int64_t n) {
  double s = 0.0;
  const int64_t chunks = (n + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
  for (int64_t c = threadIdx.x; c < chunks; c += kThreads) {
    const auto v = load_chunk<T>(g, c, n);
#pragma unroll
    for (int i = 0; i < Chunk<T>::kElems; ++i) s += (double)(float)v[i] * (double)(float)v[i];
  }
  return s;
}

__global__ void __launch_bounds__(kThreads) square_kernel(TensorList L, double *partial) {
  const int from = (int)((int64_t)L.n_chunks * blockIdx.x / gridDim.x);
  const int to = (int)((int64_t)L.n_chunks * (blockIdx.x + 1) / gridDim.x);
  double s = 0.0;
  int i = tensor_of(L, from);
  for (int c = from; c < to; ++c) {
    while (i + 1 < L.n_tensors && L.first[i + 1] <= c) ++i;
    const int64_t at = (int64_t)(c - L.first[i]) * kChunk, left = L.n[i] - at, n = left < kChunk ? left : kChunk;
    switch (L.type[i] & 15) {
      case BFS_DTYPE_F32: s += square_sum(static_cast<const float *>(L.in[i]) + at, n); break;
      case BFS_DTYPE_BF16: s += square_sum(static_cast<const __bf16 *>(L.in[i]) + at, n); break;
      default: s += square_sum(static_cast<const _Float16 *>(L.in[i]) + at, n); break;
    }
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double total_of(const double *partial, int n) {
  double s = 0.0;
  for (int i = (int)threadIdx.x; i < n; i += kThreads) s += partial[i];
  return block_sum(s);
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double *partial, int n, float *norm) {
  const double s = total_of(partial, n);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <typename T, typename U>
__device__ __forceinline__ void scale_chunk(const T *g, U *out, int64_t n, float scale) {
  constexpr int E = Chunk<T>::kElems;
  typedef U vec __attribute__((ext_vector_type(E), aligned(sizeof(U))));
  const int64_t chunks = (n + E - 1) / E;
  for (int64_t c = threadIdx.x; c < chunks; c += kThreads) {
    const auto v = load_chunk<T>(g, c, n);
    vec o;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = (U)((float)v[i] * scale);
    if ((c + 1) * E <= n) {
      *reinterpret_cast<vec *>(out + c * E) = o;
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (c * E + i < n) out[c * E + i] = o[i];
    }
  }
}

__global__ void __launch_bounds__(kThreads) clip_kernel(TensorList L, const double *partial, int n_partial, double max_norm,
                                                        float *norm) {
  const double total = total_of(partial, n_partial), root = sqrt(total);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)root;
  const double ratio = max_norm / (root + kEps);
  const float scale = isfinite(root) && ratio < 1.0 ? (float)ratio : 1.0f;
  const int back = (int)(gridDim.x - 1 - blockIdx.x);
  const int from = (int)((int64_t)L.n_chunks * back / gridDim.x);
  const int to = (int)((int64_t)L.n_chunks * (back + 1) / gridDim.x);
  int i = tensor_of(L, to - 1);
  for (int c = to - 1; c >= from; --c) {
    while (L.first[i] > c) --i;
    if (scale == 1.0f && L.in[i] == L.out[i]) continue;
    const int64_t at = (int64_t)(c - L.first[i]) * kChunk, left = L.n[i] - at, n = left < kChunk ? left : kChunk;
    const void *in = L.in[i];
    void *out = L.out[i];
    switch (L.type[i]) {
      case BFS_DTYPE_F32: scale_chunk(static_cast<const float *>(in) + at, static_cast<float *>(out) + at, n, scale); break;
      case BFS_DTYPE_BF16: scale_chunk(static_cast<const __bf16 *>(in) + at, static_cast<float *>(out) + at, n, scale); break;
      case BFS_DTYPE_F16: scale_chunk(static_cast<const _Float16 *>(in) + at, static_cast<float *>(out) + at, n, scale); break;
      case BFS_DTYPE_BF16 | BFS_DTYPE_BF16 << 4:
        scale_chunk(static_cast<const __bf16 *>(in) + at, static_cast<__bf16 *>(out) + at, n, scale);
        break;
      default:
        scale_chunk(static_cast<const _Float16 *>(in) + at, static_cast<_Float16 *>(out) + at, n, scale);
        break;
    }
  }
}

int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

// f(list, workgroups, first partial sum) over the tensors that hold something,
// kTensors at a time; the workgroups go by a list's share of the chunks.
template <typename F>
bfs_status each_list(const void *const *in, void *const *out, const int64_t *numel, const int32_t *dtypes,
                     const int32_t *out_dtypes, int32_t n, int64_t all_chunks, int32_t *n_partial, F f) {
  TensorList L;
  int32_t at = 0, partial = 0;
  while (at < n) {
    L.n_tensors = 0;
    int64_t chunks = 0;
    for (; at < n && L.n_tensors < kTensors; ++at) {
      if (numel[at] == 0) continue;
      const int i = L.n_tensors++;
      L.in[i] = in[at];
      L.out[i] = out ? out[at] : nullptr;
      L.n[i] = numel[at];
      L.first[i] = (int32_t)chunks;
      L.type[i] = (uint8_t)(dtypes[at] | (out ? out_dtypes[at] << 4 : 0));
      chunks += chunks_of(numel[at]);
    }
    if (L.n_tensors == 0) break;
    L.n_chunks = (int32_t)chunks;
    int64_t blocks = (kBlocks * chunks + all_chunks - 1) / all_chunks;
    blocks = blocks < chunks ? blocks : chunks;
    bfs_status st = f(L, (int32_t)blocks, partial);
    if (st != BFS_OK) return st;
    partial += (int32_t)blocks;
  }
  *n_partial = partial;
  return BFS_OK;
}

bfs_status check_list(const char *what, const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n,
                      int64_t *all_chunks) {
  if (n < 0 || (n > 0 && (!grads || !numel || !dtypes))) return fail(BFS_E_INVALID, std::string(what) + ": bad tensor list");
  *all_chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (numel[i] < 0) return fail(BFS_E_INVALID, std::string(what) + ": negative tensor size");
    if (numel[i] > 0 && !grads[i]) return fail(BFS_E_INVALID, std::string(what) + ": null tensor");
    if (dtypes[i] < BFS_DTYPE_F32 || dtypes[i] > BFS_DTYPE_F16) return fail(BFS_E_INVALID, std::string(what) + ": unknown dtype");
    if (numel[i] >> 43 || (*all_chunks += chunks_of(numel[i])) > INT32_MAX)
      return fail(BFS_E_RESOURCE, std::string(what) + ": more than 2^43 elements");
  }
  return BFS_OK;
}

int64_t workspace_of(int32_t n_tensors) {
  return ((int64_t)kBlocks + (n_tensors + kTensors - 1) / kTensors + 1) * (int64_t)sizeof(double);
}

bfs_status check_workspace(const char *what, const void *workspace, int64_t bytes, int32_t n) {
  if (!workspace || bytes < workspace_of(n))
    return fail(BFS_E_INVALID, std::string(what) + ": workspace of " + std::to_string(workspace_of(n)) + " bytes needed");
  if ((uintptr_t)workspace % sizeof(double)) return fail(BFS_E_INVALID, std::string(what) + ": workspace not aligned to 8 bytes");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_grad_workspace(int32_t n_tensors, int64_t *bytes) {
  return entry([&]() -> bfs_status {
    if (n_tensors < 0 || !bytes) return fail(BFS_E_INVALID, "grad_workspace: bad argument");
    *bytes = workspace_of(n_tensors);
    return BFS_OK;
  });
}

bfs_status bfs_grad_norm(const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n_tensors,
                         float *norm, void *workspace, int64_t workspace_bytes, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    int64_t all = 0;
    bfs_status st = check_list("grad_norm", grads, numel, dtypes, n_tensors, &all);
    if (st == BFS_OK) st = check_workspace("grad_norm", workspace, workspace_bytes, n_tensors);
    if (st == BFS_OK && !norm) st = fail(BFS_E_INVALID, "grad_norm: null result");
    if (st != BFS_OK) return st;
    double *partial = static_cast<double *>(workspace);
    int32_t n = 0;
    st = each_list(grads, nullptr, numel, dtypes, nullptr, n_tensors, all, &n, [&](const TensorList &L, int32_t blocks, int32_t at) {
      return launch("grad_norm", square_kernel, blocks, kThreads, 0, stream, L, partial + at);
    });
    if (st != BFS_OK) return st;
    return launch("grad_norm", norm_kernel, 1, kThreads, 0, stream, partial, n, norm);
  });
}

bfs_status bfs_grad_clip(const void *const *grads, void *const *outs, const int64_t *numel, const int32_t *dtypes,
                         const int32_t *out_dtypes, int32_t n_tensors, double max_norm, float *norm, void *workspace,
                         int64_t workspace_bytes, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    int64_t all = 0;
    bfs_status st = check_list("grad_clip", grads, numel, dtypes, n_tensors, &all);
    if (st == BFS_OK) st = check_workspace("grad_clip", workspace, workspace_bytes, n_tensors);
    if (st != BFS_OK) return st;
    if (!(max_norm >= 0.0)) return fail(BFS_E_INVALID, "grad_clip: max_norm must not be negative");
    if (n_tensors > 0 && (!outs || !out_dtypes)) return fail(BFS_E_INVALID, "grad_clip: bad output list");
    for (int32_t i = 0; i < n_tensors; ++i) {
      if (numel[i] > 0 && !outs[i]) return fail(BFS_E_INVALID, "grad_clip: null output");
      if (out_dtypes[i] != BFS_DTYPE_F32 && out_dtypes[i] != dtypes[i])
        return fail(BFS_E_INVALID, "grad_clip: an output is fp32 or has its gradient's type");
    }
    double *partial = static_cast<double *>(workspace);
    int32_t n = 0, m = 0;
    st = each_list(grads, outs, numel, dtypes, out_dtypes, n_tensors, all, &n, [&](const TensorList &L, int32_t blocks, int32_t at) {
      return launch("grad_clip", square_kernel, blocks, kThreads, 0, stream, L, partial + at);
    });
    if (st != BFS_OK) return st;
    if (n == 0) return norm ? launch("grad_clip", norm_kernel, 1, kThreads, 0, stream, partial, 0, norm) : BFS_OK;
    float *first = norm;
    return each_list(grads, outs, numel, dtypes, out_dtypes, n_tensors, all, &m, [&](const TensorList &L, int32_t blocks, int32_t) {
      bfs_status s = launch("grad_clip", clip_kernel, blocks, kThreads, 0, stream, L, partial, n, max_norm, first);
      first = nullptr;
      return s;
    });
  });
}

}  // extern "C"
