// Global gradient norm over many tensors, and clipping:
//
//   norm = sqrt(sum of g^2 over all elements of all tensors)
//   out  = g * min(1, max_norm / (norm + 1e-6))
//
// Squares are summed in 64 bits (an fp32 or bf16 gradient's square passes
// fp32's range from 2^64 on, and the sum is as long as the model), each
// workgroup over its own chunks in their order, the workgroups' sums in the
// order of the workgroups: the same bits in every run.  A norm that is not
// finite in fp32, as it is reported, leaves in-place gradients as they are and
// copies them (cast) to a separate output, so that the caller sees them next to
// the norm that says so: an infinite norm always has unscaled gradients beside it,
// whether the 64-bit sum held it or not.
//
// Two passes over the gradients, since the scale depends on all of them;
// bound by memory.  The second goes over the chunks in the opposite order, so
// that it begins with what the 256 MiB last-level cache still holds.  The
// tensors' table is made on the host and laid into device memory by the
// caller, once for a set of tensors: one launch for each pass whatever their
// number (as launch arguments, 128 tensors a launch, 2^28 bf16 gradients in 290
// tensors took six launches and 510 us).
//
// 2^28 bf16 gradients in 290 tensors into fp32: 370 us, 5.8 TB/s over both
// passes (a large copy's rate is 5.3; 408 us on another device, on which the
// comparisons of chunks, workgroups, orders and stores below were made); 2^20 fp32
// in 24: 7.4 us, two short launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kThreads = 256;
// Elements a workgroup takes at once, less where the tensors would leave
// workgroups idle (2^28 bf16 in 290 tensors: 408 us with 8192, 422 with 16384,
// whose last chunks are less even over the workgroups).
constexpr int64_t kMaxChunk = 8192, kMinChunk = 2048;
// Workgroups: 1024, from four chunks for each of 4096 on these (clipping bf16,
// 2^28: 413 us with 1024, 408 with 4096; fp32 596 and 586; 2^26 bf16, which would
// have two for each: 91 and 97).
// Numbers between leave a part of the device idle at the end (2^25 with 1030
// of them 51 us, with 1024 48).
constexpr int kBlocks = 1024, kMostBlocks = 4096, kChunksEach = 4;
// Gradients' bytes from which the norm alone reads past the caches: they do not
// fit the last-level one anyway (2^28 fp32: 188 us with plain loads, 165 with
// these; 2^27 bf16 of one set again and again 51 and 55, 2^26 27 and 29.5, which of
// three sets in turn are 30 and 28).  A clipping's first pass leaves there what it
// can for the second.
constexpr int64_t kStreamNorm = 256 << 20;
// LDS that a workgroup of either pass takes, though it needs little of it, so
// that four are resident on a compute unit (160 KB): with seven and eight, as the
// registers allow, memory serves more places at once and is slower (2^28 bf16 into
// fp32: 380 us, so 371, the norm alone 89.6 and 86.1; 2^27 fp16 184 and 181; 2^20
// fp32 7.5 and 7.4).
constexpr size_t kHeldLds = 39 << 10;
constexpr int64_t kMaxElements = (int64_t)1 << 43;
constexpr double kEps = 1e-6;

// A tensor of the table: its chunks are first .. first + chunks - 1 of all.
struct Entry {
  const void *in;
  void *out;
  int64_t n;
  int32_t first, chunks;
  int32_t type;                  // bfs_dtype of in | of out << 4
  int32_t index;                 // in the table
};

// The table in device memory: the entries, then for each workgroup a copy of
// the entry that holds its first chunk (one access instead of two in a row).
struct Table {
  const Entry *entry;
  const Entry *start;
  int64_t chunk;
  int32_t n_chunks;
};

// Workgroup b of n runs chunks from .. to - 1.
__device__ __forceinline__ int first_chunk(const Table &t, int b) { return (int)((int64_t)t.n_chunks * b / gridDim.x); }

// The workgroup whose chunks this one scales: eight at a time in the opposite
// order, where more run than are resident, and on the same of the eight XCDs
// (workgroups go to them in turn), whose L2 still holds them after the first
// pass.  2^23 bf16: 19.1 us in the plain opposite order, 17.3 so, 17.0 in the first
// pass's own order; 2^25 fp32 76.6, 72.4 and 77.5; 2^28 fp32 586, 586 and 603.
__device__ __forceinline__ int opposite() {
  const uint32_t n = gridDim.x, b = blockIdx.x;
  return (int)(n % 8 ? b : (n - 8 - (b & ~7u)) | (b & 7u));
}

// Sum of s over the workgroup, in a fixed order, for every thread.
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

// f on this lane's vectors, of which at most 2 U - 1 are left: U of them with
// all accesses issued before the first is used, then U / 2, ...
template <int U, bool kStream, typename Vec, int V, typename T, typename F>
__device__ __forceinline__ void each_vector(const T *g, int64_t at, int64_t end, F f) {
  constexpr int kStep = kThreads * V;
  if (at + (U - 1) * kStep < end) {
    Vec v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      auto p = reinterpret_cast<const Vec *>(g + at + u * kStep);
      v[u] = kStream ? __builtin_nontemporal_load(p) : *p;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) f(at + u * kStep, v[u]);
    at += U * kStep;
  }
  if constexpr (U > 1) each_vector<U / 2, kStream, Vec, V>(g, at, end, f);
}

// Chunk c of a tensor of n elements at g, `chunks` of them in all, whose first
// whole line (of g itself or of the output) begins at element head:
// chunks begin with a line, the first one at element 0, the last one takes
// what is left.  f(first element, vector) for this lane's vectors, those of a
// whole chunk in flight at once (eight accesses where a vector has four elements,
// four where it has eight), one(element) for the elements that no vector holds.
template <bool kStream, typename Vec, int V, typename T, typename F, typename One>
__device__ __forceinline__ void each_element(const T *g, int64_t n, int head, int64_t chunk, int c, int chunks, F f, One one) {
  const int64_t from = head + c * chunk, to = c + 1 == chunks || from + chunk > n ? n : from + chunk;
  if (c == 0 && (int)threadIdx.x < head) one((int64_t)threadIdx.x);
  if (from >= to) return;
  const int64_t end = to - (to - from) % V;
  constexpr int kMost = (int)(kMaxChunk / (kThreads * V));        // vectors of a lane in a chunk, at most
  static_assert(kMost * kThreads * V == kMaxChunk && (kMost & (kMost - 1)) == 0, "a chunk's vectors, by halves");
  each_vector<kMost, kStream, Vec, V>(g, from + (int64_t)threadIdx.x * V, end, f);
  if (end + threadIdx.x < to) one(end + threadIdx.x);
}

template <bool kStream, typename T>
__device__ __forceinline__ double square_sum(const Entry &e, int64_t chunk, int c) {
  constexpr int V = Chunk<T>::kElems;
  typedef typename Chunk<T>::vec vec;
  const T *g = static_cast<const T *>(e.in);
  double s = 0.0;
  each_element<kStream, vec, V>(
      g, e.n, head_of(g, e.n), chunk, c, e.chunks,
      [&](int64_t, vec v) {
#pragma unroll
        for (int i = 0; i < V; ++i) s += (double)(float)v[i] * (double)(float)v[i];
      },
      [&](int64_t i) { s += (double)(float)g[i] * (double)(float)g[i]; });
  return s;
}

template <bool kStream>
__global__ void __launch_bounds__(kThreads) square_kernel(Table t, double *partial) {
  const int from = first_chunk(t, (int)blockIdx.x), to = first_chunk(t, (int)blockIdx.x + 1);
  double s = 0.0;
  Entry e = t.start[blockIdx.x];
  for (int c = from; c < to; ++c) {
    if (e.first + e.chunks <= c) e = t.entry[e.index + 1];
    switch (e.type & 15) {
      case BFS_DTYPE_F32: s += square_sum<kStream, float>(e, t.chunk, c - e.first); break;
      case BFS_DTYPE_BF16: s += square_sum<kStream, __bf16>(e, t.chunk, c - e.first); break;
      default: s += square_sum<kStream, _Float16>(e, t.chunk, c - e.first); break;
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

struct Scale {
  float first, then;             // g * first is exact wherever the result is not 0
};

// Below 2^-100 a factor of 2^-63 is taken out first: the rest stays a normal
// number (huge gradients and a small max_norm), and what that factor makes
// subnormal would round to 0 in the end.
__device__ __forceinline__ Scale scale_of(double ratio) {
  return ratio < 0x1p-100 ? Scale{0x1p-63f, (float)(ratio * 0x1p63)} : Scale{1.0f, (float)ratio};
}

// A lane's access is 16 bytes of the output, where the chunks begin with a
// line: into a flat vector, in which tensors begin anywhere, whole lines are
// written.  Nontemporal stores leave the last-level cache to the gradients that
// the pass is still to read (2^25 fp32, both passes: 95 us with plain stores, 72
// with these; 2^23: 22.4 and 21.1; 2^28 bf16 into fp32: 570 and 408).
template <typename T, typename U>
__device__ __forceinline__ void scale_chunk(const Entry &e, int64_t chunk, int c, Scale s) {
  constexpr int V = Chunk<U>::kElems;
  typedef T in_vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  typedef typename Chunk<U>::vec vec;
  const T *g = static_cast<const T *>(e.in);
  U *out = static_cast<U *>(e.out);
  each_element<false, in_vec, V>(
      g, e.n, head_of(out, e.n), chunk, c, e.chunks,
      [&](int64_t i, in_vec v) {
        vec o;
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = (U)((float)v[j] * s.first * s.then);
        __builtin_nontemporal_store(o, reinterpret_cast<vec *>(out + i));
      },
      [&](int64_t i) { out[i] = (U)((float)g[i] * s.first * s.then); });
}

__global__ void __launch_bounds__(kThreads) clip_kernel(Table t, const double *partial, double max_norm, float *norm) {
  const int back = opposite();
  Entry e = t.start[back];                         // on its way under the sums
  const double root = sqrt(total_of(partial, (int)gridDim.x));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)root;
  const double ratio = max_norm / (root + kEps);
  const bool clips = isfinite((float)root) && ratio < 1.0;
  const Scale scale = scale_of(clips ? ratio : 1.0);
  const int from = first_chunk(t, back), to = first_chunk(t, back + 1);
  while (e.first + e.chunks < to) e = t.entry[e.index + 1];
  for (int c = to - 1; c >= from; --c) {
    if (e.first > c) e = t.entry[e.index - 1];
    if (!clips && e.in == e.out) continue;
    switch (e.type) {
      case BFS_DTYPE_F32: scale_chunk<float, float>(e, t.chunk, c - e.first, scale); break;
      case BFS_DTYPE_BF16: scale_chunk<__bf16, float>(e, t.chunk, c - e.first, scale); break;
      case BFS_DTYPE_F16: scale_chunk<_Float16, float>(e, t.chunk, c - e.first, scale); break;
      case BFS_DTYPE_BF16 | BFS_DTYPE_BF16 << 4: scale_chunk<__bf16, __bf16>(e, t.chunk, c - e.first, scale); break;
      default: scale_chunk<_Float16, _Float16>(e, t.chunk, c - e.first, scale); break;
    }
  }
}

// Whether an output shares memory with another one, or with a gradient that is
// not its own (or its own, elsewhere): no order of the writes is right then.
bool overlaps(const void *const *grads, void *const *outs, const int64_t *numel, const int32_t *dtypes,
              const int32_t *out_dtypes, int32_t n) {
  struct Span {
    uintptr_t from, to;
    int32_t i;
  };
  auto span = [&](const void *p, int32_t i, int32_t dtype) {
    const uintptr_t from = (uintptr_t)p;
    return Span{from, from + (uintptr_t)numel[i] * (dtype == BFS_DTYPE_F32 ? 4 : 2), i};
  };
  std::vector<Span> out;
  for (int32_t i = 0; i < n; ++i)
    if (numel[i] > 0) out.push_back(span(outs[i], i, out_dtypes[i]));
  std::sort(out.begin(), out.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
  for (size_t i = 1; i < out.size(); ++i)
    if (out[i].from < out[i - 1].to) return true;
  for (int32_t i = 0; i < n; ++i) {
    if (numel[i] == 0) continue;
    const Span g = span(grads[i], i, dtypes[i]);
    // the outputs are apart, so ends ascend too: from the first that ends behind g's start
    auto o = std::upper_bound(out.begin(), out.end(), g.from, [](uintptr_t a, const Span &b) { return a < b.to; });
    for (; o != out.end() && o->from < g.to; ++o)
      if (o->i != i || o->from != g.from) return true;
  }
  return false;
}

int64_t chunks_of(int64_t n, int64_t chunk) { return (n + chunk - 1) / chunk; }

Table table_of(const bfs_grad_set &set, const void *image) {
  Table t;
  t.entry = static_cast<const Entry *>(image);
  t.start = t.entry + set.n_entries;
  t.chunk = set.chunk;
  t.n_chunks = set.n_chunks;
  return t;
}

bfs_status check_call(const char *what, const bfs_grad_set *set, const void *image, const void *workspace, int64_t bytes) {
  if (!set) return fail(BFS_E_INVALID, std::string(what) + ": null set");
  if (set->n_entries < 0 || set->n_chunks < set->n_entries || set->n_blocks < 0 || set->n_blocks > kMostBlocks ||
      (set->n_chunks > 0 && set->n_blocks < 1) || set->chunk < kMinChunk || set->chunk > kMaxChunk)
    return fail(BFS_E_INVALID, std::string(what) + ": not a set that bfs_grad_table made");
  if (set->n_chunks > 0 && (!image || (uintptr_t)image % 16)) return fail(BFS_E_INVALID, std::string(what) + ": bad table address");
  if (!workspace || bytes < set->workspace_bytes || bytes < set->n_blocks * (int64_t)sizeof(double))
    return fail(BFS_E_INVALID, std::string(what) + ": workspace of " + std::to_string(set->workspace_bytes) + " bytes needed");
  if ((uintptr_t)workspace % sizeof(double)) return fail(BFS_E_INVALID, std::string(what) + ": workspace not aligned to 8 bytes");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_grad_table(const void *const *grads, void *const *outs, const int64_t *numel, const int32_t *dtypes,
                          const int32_t *out_dtypes, int32_t n_tensors, bfs_grad_set *set, void *image, int64_t image_bytes) {
  return entry([&]() -> bfs_status {
    if (n_tensors < 0 || !set || (n_tensors > 0 && (!grads || !outs || !numel || !dtypes || !out_dtypes)))
      return fail(BFS_E_INVALID, "grad_table: bad tensor list");
    int64_t elements = 0, bytes = 0;
    int32_t held = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
      if (numel[i] < 0) return fail(BFS_E_INVALID, "grad_table: negative tensor size");
      if (numel[i] > 0 && (!grads[i] || !outs[i])) return fail(BFS_E_INVALID, "grad_table: null tensor");
      if (dtypes[i] < BFS_DTYPE_F32 || dtypes[i] > BFS_DTYPE_F16) return fail(BFS_E_INVALID, "grad_table: unknown dtype");
      if (out_dtypes[i] != BFS_DTYPE_F32 && out_dtypes[i] != dtypes[i])
        return fail(BFS_E_INVALID, "grad_table: an output is fp32 or has its gradient's type");
      if (numel[i] > 0 && grads[i] == outs[i] && out_dtypes[i] != dtypes[i])
        return fail(BFS_E_INVALID, "grad_table: in place needs the gradient's type");
      if ((uintptr_t)grads[i] % (dtypes[i] == BFS_DTYPE_F32 ? 4 : 2) || (uintptr_t)outs[i] % (out_dtypes[i] == BFS_DTYPE_F32 ? 4 : 2))
        return fail(BFS_E_INVALID, "grad_table: a tensor is not aligned to its elements");
      if (numel[i] > kMaxElements || (elements += numel[i]) > kMaxElements)
        return fail(BFS_E_RESOURCE, "grad_table: more than 2^43 elements");
      bytes += numel[i] * (dtypes[i] == BFS_DTYPE_F32 ? 4 : 2);
      held += numel[i] > 0;
    }
    bfs_grad_set s{};
    s.chunk = kMaxChunk;
    while (s.chunk > kMinChunk && elements < s.chunk * kBlocks) s.chunk /= 2;
    int64_t chunks = 0;
    for (int32_t i = 0; i < n_tensors; ++i) chunks += chunks_of(numel[i], s.chunk);
    if (chunks > INT32_MAX) return fail(BFS_E_RESOURCE, "grad_table: more than 2^31 - 1 chunks");
    s.grad_bytes = bytes;
    s.n_entries = held;
    s.n_chunks = (int32_t)chunks;
    s.n_blocks = chunks >= kMostBlocks * (int64_t)kChunksEach ? kMostBlocks : chunks < kBlocks ? (int32_t)chunks : kBlocks;
    s.workspace_bytes = (s.n_blocks > 0 ? s.n_blocks : 1) * (int64_t)sizeof(double);
    s.overlap = overlaps(grads, outs, numel, dtypes, out_dtypes, n_tensors);
    s.image_bytes = ((int64_t)held + s.n_blocks) * (int64_t)sizeof(Entry);
    if (image) {
      if (image_bytes < s.image_bytes) return fail(BFS_E_INVALID, "grad_table: image of " + std::to_string(s.image_bytes) + " bytes needed");
      unsigned char *p = static_cast<unsigned char *>(image);
      int64_t first = 0;
      int32_t b = 0, k = 0;
      for (int32_t i = 0; i < n_tensors; ++i) {
        if (numel[i] == 0) continue;
        Entry e{};
        e.in = grads[i];
        e.out = outs[i];
        e.n = numel[i];
        e.first = (int32_t)first;
        e.chunks = (int32_t)chunks_of(numel[i], s.chunk);
        e.type = dtypes[i] | out_dtypes[i] << 4;
        e.index = k;
        first += e.chunks;
        std::memcpy(p + k++ * sizeof(Entry), &e, sizeof e);
        // workgroups that begin in this tensor
        for (; b < s.n_blocks && chunks * b / s.n_blocks < first; ++b)
          std::memcpy(p + ((int64_t)held + b) * sizeof(Entry), &e, sizeof e);
      }
    }
    *set = s;
    return BFS_OK;
  });
}

bfs_status bfs_grad_norm(const bfs_grad_set *set, const void *dev_image, float *norm, void *workspace,
                         int64_t workspace_bytes, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_call("grad_norm", set, dev_image, workspace, workspace_bytes);
    if (st == BFS_OK && !norm) st = fail(BFS_E_INVALID, "grad_norm: null result");
    if (st != BFS_OK) return st;
    double *partial = static_cast<double *>(workspace);
    if (set->n_blocks > 0)
      st = launch("grad_norm", set->grad_bytes >= kStreamNorm ? square_kernel<true> : square_kernel<false>, set->n_blocks, kThreads,
                  kHeldLds, stream, table_of(*set, dev_image), partial);
    if (st != BFS_OK) return st;
    return launch("grad_norm", norm_kernel, 1, kThreads, 0, stream, partial, set->n_blocks, norm);
  });
}

bfs_status bfs_grad_clip(const bfs_grad_set *set, const void *dev_image, double max_norm, float *norm, void *workspace,
                         int64_t workspace_bytes, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_call("grad_clip", set, dev_image, workspace, workspace_bytes);
    if (st == BFS_OK && !(max_norm >= 0.0)) st = fail(BFS_E_INVALID, "grad_clip: max_norm must not be negative");
    if (st == BFS_OK && set->overlap)
      st = fail(BFS_E_INVALID, "grad_clip: an output overlaps another one or a gradient that is not its own");
    if (st != BFS_OK) return st;
    double *partial = static_cast<double *>(workspace);
    if (set->n_blocks == 0) return norm ? launch("grad_clip", norm_kernel, 1, kThreads, 0, stream, partial, 0, norm) : BFS_OK;
    const Table t = table_of(*set, dev_image);
    st = launch("grad_clip", square_kernel<false>, set->n_blocks, kThreads, kHeldLds, stream, t, partial);
    if (st != BFS_OK) return st;
    return launch("grad_clip", clip_kernel, set->n_blocks, kThreads, kHeldLds, stream,
                  t, partial, max_norm, norm);
  });
}

}  // extern "C"
