// Router of a mixture of experts: for each token's logits z[0 .. E-1]
//
//   e_1 .. e_k   the experts of the k largest logits, largest first, equal
//                logits by the lower index; an expert at -inf is masked and
//                never chosen (-1, weight 0, where fewer than k are left);
//   w_j        = exp(z[e_j] - m) / sum over all experts of exp(z - m), or over
//                the chosen ones (renormalized), m the largest logit;
//
// and the gradient for given dw:
//
//   all experts   dz[i] = p[i] (sum of dw_j over e_j = i  -  s),
//                 s = sum over j of dw_j p[e_j]
//   renormalized  dz[e_j] += w_j (dw_j - sum over i of dw_i w_i), else 0.
//
// A row lies in the registers of 16 lanes (four rows per wave) up to 256
// experts, of a whole wave beyond, N values each, so that a reduction takes
// four lane-rotating instructions (and two cross-lane reads beyond 16 lanes).
// Logits are compared as unsigned keys in the order of the floats, -0 as +0,
// NaN above everything; the softmax is in fp32 whatever the logits' type.
#include <cmath>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = 1024, kMaxK = 16;
constexpr uint32_t kMaskedKey = 0x007fffffu;       // key of -inf; 0: no expert
constexpr uint32_t kNanKey = 0xffffffffu;

__device__ __forceinline__ uint32_t key_of(float z) {
  if (z != z) return kNanKey;
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// Lane l of a group holds elements (c * G + l) * V + v: V consecutive ones in
// one access.
template <int G, int N>
struct Layout {
  static constexpr int V = N < 4 ? N : 4;
  __device__ static int index(int l, int i) { return ((i / V) * G + l) * V + i % V; }
};

template <typename T, int G, int N>
__device__ __forceinline__ void load_row(const T *row, int l, int n_experts, float (&z)[N]) {
  constexpr int V = Layout<G, N>::V;
  typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
#pragma unroll
  for (int c = 0; c < N / V; ++c) {
    const int e0 = Layout<G, N>::index(l, c * V);
    if (e0 + V <= n_experts) {
      const vec v = *reinterpret_cast<const vec *>(row + e0);
#pragma unroll
      for (int i = 0; i < V; ++i) z[c * V + i] = (float)v[i];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) z[c * V + i] = e0 + i < n_experts ? (float)row[e0 + i] : -INFINITY;
    }
  }
}

template <typename T, int G, int N>
__global__ void __launch_bounds__(kThreads) route_kernel(const T *logits, int64_t n_tokens, int n_experts, int64_t stride,
                                                         int k, int renorm, int32_t *experts, float *weights) {
  using L = Layout<G, N>;
  const int l = (int)(threadIdx.x % G);
  const int64_t token = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const bool live = token < n_tokens;
  float z[N];
  load_row<T, G, N>(logits + (live ? token : 0) * stride, l, n_experts, z);
  uint32_t key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = L::index(l, i) < n_experts ? key_of(z[i]) : 0u;
  int32_t my_expert = -1;
  uint32_t my_key = 0, top = 0;
  for (int j = 0; j < k; ++j) {
    uint32_t m = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = key[i] > m ? key[i] : m;
    m = group_max<G>(m);
    uint32_t e = 0x7fffffffu;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) e = key[i] == m ? (uint32_t)L::index(l, i) : e;
    e = group_min<G>(e);
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = (uint32_t)L::index(l, i) == e ? 0u : key[i];
    if (j == 0) top = m;
    if (l == j && m > kMaskedKey) {
      my_expert = (int32_t)e;
      my_key = m;
    }
  }
  const float m = value_of(top);
  const float mine = my_expert >= 0 ? expf(value_of(my_key) - m) : 0.0f;
  float total;
  if (renorm) {
    total = group_sum<G>(mine);
  } else {
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) total += expf(z[i] - m);
    total = group_sum<G>(total);
  }
  if (live && l < k) {
    experts[token * k + l] = my_expert;
    weights[token * k + l] = my_expert >= 0 ? mine / total : 0.0f;
  }
}

// Lane j's value of each group, for all its lanes.
template <int G>
__device__ __forceinline__ uint32_t group_read(uint32_t x, int j) {
  if (G == 64) return (uint32_t)__builtin_amdgcn_readlane((int)x, j);
  return (uint32_t)__shfl((int)x, (int)(threadIdx.x & 48u) + j);
}

template <typename T, int G, int N>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const T *logits, int64_t n_tokens, int n_experts,
                                                              int64_t stride, const int32_t *experts, int k,
                                                              const float *grad_weights, int renorm, T *grad_logits,
                                                              int64_t grad_stride) {
  using L = Layout<G, N>;
  constexpr int V = L::V;
  const int l = (int)(threadIdx.x % G);
  const int64_t token = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const bool live = token < n_tokens;
  const T *row = logits + (live ? token : 0) * stride;
  // lane j < k: the j-th chosen expert, its logit and its weight's gradient
  int32_t e = -1;
  float g = 0.0f, ze = -INFINITY;
  if (live && l < k) {
    e = experts[token * k + l];
    if ((uint32_t)e < (uint32_t)n_experts) {
      g = grad_weights[token * k + l];
      ze = (float)row[e];
    } else {
      e = -1;
    }
  }
  float z[N], dz[N];
  float p, v;                 // the chosen expert's probability and its term of dz
  if (renorm) {
    const float m = group_maxf<G>(ze);
    p = ze == -INFINITY ? 0.0f : expf(ze - m);
    const float total = group_sum<G>(p);
    p = total == 0.0f ? 0.0f : p / total;
    v = p * (g - group_sum<G>(p * g));
#pragma unroll
    for (int i = 0; i < N; ++i) dz[i] = 0.0f;
  } else {
    load_row<T, G, N>(row, l, n_experts, z);
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    m = group_maxf<G>(m);
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] = z[i] == -INFINITY ? 0.0f : expf(z[i] - m);
      total += z[i];
    }
    total = group_sum<G>(total);
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    p = ze == -INFINITY ? 0.0f : expf(ze - m) * inv;
    const float s = group_sum<G>(p * g);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] *= inv;
      dz[i] = -s;
    }
    v = g;
  }
  for (int j = 0; j < k; ++j) {
    const uint32_t ej = group_read<G>((uint32_t)e, j);
    const float vj = __uint_as_float(group_read<G>(__float_as_uint(v), j));
#pragma unroll
    for (int i = 0; i < N; ++i) dz[i] += (uint32_t)L::index(l, i) == ej ? vj : 0.0f;
  }
  if (!renorm) {
#pragma unroll
    for (int i = 0; i < N; ++i) dz[i] *= z[i];
  }
  if (!live) return;
  T *out = grad_logits + token * grad_stride;
  typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
#pragma unroll
  for (int c = 0; c < N / V; ++c) {
    const int e0 = L::index(l, c * V);
    if (e0 + V <= n_experts) {
      vec o;
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = (T)dz[c * V + i];
      *reinterpret_cast<vec *>(out + e0) = o;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i < n_experts) out[e0 + i] = (T)dz[c * V + i];
    }
  }
}

// f(group lanes, values per lane) for a row of n_experts.
template <typename F>
bfs_status with_layout(int n_experts, F f) {
  using std::integral_constant;
  if (n_experts <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (n_experts <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (n_experts <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (n_experts <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (n_experts <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  if (n_experts <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

bfs_status check_route(const char *what, int64_t n_tokens, int32_t n_experts, int64_t stride, int32_t k, uint32_t flags) {
  if (n_tokens < 0 || n_experts < 1 || k < 1) return fail(BFS_E_INVALID, std::string(what) + ": a negative or zero size");
  if (k > n_experts) return fail(BFS_E_INVALID, std::string(what) + ": k exceeds the number of experts");
  if (n_experts > kMaxExperts || k > kMaxK || n_tokens >= (int64_t)1 << 31)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 1024 experts, 16 per token and 2^31 - 1 tokens");
  if (stride < 0) return fail(BFS_E_INVALID, std::string(what) + ": negative stride");
  if (flags & ~BFS_MOE_RENORMALIZE) return fail(BFS_E_INVALID, std::string(what) + ": unknown flags");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_moe_route(const void *logits, int32_t dtype, int64_t n_tokens, int32_t n_experts, int64_t logits_stride,
                         int32_t k, uint32_t flags, int32_t *experts, float *weights, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_route("moe_route", n_tokens, n_experts, logits_stride, k, flags);
    if (st != BFS_OK) return st;
    return with_type(dtype, [&](auto t) -> bfs_status {
      using T = decltype(t);
      if (n_tokens == 0) return BFS_OK;
      if (!logits || !experts || !weights) return fail(BFS_E_INVALID, "moe_route: null buffer");
      return with_layout(n_experts, [&](auto g, auto n) {
        constexpr int G = decltype(g)::value, N = decltype(n)::value, kRows = kThreads / G;
        return launch("moe_route", route_kernel<T, G, N>, (n_tokens + kRows - 1) / kRows, kThreads, 0, stream,
                      static_cast<const T *>(logits), n_tokens, n_experts, logits_stride, k,
                      (int)(flags & BFS_MOE_RENORMALIZE), experts, weights);
      });
    });
  });
}

bfs_status bfs_moe_route_grad(const void *logits, int32_t dtype, int64_t n_tokens, int32_t n_experts,
                              int64_t logits_stride, const int32_t *experts, int32_t k, const float *grad_weights,
                              uint32_t flags, void *grad_logits, int64_t grad_stride, struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_route("moe_route_grad", n_tokens, n_experts, logits_stride, k, flags);
    if (st != BFS_OK) return st;
    if (grad_stride < n_experts) return fail(BFS_E_INVALID, "moe_route_grad: the gradient's rows overlap");
    return with_type(dtype, [&](auto t) -> bfs_status {
      using T = decltype(t);
      if (n_tokens == 0) return BFS_OK;
      if (!logits || !experts || !grad_weights || !grad_logits) return fail(BFS_E_INVALID, "moe_route_grad: null buffer");
      return with_layout(n_experts, [&](auto g, auto n) {
        constexpr int G = decltype(g)::value, N = decltype(n)::value, kRows = kThreads / G;
        return launch("moe_route_grad", route_grad_kernel<T, G, N>, (n_tokens + kRows - 1) / kRows, kThreads, 0, stream,
                      static_cast<const T *>(logits), n_tokens, n_experts, logits_stride, experts, k, grad_weights,
                      (int)(flags & BFS_MOE_RENORMALIZE), static_cast<T *>(grad_logits), grad_stride);
      });
    });
  });
}

}  // extern "C"
