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
// four lane-rotating instructions (for a whole wave two more, which join the rows
// of 16 lanes, and a read of the last lane into a scalar register).
//
// Logits are compared as unsigned keys in the order of the floats, -0 as +0, NaN
// above everything.  A 16-bit logit's key and its expert's number make one word,
// all different, so that a maximum finds the lowest of equal ones by itself; of
// fp32 logits the upper part of the key does (select), or the lanes that hold the
// maximum are counted.
//
// The softmax is in fp32 whatever the logits' type; exponentials are exp2 of
// the product with log2 e, off by some 2 |z - m| 2^-24 relative to themselves;
// weights below fp32's normal numbers become 0.
//
// Bound by instructions for many tokens (the lanes' sorts and k rounds of a
// maximum).  32768 tokens, k = 8: 64 experts, bf16: 4.3 us, where reading and
// writing would take 1.2 (4.9 with a maximum over all values of a lane in every
// round, 6.6 with equal keys found by a second reduction); 256 experts: bf16 9.4 us
// (11.7, reading 3.2), fp32 11.8 (15.3, reading 6.3).  Of these the vector
// instructions alone, 213, 516 and 492 a wave, 8 waves a SIMD, four clocks each
// at 2.4 GHz, are 2.8, 6.9 and 6.6 us; of 512 experts fp32 (20.1 us, reading
// 12.7), 346 a wave, 32 waves a SIMD, 18.5.  1024 experts: bf16 27, fp32 35 us.
//
// The gradient of 16384 tokens, 256 experts, fp32: 8.4 us over all experts (11.5
// with the k terms compared with every expert), where reading and writing would
// take 6.5, and 6.5 over the chosen ones, which reads k logits of a row.
#include <cmath>
#include <utility>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = 1024, kMaxK = 16;

// Keys in the order of the logits; the key of a masked or absent expert is at
// most kMasked.  value gives a key's logit.
template <typename T>
struct Key;

template <>
struct Key<float> {
  static constexpr uint32_t kMasked = 0x007fffffu, kNan = 0xffffffffu;
  __device__ static uint32_t of(float z, int) {
    if (z != z) return kNan;
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  }
  __device__ static float value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
};

// The logit's 16 bits above the expert's number from 65535 down.
template <typename T>
struct Key16 {
  __device__ static uint32_t of(float z, int e) {
    const uint32_t u = __builtin_bit_cast(uint16_t, (T)(z + 0.0f));
    const uint32_t k = z != z ? 0xffffu : u ^ (u & 0x8000u ? 0xffffu : 0x8000u);
    return k << 16 | (0xffffu - (uint32_t)e);
  }
  __device__ static int expert(uint32_t key) { return (int)(0xffffu - (key & 0xffffu)); }
  __device__ static float value(uint32_t key) {
    const uint32_t k = key >> 16;
    return (float)__builtin_bit_cast(T, (uint16_t)(k ^ (k & 0x8000u ? 0x8000u : 0xffffu)));
  }
};

template <>
struct Key<__bf16> : Key16<__bf16> {
  static constexpr uint32_t kMasked = 0x007fffffu;      // -inf: 0xff80
};

template <>
struct Key<_Float16> : Key16<_Float16> {
  static constexpr uint32_t kMasked = 0x03ffffffu;      // -inf: 0xfc00
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

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

// Batcher's odd-even merging network for N values: `n` comparisons of a[] < b[].
template <int N>
struct Network {
  int a[64] = {}, b[64] = {}, n = 0;
  constexpr Network() {
    for (int p = 1; p < N; p <<= 1)
      for (int q = p; q >= 1; q >>= 1)
        for (int j = q % p; j + q < N; j += 2 * q)
          for (int i = j; i < j + q && i + q < N; ++i)
            if (i / (2 * p) == (i + q) / (2 * p)) {
              a[n] = i;
              b[n++] = i + q;
            }
  }
};

// v in descending order.
template <int N, size_t... I>
__device__ __forceinline__ void sort_down(uint32_t (&v)[N], std::index_sequence<I...>) {
  constexpr Network<N> net{};
  auto order = [](uint32_t &x, uint32_t &y) {
    const uint32_t hi = x > y ? x : y, lo = x > y ? y : x;
    x = hi;
    y = lo;
  };
  (order(v[net.a[I]], v[net.b[I]]), ...);
}

// The `rounds` <= R largest of each group's keys, all different but for 0:
// lane j gets the j-th, every lane the first (`most`), the last one, and the one
// before it.  Each lane sorts its own, so that a round looks at the lanes' first
// ones alone; of what is behind them only as many as there are rounds left move up.
template <int G, int N, int R, int J = 0>
__device__ __forceinline__ void take_rounds(uint32_t (&key)[N], int l, int rounds, uint32_t &mine, uint32_t &most, uint32_t &last,
                                            uint32_t &before) {
  if constexpr (J < R) {
    if (J >= rounds) return;
    const uint32_t m = group_max<G>(key[0]);
    const bool hit = key[0] == m;
#pragma unroll
    for (int i = 0; i < (N < R - 1 - J ? N : R - 1 - J); ++i) key[i] = hit ? (i + 1 < N ? key[i + 1] : 0u) : key[i];
    mine = l == J ? m : mine;
    if (J == 0) most = m;
    before = last;
    last = m;
    take_rounds<G, N, R, J + 1>(key, l, rounds, mine, most, last, before);
  }
}

template <int G, int N, int R>
__device__ __forceinline__ uint32_t take_largest(uint32_t (&key)[N], int l, int rounds, uint32_t &most, uint32_t &last, uint32_t &before) {
  sort_down(key, std::make_index_sequence<(size_t)Network<N>{}.n>{});
  uint32_t mine = most = last = before = 0;
  take_rounds<G, N, R>(key, l, rounds, mine, most, last, before);
  return mine;
}

// Lane J's value of each group, for all its lanes.
template <int G, int J>
__device__ __forceinline__ uint32_t group_read(uint32_t x) {
  if (G == 64) return (uint32_t)__builtin_amdgcn_readlane((int)x, J);
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + J, 0xf, 0xf, false);       // row_newbcast
}

// Exact for any fp32 keys: a maximum in each round, and the lowest of the
// experts that hold it; with kCount these are looked for only where several
// lanes of a row hold it (fewer instructions, more registers).  In lane j < k
// the j-th key and its expert, -1 without one; top: the largest key.
template <int G, int N, bool kCount>
__device__ __forceinline__ int select_ties(uint32_t (&key)[N], int l, int k, uint32_t &my_key, uint32_t &top) {
  using L = Layout<G, N>;
  // the lane that holds the maximum leaves it and its expert for lane j
  __shared__ uint2 found[kThreads / G][kMaxK];
  uint2 *mine = found[threadIdx.x / G];
  for (int j = 0; j < k; ++j) {
    uint32_t own = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) own = key[i] > own ? key[i] : own;
    const uint32_t m = group_max<G>(own);
    if (j == 0) top = m;
    bool has = own == m;
    uint32_t e = 0;
    if (!kCount || __builtin_popcountll(__ballot(has)) != kWave / G) {
      e = 0x7fffffffu;
#pragma unroll
      for (int i = N - 1; i >= 0; --i) e = key[i] == m ? (uint32_t)L::index(l, i) : e;
      has = e == group_min<G>(e);
    }
    bool left = has;
#pragma unroll
    for (int i = 0; i < N; ++i) {                                  // experts ascend: the first of equal ones
      const bool hit = left && key[i] == m;
      key[i] = hit ? 0u : key[i];
      if (kCount) e = hit ? (uint32_t)L::index(l, i) : e;
      left = left && !hit;
    }
    if (has) mine[j] = make_uint2(m, e);
  }
  wave_sync();
  const uint2 f = l < k ? mine[l] : make_uint2(0, 0);
  my_key = f.x;
  return f.x > Key<float>::kMasked ? (int)f.y : -1;
}

// Whether a row is sorted.  fp32 rows of few values a lane, or of which few are
// wanted, go by their whole keys at once (32768 tokens: 64 experts, k = 4: 4.4
// us, sorted 4.5; 256, k = 2: 8.7 and 8.8, k = 4: 10.7 and 9.4).
template <typename T, int N, int K>
constexpr bool kSorts = sizeof(T) == 2 || (N >= 8 && K > 2);

// The k largest logits of each group's row: in lane j < k the j-th's expert
// and value (-1 and -inf without one), in every lane the largest value.
// fp32 logits are compared by what of a key stands above the bits of the
// expert's number, then the chosen ones read again: where two of them, or the
// last and any that is left, agree in that part and not in the whole (a few in
// a hundred rows of random logits), the wave takes the exact way.
template <typename T, int G, int N, int K>
__device__ __forceinline__ void select(const T *row, const float (&z)[N], int l, int n_experts, int k, int &my_expert,
                                       float &my_value, float &top) {
  using L = Layout<G, N>;
  uint32_t key[N], most, last, before;
  my_expert = -1;
  my_value = -INFINITY;
  auto whole_keys = [&] {
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = L::index(l, i) < n_experts ? Key<T>::of(z[i], L::index(l, i)) : 0u;
  };
  if constexpr (!kSorts<T, N, K>) {
    uint32_t mine, most;
    whole_keys();
    my_expert = select_ties<G, N, true>(key, l, k, mine, most);
    if (my_expert >= 0) my_value = Key<T>::value(mine);
    top = Key<T>::value(most);
  } else if constexpr (sizeof(T) == 2) {
    whole_keys();
    const uint32_t mine = take_largest<G, N, K>(key, l, k, most, last, before);
    if (mine > Key<T>::kMasked) {
      my_expert = Key<T>::expert(mine);
      my_value = Key<T>::value(mine);
    }
    top = Key<T>::value(most);
  } else {
    constexpr uint32_t kNumber = G * N - 1;                        // bits of an expert's number
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t e = (uint32_t)L::index(l, i);
      key[i] = (int)e < n_experts ? (Key<T>::of(z[i], 0) & ~kNumber) | (kNumber - e) : 0u;
    }
    const uint32_t mine = take_largest<G, N, K + 1>(key, l, k + 1, most, last, before);
    const bool valid = l < k && mine > Key<T>::kMasked;
    if (valid) {
      my_expert = (int)(kNumber - (mine & kNumber));
      my_value = row[my_expert];
    }
    const uint32_t whole = Key<T>::of(my_value, 0);
    const uint32_t next = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0x101, 0xf, 0xf, true);        // row_shl:1
    const uint32_t next_whole = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)whole, 0x101, 0xf, 0xf, true);
    bool unclear = valid && l + 1 < k && ((mine ^ next) & ~kNumber) == 0 && whole != next_whole;
    const bool border = before > Key<T>::kMasked && ((before ^ last) & ~kNumber) == 0;
    if (__ballot(border)) {                                        // clear where all that agree in part agree in the whole
      const uint32_t at = (uint32_t)__shfl((int)whole, (lane_index() & ~(G - 1)) + k - 1);
#pragma unroll
      for (int i = 0; i < N; ++i) unclear |= border && (Key<T>::of(z[i], 0) ^ at) - 1 < kNumber;
    }
    if (__ballot(unclear)) {
      uint32_t key_of_mine;
      whole_keys();
      my_expert = select_ties<G, N, false>(key, l, k, key_of_mine, most);
      my_value = my_expert >= 0 ? Key<T>::value(key_of_mine) : -INFINITY;
    }
    top = __uint_as_float(group_read<G, 0>(__float_as_uint(my_value)));
  }
}

template <typename T, int G, int N, int K>
__global__ void __launch_bounds__(kThreads) route_kernel(const T *logits, int64_t n_tokens, int n_experts, int64_t stride,
                                                         int k, int renorm, int32_t *experts, float *weights) {
  const int l = (int)(threadIdx.x % G);
  const int64_t token = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const bool live = token < n_tokens;
  const T *row = logits + (live ? token : 0) * stride;
  float z[N], my_value, m;
  load_row<T, G, N>(row, l, n_experts, z);
  int my_expert;
  select<T, G, N, K>(row, z, l, n_experts, k, my_expert, my_value, m);
  const float mine = my_expert >= 0 ? exp_of(my_value - m) : 0.0f;
  float total;
  if (renorm) {
    total = group_sum<G>(mine);
  } else {
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) total += exp_of(z[i] - m);
    total = group_sum<G>(total);
  }
  if (live && l < k) {
    experts[token * k + l] = my_expert;
    weights[token * k + l] = my_expert >= 0 ? mine / total : 0.0f;
  }
}

// Sum of v over the lanes j < k of a group with this lane's e, in their order.
template <int G, int J = 0>
__device__ __forceinline__ float sum_equal(int e, float v, int k, float sum = 0.0f) {
  if constexpr (J < kMaxK) {
    if (J >= k) return sum;
    const uint32_t ej = group_read<G, J>((uint32_t)e);
    const float vj = __uint_as_float(group_read<G, J>(__float_as_uint(v)));
    return sum_equal<G, J + 1>(e, v, k, sum + ((int)ej == e ? vj : 0.0f));
  }
  return sum;
}

// The k terms are laid out over the row's experts in LDS: zeros, then each
// chosen expert's term (slots that name the same expert write the same sum of
// theirs), then every lane reads its experts'.
template <typename T, int G, int N>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const T *logits, int64_t n_tokens, int n_experts,
                                                              int64_t stride, const int32_t *experts, int k,
                                                              const float *grad_weights, int renorm, T *grad_logits,
                                                              int64_t grad_stride) {
  using L = Layout<G, N>;
  constexpr int V = L::V;
  __shared__ __attribute__((aligned(16))) float lds[kThreads / G][G * N];
  typedef float fvec __attribute__((ext_vector_type(V)));
  float *terms = lds[threadIdx.x / G];
  const int l = (int)(threadIdx.x % G);
  const int64_t token = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const bool live = token < n_tokens;
  const T *row = logits + (live ? token : 0) * stride;
  // lane j < k: the j-th chosen expert, its logit and its weight's gradient
  int e = -1;
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
#pragma unroll
  for (int c = 0; c < N / V; ++c) *reinterpret_cast<fvec *>(&terms[L::index(l, c * V)]) = fvec(0.0f);
  float z[N], s = 0.0f, term;
  if (renorm) {
    const float m = group_maxf<G>(ze);
    float p = ze == -INFINITY ? 0.0f : exp_of(ze - m);
    const float total = group_sum<G>(p);
    p = total == 0.0f ? 0.0f : p / total;
    term = p * (g - group_sum<G>(p * g));
  } else {
    load_row<T, G, N>(row, l, n_experts, z);
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    m = group_maxf<G>(m);
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] = z[i] == -INFINITY ? 0.0f : exp_of(z[i] - m);
      total += z[i];
    }
    total = group_sum<G>(total);
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const float p = ze == -INFINITY ? 0.0f : exp_of(ze - m) * inv;
    s = group_sum<G>(p * g);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= inv;
    term = g;
  }
  term = sum_equal<G>(e, term, k);
  wave_sync();
  if (e >= 0) terms[e] = term;
  wave_sync();
  if (!live) return;
  T *out = grad_logits + token * grad_stride;
  typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
#pragma unroll
  for (int c = 0; c < N / V; ++c) {
    const int e0 = L::index(l, c * V);
    fvec d = *reinterpret_cast<const fvec *>(&terms[e0]);
    if (!renorm) {
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = z[c * V + i] * (d[i] - s);
    }
    if (e0 + V <= n_experts) {
      vec o;
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = (T)d[i];
      *reinterpret_cast<vec *>(out + e0) = o;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i < n_experts) out[e0 + i] = (T)d[i];
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
  if (n_experts > kMaxExperts || k > kMaxK || n_tokens > kMaxTokens)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 1024 experts, 16 per token and 2^24 - 1 tokens");
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
        auto kernel = route_kernel<T, G, N, 2>;
        if constexpr (kSorts<T, N, kMaxK>)
          if (k > 2) kernel = k <= 8 ? route_kernel<T, G, N, 8> : route_kernel<T, G, N, kMaxK>;
        return launch("moe_route", kernel, (n_tokens + kRows - 1) / kRows, kThreads, 0, stream,
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
