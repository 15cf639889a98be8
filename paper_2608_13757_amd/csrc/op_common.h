// What the operators beside the plans share: element types, rows in 16-byte
// chunks, reductions inside a wave and the launch call.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <tuple>
#include <type_traits>

#include "bfs_internal.h"

namespace bfsop {

using bfs::fail;

constexpr int kWave = 64;
// With these and at most 64 slots a token, byte counts stay below 2^63.
constexpr int64_t kMaxTokens = ((int64_t)1 << 24) - 1, kMaxWidth = (int64_t)1 << 28;

// 16 bytes of a row.  Rows start at any element (odd widths, views), so the
// alignment is the element's; global accesses of four words need no more.
template <typename T>
struct Chunk {
  static constexpr int kElems = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ T zero_of() {
  return (T)0.0f;
}

// Elements [c * kElems, ...) of a row of n elements: a whole chunk in one
// access, the row's last partial one by elements (zeros past the end).
template <typename T>
__device__ __forceinline__ typename Chunk<T>::vec load_chunk(const T *row, int64_t c, int64_t n) {
  constexpr int E = Chunk<T>::kElems;
  typename Chunk<T>::vec v;
  if ((c + 1) * E <= n) {
    v = *reinterpret_cast<const typename Chunk<T>::vec *>(row + c * E);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = c * E + i < n ? row[c * E + i] : zero_of<T>();
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void store_chunk(T *row, int64_t c, int64_t n, typename Chunk<T>::vec v) {
  constexpr int E = Chunk<T>::kElems;
  if ((c + 1) * E <= n) {
    *reinterpret_cast<typename Chunk<T>::vec *>(row + c * E) = v;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (c * E + i < n) row[c * E + i] = v[i];
  }
}

template <int N>
using Int = std::integral_constant<int, N>;

// f(U, c) for this lane's chunks c, c + step, ..., U of them at once, then with
// U / 2.
template <int U, typename F>
__device__ __forceinline__ void each_chunk(int64_t c, int64_t chunks, int64_t step, F f) {
  for (; c + (U - 1) * step < chunks; c += U * step) f(Int<U>{}, c);
  if constexpr (U > 1) each_chunk<U / 2>(c, chunks, step, f);
}

// Bytes that a call moves from which its accesses are nontemporal: so much is
// not worth keeping in the caches, and memory serves reads and writes faster
// when they pass them by (16384 tokens of 8 rows of 2048 bf16 combined, 605 MB:
// 120 us with plain accesses, 103 with nontemporal loads, 100 with both; 70 MB:
// 13.4 and 14.9; 9 MB: 3.3 and 3.7).
constexpr int64_t kStreamFrom = 96 << 20;

// An access to 16 bytes, nontemporal with kStream.
template <bool kStream, typename T>
__device__ __forceinline__ typename Chunk<T>::vec load(const T *p) {
  auto q = reinterpret_cast<const typename Chunk<T>::vec *>(p);
  return kStream ? __builtin_nontemporal_load(q) : *q;
}

template <bool kStream, typename T>
__device__ __forceinline__ void store(T *p, typename Chunk<T>::vec v) {
  auto q = reinterpret_cast<typename Chunk<T>::vec *>(p);
  if (kStream) __builtin_nontemporal_store(v, q);
  else *q = v;
}

// Whether a group of lanes (8, 16 or 32, a chunk each) takes a token, where a
// wave would leave most of its lanes idle.  One rule for the three operators, from
// where the gradient's two forms cross (us with a wave and with a group, bf16;
// two rows of 64: 32768 tokens 18.7 and 6.1, 6000 4.0 and 3.3, 4000 3.1 and 3.2;
// eight of 128: 6000 9.9 and 9.2, 4000 7.4 and 8.2; four of 256: 8000 9.2 and 9.0,
// 6000 7.8 and 7.7).  The combination's cross earlier (two of 64: 32768 tokens
// 10.8 and 3.8, 6000 3.3 and 2.4, 3000 2.6 and 2.35, 1000 2.25 and 2.3; eight of
// 128: 3000 4.0 and 4.2), the copies of the dispatch near it (8000 tokens, eight
// of 64 11.4 and 10.5, four of 256 11.2 and 11.8).  Eight rows of 256 combined for
// 32768 tokens: 26.4 and 33.1, four 16.2 and 14.8.
inline bool narrow_rows(int64_t chunks, int64_t n_tokens, int32_t k) {
  return chunks <= (k <= 4 ? 32 : 16) && n_tokens >= 6144;
}

// f(lanes of a group) for rows of up to 32 chunks.
template <typename F>
bfs_status with_group(int64_t chunks, F f) {
  if (chunks <= 8) return f(Int<8>{});
  if (chunks <= 16) return f(Int<16>{});
  return f(Int<32>{});
}

constexpr int kLine = 128;                        // bytes of a cache line

// Elements before the first whole line at p.
template <typename T>
__device__ __forceinline__ int head_of(const T *p, int64_t n) {
  const int h = (int)((kLine - (uintptr_t)p % kLine) % kLine / sizeof(T));
  return h < n ? h : (int)n;
}

// Waves that share a token's row of `most` steps of a wave: one round of four
// steps for each (32768 tokens, 2 rows of 4096 bf16 combined: 129 us, with one
// wave for all eight steps 138), one step where that leaves the compute units
// without 4096 waves.
inline int64_t spans_of(int64_t most, int64_t n_tokens) {
  const int64_t rounds = (most + 3) / 4, wanted = (4095 + n_tokens) / n_tokens;
  return wanted < rounds ? rounds : wanted < most ? wanted : most;
}

// Lane i's value from lane i - s of its row of 16 lanes, the row as a ring.
template <int s>
__device__ __forceinline__ uint32_t ror16(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + s, 0xf, 0xf, false);
}

// Reductions over groups of G consecutive lanes (16 or 64); every lane gets
// the same result: inside a row of 16 each step pairs values symmetrically, and
// four rows are joined in the last one's last lane.  none: f(x, none) is x.
template <int G, typename F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t x, uint32_t none, F f) {
  static_assert(G == 16 || G == 64, "groups of 16 or 64 lanes");
  x = f(x, ror16<8>(x));
  x = f(x, ror16<4>(x));
  x = f(x, ror16<2>(x));
  x = f(x, ror16<1>(x));
  if (G == 64) {
    x = f(x, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, 0x142, 0xa, 0xf, false));      // row_bcast:15
    x = f(x, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, 0x143, 0xc, 0xf, false));      // row_bcast:31
    x = (uint32_t)__builtin_amdgcn_readlane((int)x, kWave - 1);
  }
  return x;
}

template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  return group_reduce<G>(x, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

template <int G>
__device__ __forceinline__ uint32_t group_min(uint32_t x) {
  return group_reduce<G>(x, 0xffffffffu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

template <int G>
__device__ __forceinline__ float group_maxf(float x) {
  return __uint_as_float(group_reduce<G>(__float_as_uint(x), 0xff800000u, [](uint32_t a, uint32_t b) {      // -inf
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}

template <int G>
__device__ __forceinline__ float group_sum(float x) {
  return __uint_as_float(group_reduce<G>(__float_as_uint(x), 0x80000000u, [](uint32_t a, uint32_t b) {      // -0
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

// Sum over the lanes up to this one, of all 64: inside each row of 16 lanes, then
// the last lane of a row to the row (of two: to the two) behind it.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);      // row_shr:1
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);      // row_bcast:15
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);      // row_bcast:31
  return x;
}

// Wave index in the workgroup, in a scalar register.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }
__device__ __forceinline__ int lane_index() { return (int)(threadIdx.x & 63u); }

// Between LDS accesses of a wave's lanes to each other's words.  The hardware
// completes a wave's LDS accesses in order; the fences, which cost no
// instruction at this scope, keep the compiler from taking a value that this
// lane stored for one that another lane may have stored since.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename... P, typename... A>
bfs_status launch(const char *what, void (*kernel)(P...), int64_t blocks, int threads, size_t lds, void *stream, A... a) {
  if (blocks * threads >= (int64_t)1 << 32) return fail(BFS_E_RESOURCE, std::string(what) + ": more than 2^32 - 1 threads");
  std::tuple<P...> params(static_cast<P>(a)...);
  void *ptrs[sizeof...(P)];
  std::apply([&](auto &...p) {
    int i = 0;
    ((ptrs[i++] = (void *)&p), ...);
  }, params);
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((uint32_t)blocks), dim3((uint32_t)threads),
                                 ptrs, lds, (hipStream_t)stream);
  if (e != hipSuccess) return fail(BFS_E_DEVICE, std::string(what) + ": launch: " + hipGetErrorString(e));
  return BFS_OK;
}

// No C++ exception leaves a C entry point (the error texts allocate).
template <typename F>
bfs_status entry(F f) noexcept {
  try {
    return f();
  } catch (...) {
    return BFS_E_RESOURCE;
  }
}

// f(T{}) with the element type of a bfs_dtype.
template <typename F>
bfs_status with_type(int32_t dtype, F f) {
  switch (dtype) {
    case BFS_DTYPE_F32: return f(float{});
    case BFS_DTYPE_BF16: return f(__bf16{});
    case BFS_DTYPE_F16: return f(_Float16{});
    default: return fail(BFS_E_INVALID, "unknown dtype");
  }
}

}  // namespace bfsop
