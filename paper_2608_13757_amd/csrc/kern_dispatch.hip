// Dispatch of a mixture of experts: the slots t * k + j of the tokens' chosen
// experts in a stable order by expert, and the tokens' rows in that order.
//
//   expert_off[e]  first row of expert e, expert_off[E] the rows in all;
//   pos[t][j]      the row of slot (t, j): expert_off[e] + the number of
//                  earlier slots of e; -1 for a slot without an expert (an id
//                  outside 0 .. E - 1);
//   perm[pos]      the row's token;   rows[pos] = x[t].
//
// A counting sort without atomics on results: a wave ranks 64 slots at once
// (one ballot per bit of the ids gives each lane the lanes with its expert),
// adds the counts of the earlier batches, waves and groups of slots, so that
// rows come in the same order in every run.  LDS atomics only count.
//
// Up to kSmallSlots slots one launch does all: every workgroup ranks all the
// slots by itself and copies its share of the rows.  Beyond, three: counts of
// each group of slots; ranks, every group summing the counts of the groups
// before it; the copy.
#include <tuple>

#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kMaxExperts = 1024, kMaxK = 64;
constexpr int kSmallWaves = 4, kSmallSlots = 1024;
constexpr int kGroupWaves = 16, kGroupSlots = 4096;
constexpr int kBatches = 4;                            // batches of 64 slots per wave
static_assert(kSmallSlots == kSmallWaves * kBatches * kWave && kGroupSlots == kGroupWaves * kBatches * kWave, "");

struct DispatchParams {
  const int32_t *experts;
  const void *x;
  int32_t *perm, *off, *pos;
  void *rows;
  uint32_t *counts;              // [groups][n_experts]
  int64_t n_slots, x_stride, rows_stride, width;
  int32_t k, n_experts, n_groups, bits;
};

// The ids of this lane's slots: wave w holds batches w * kBatches ... of the
// group that starts at `first`; -1 without an expert or past the end.
__device__ __forceinline__ void load_ids(const DispatchParams &P, int64_t first, int wave, int lane, int (&id)[kBatches]) {
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    const int64_t s = first + (wave * kBatches + b) * kWave + lane;
    const int e = s < P.n_slots ? P.experts[s] : -1;
    id[b] = (uint32_t)e < (uint32_t)P.n_experts ? e : -1;
  }
}

// Counts of each wave's slots by expert, then for each wave the slots of the
// waves before it; total[e] the group's.  hist: [kWaves][n_experts], zeroed
// here.
template <int kWaves>
__device__ __forceinline__ void count_waves(const DispatchParams &P, const int (&id)[kBatches], int wave, uint32_t *hist,
                                            uint32_t *total) {
  const int E = P.n_experts;
  for (int i = (int)threadIdx.x; i < kWaves * E; i += kWaves * kWave) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBatches; ++b)
    if (id[b] >= 0) atomicAdd(&hist[wave * E + id[b]], 1u);
  __syncthreads();
  for (int e = (int)threadIdx.x; e < E; e += kWaves * kWave) {
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = hist[w * E + e];
      hist[w * E + e] = run;
      run += c;
    }
    total[e] = run;
  }
  __syncthreads();
}

// start[e] = sum of total[e'] over e' < e, start[n_experts] = all; wave 0.
__device__ __forceinline__ void expert_starts(int n_experts, const uint32_t *total, uint32_t *start, int wave, int lane) {
  if (wave == 0) {
    uint32_t before = 0;
    for (int e0 = 0; e0 < n_experts; e0 += kWave) {
      const int e = e0 + lane;
      const uint32_t c = e < n_experts ? total[e] : 0;
      uint32_t sum = c;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t up = (uint32_t)__shfl_up((int)sum, d);
        sum += lane >= d ? up : 0;
      }
      if (e < n_experts) start[e] = before + sum - c;
      before += (uint32_t)__builtin_amdgcn_readlane((int)sum, kWave - 1);
    }
    if (lane == 0) start[n_experts] = before;
  }
  __syncthreads();
}

// The row of each of this lane's slots (-1 without an expert): base[e] the
// first row of the group's slots of e, hist the wave's slots before it.  A
// wave's LDS accesses complete in order, so a batch sees the counts that the
// batch before it left.
template <int kWaves>
__device__ __forceinline__ void rank_slots(const DispatchParams &P, const int (&id)[kBatches], int wave, int lane,
                                           uint32_t *hist, const uint32_t *base, int (&row)[kBatches]) {
  const int E = P.n_experts;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    uint64_t same = __ballot(id[b] >= 0);
    row[b] = -1;
    if (same == 0) continue;
    for (int bit = 0; bit < P.bits; ++bit) {
      const uint64_t set = __ballot((id[b] >> bit) & 1);
      same &= (id[b] >> bit) & 1 ? set : ~set;
    }
    if (id[b] >= 0) {
      uint32_t *h = &hist[wave * E + id[b]];
      const uint32_t before = __hip_atomic_load(h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      const int rank = __popcll(same & below);
      row[b] = (int)(base[id[b]] + before) + rank;
      __builtin_amdgcn_wave_barrier();
      if (rank == 0)
        __hip_atomic_store(h, before + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// pos and perm of this lane's slots.
__device__ __forceinline__ void store_ranks(const DispatchParams &P, int64_t first, int wave, int lane, const int (&row)[kBatches]) {
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    const int64_t s = first + (wave * kBatches + b) * kWave + lane;
    if (s < P.n_slots) {
      P.pos[s] = row[b];
      if (row[b] >= 0) P.perm[row[b]] = (int32_t)(s / P.k);
    }
  }
}

// Token t's row to the rows of its slots, lane j's `slot` the row of slot j;
// `c`, `step`: this lane's chunks.
template <typename T>
__device__ __forceinline__ void copy_row(const DispatchParams &P, int64_t t, int64_t c, int64_t step, int slot) {
  const T *x = static_cast<const T *>(P.x) + t * P.x_stride;
  T *out = static_cast<T *>(P.rows);
  const int64_t chunks = (P.width + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
  for (; c < chunks; c += step) {
    const auto v = load_chunk<T>(x, c, P.width);
    for (int j = 0; j < P.k; ++j) {
      const int row = __builtin_amdgcn_readlane(slot, j);
      if (row >= 0) store_chunk<T>(out + (int64_t)row * P.rows_stride, c, P.width, v);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kSmallWaves *kWave) dispatch_small_kernel(DispatchParams P, int64_t spans) {
  extern __shared__ uint32_t lds[];
  uint32_t *hist = lds, *total = hist + kSmallWaves * P.n_experts, *start = total + P.n_experts;
  int32_t *rows = reinterpret_cast<int32_t *>(start + P.n_experts + 1);
  const int wave = wave_index(), lane = lane_index();
  int id[kBatches], row[kBatches];
  load_ids(P, 0, wave, lane, id);
  count_waves<kSmallWaves>(P, id, wave, hist, total);
  expert_starts(P.n_experts, total, start, wave, lane);
  rank_slots<kSmallWaves>(P, id, wave, lane, hist, start, row);
  if (blockIdx.x == 0) {
    store_ranks(P, 0, wave, lane, row);
    for (int e = (int)threadIdx.x; e <= P.n_experts; e += kSmallWaves * kWave) P.off[e] = (int32_t)start[e];
  }
  if (!P.x) return;
#pragma unroll
  for (int b = 0; b < kBatches; ++b) rows[(wave * kBatches + b) * kWave + lane] = row[b];
  __syncthreads();
  // a token's row is copied by `spans` waves
  const int64_t tokens = P.n_slots / P.k, waves = (int64_t)gridDim.x * kSmallWaves;
  for (int64_t u = (int64_t)blockIdx.x * kSmallWaves + wave; u < tokens * spans; u += waves) {
    const int64_t t = u / spans;
    copy_row<T>(P, t, (u - t * spans) * kWave + lane, spans * kWave, lane < P.k ? rows[t * P.k + lane] : -1);
  }
}

__global__ void __launch_bounds__(kGroupWaves *kWave) count_kernel(DispatchParams P) {
  extern __shared__ uint32_t lds[];
  const int wave = wave_index(), lane = lane_index();
  int id[kBatches];
  load_ids(P, (int64_t)blockIdx.x * kGroupSlots, wave, lane, id);
  for (int e = (int)threadIdx.x; e < P.n_experts; e += kGroupWaves * kWave) lds[e] = 0;
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBatches; ++b)
    if (id[b] >= 0) atomicAdd(&lds[id[b]], 1u);
  __syncthreads();
  for (int e = (int)threadIdx.x; e < P.n_experts; e += kGroupWaves * kWave)
    P.counts[(int64_t)blockIdx.x * P.n_experts + e] = lds[e];
}

__global__ void __launch_bounds__(kGroupWaves *kWave) rank_kernel(DispatchParams P) {
  extern __shared__ uint32_t lds[];
  const int E = P.n_experts;
  uint32_t *hist = lds, *total = hist + kGroupWaves * E, *start = total + E, *before = start + E + 1;
  const int wave = wave_index(), lane = lane_index();
  const int64_t first = (int64_t)blockIdx.x * kGroupSlots;
  int id[kBatches], row[kBatches];
  load_ids(P, first, wave, lane, id);
  count_waves<kGroupWaves>(P, id, wave, hist, total);
  for (int e = (int)threadIdx.x; e < E; e += kGroupWaves * kWave) {
    uint32_t all = 0, mine = 0;
    for (int g = 0; g < P.n_groups; ++g) {
      const uint32_t c = P.counts[(int64_t)g * E + e];
      all += c;
      mine += g < (int)blockIdx.x ? c : 0;
    }
    total[e] = all;
    before[e] = mine;
  }
  __syncthreads();
  expert_starts(E, total, start, wave, lane);
  for (int e = (int)threadIdx.x; e <= E; e += kGroupWaves * kWave) {
    if (blockIdx.x == 0) P.off[e] = (int32_t)start[e];
    if (e < E) before[e] += start[e];
  }
  __syncthreads();
  rank_slots<kGroupWaves>(P, id, wave, lane, hist, before, row);
  store_ranks(P, first, wave, lane, row);
}

template <typename T>
__global__ void __launch_bounds__(256) copy_kernel(DispatchParams P) {
  const int64_t t = (int64_t)blockIdx.x * 4 + wave_index();
  if (t >= P.n_slots / P.k) return;
  const int lane = lane_index();
  copy_row<T>(P, t, lane, kWave, lane < P.k ? P.pos[t * P.k + lane] : -1);
}

int64_t groups_of(int64_t slots) { return slots <= kSmallSlots ? 0 : (slots + kGroupSlots - 1) / kGroupSlots; }

bfs_status check_sizes(const char *what, int64_t n_tokens, int32_t k, int32_t n_experts) {
  if (n_tokens < 0 || k < 1 || n_experts < 1) return fail(BFS_E_INVALID, std::string(what) + ": a negative or zero size");
  if (n_experts > kMaxExperts || k > kMaxK || n_tokens > ((int64_t)1 << 31) / k - 1)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 1024 experts, 64 per token and 2^31 - 1 slots");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_moe_dispatch_workspace(int64_t n_tokens, int32_t k, int32_t n_experts, int64_t *bytes) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_sizes("moe_dispatch_workspace", n_tokens, k, n_experts);
    if (st != BFS_OK) return st;
    if (!bytes) return fail(BFS_E_INVALID, "moe_dispatch_workspace: null result");
    *bytes = groups_of(n_tokens * k) * n_experts * (int64_t)sizeof(uint32_t);
    return BFS_OK;
  });
}

bfs_status bfs_moe_dispatch(const int32_t *experts, int64_t n_tokens, int32_t k, int32_t n_experts, int32_t *perm,
                            int32_t *expert_off, int32_t *pos, const void *x, int32_t dtype, int64_t width,
                            int64_t x_stride, void *rows, int64_t rows_stride, void *workspace, int64_t workspace_bytes,
                            struct ihipStream_t *stream) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_sizes("moe_dispatch", n_tokens, k, n_experts);
    if (st != BFS_OK) return st;
    const int64_t slots = n_tokens * k, groups = groups_of(slots), need = groups * n_experts * (int64_t)sizeof(uint32_t);
    if (!expert_off || (slots > 0 && (!experts || !perm || !pos))) return fail(BFS_E_INVALID, "moe_dispatch: null buffer");
    if ((x == nullptr) != (rows == nullptr) && slots > 0)
      return fail(BFS_E_INVALID, "moe_dispatch: x and rows are given together");
    if (x && (width < 0 || x_stride < 0 || rows_stride < width))
      return fail(BFS_E_INVALID, "moe_dispatch: negative stride or width, or rows that overlap");
    if (need > 0 && (!workspace || workspace_bytes < need))
      return fail(BFS_E_INVALID, "moe_dispatch: workspace of " + std::to_string(need) + " bytes needed");
    if ((uintptr_t)workspace % sizeof(uint32_t)) return fail(BFS_E_INVALID, "moe_dispatch: workspace not aligned to 4 bytes");
    DispatchParams P{};
    P.experts = experts;
    P.x = slots > 0 && width > 0 ? x : nullptr;
    P.perm = perm;
    P.off = expert_off;
    P.pos = pos;
    P.rows = rows;
    P.counts = static_cast<uint32_t *>(workspace);
    P.n_slots = slots;
    P.x_stride = x_stride;
    P.rows_stride = rows_stride;
    P.width = width;
    P.k = k;
    P.n_experts = n_experts;
    P.n_groups = (int32_t)groups;
    while ((1 << P.bits) < n_experts) ++P.bits;
    auto copy = [&](auto t) -> bfs_status {
      using T = decltype(t);
      if (groups == 0) {
        const size_t lds = ((kSmallWaves + 2) * (size_t)n_experts + 1 + kSmallSlots) * sizeof(uint32_t);
        int64_t spans = 1, blocks = 1;
        if (P.x) {
          // four chunks for a lane at most while that leaves compute units idle
          const int64_t chunks = (width + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
          const int64_t most = (chunks + kWave - 1) / kWave, wanted = (1024 + n_tokens - 1) / n_tokens;
          spans = most < wanted ? most : wanted;
          blocks = (n_tokens * spans + kSmallWaves - 1) / kSmallWaves;
          blocks = blocks < 512 ? blocks : 512;
        }
        return launch("moe_dispatch", dispatch_small_kernel<T>, blocks, kSmallWaves * kWave, lds, stream, P, spans);
      }
      const size_t lds = ((kGroupWaves + 3) * (size_t)n_experts + 1) * sizeof(uint32_t);
      bfs_status s = launch("moe_dispatch", count_kernel, groups, kGroupWaves * kWave, n_experts * sizeof(uint32_t), stream, P);
      if (s == BFS_OK && lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(rank_kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) s = fail(BFS_E_DEVICE, std::string("moe_dispatch: attribute: ") + hipGetErrorString(e));
      }
      if (s == BFS_OK) s = launch("moe_dispatch", rank_kernel, groups, kGroupWaves * kWave, lds, stream, P);
      if (s == BFS_OK && P.x) s = launch("moe_dispatch", copy_kernel<T>, (n_tokens + 3) / 4, 256, 0, stream, P);
      return s;
    };
    // rows are moved, not computed with: the element's size decides
    switch (dtype) {
      case BFS_DTYPE_F32: return copy(float{});
      case BFS_DTYPE_BF16:
      case BFS_DTYPE_F16: return copy(_Float16{});
      default: return fail(BFS_E_INVALID, "moe_dispatch: unknown dtype");
    }
  });
}

}  // extern "C"
