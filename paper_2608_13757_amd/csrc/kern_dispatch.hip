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
// The slots go in groups of up to 1024, a workgroup ranks a whole group.  Up to
// 8192 slots it counts the other groups' too.  Beyond, one launch counts each
// group's slots by expert, and the ranking workgroups sum the groups before
// theirs, or, where that table is long, read sums that one more launch makes.
// The rows are copied by the ranking workgroups where 512 of them give each
// wave one part of a row, or a few in the caches: several then rank the same
// group, each for itself, and one launch is saved (2048 tokens of 4096 bf16 to
// eight experts each: 32 us, with the copy in a launch of its own 35; 128 tokens
// to two: 3.9 us in a single launch).  Beyond, the copy is a launch of its own,
// whose waves end with their stores under way.
//
// Bound by memory: 32768 tokens of 4096 bf16 to two experts of 64 each, 806 MB,
// in 150 us (5.4 TB/s, a large copy's rate), some 9 us of them the ranking.
#include "op_common.h"

using namespace bfsop;

namespace {

constexpr int kMaxExperts = 1024, kMaxK = 64;
// Ranking: a group's batches of 64 slots over eight waves, two each (1000 tokens
// to two of 64 experts 5.3 us, over four waves, four each, 6.3; 4000 to one 7.6
// and 10.6; 8 tokens 3.9 and 3.7).
constexpr int kWaves = 8, kThreads = kWaves * kWave;
constexpr int kBatches = 2;
constexpr int kCopyWaves = 4, kCopyThreads = kCopyWaves * kWave;
constexpr int kGroupSlots = kWaves * kBatches * kWave;
constexpr int kBlocks = 512;                          // workgroups that rank and copy, at most
// Slots up to which every ranking workgroup counts all by itself (3000 tokens of
// 512 bf16 to two experts of 64: 8.5 us, with a launch that counts 9.4; 16000 to
// one of 16: 19.3 and 18.0).
constexpr int kAlone = 8192;
// Counts that every ranking workgroup sums by itself (8000 tokens to eight of 128
// experts, 8064 counts: 24.7 us, with a launch that sums them 23.4).
constexpr int64_t kSumEntries = 4096;

struct DispatchParams {
  const int32_t *experts;
  const void *x;
  int32_t *perm, *off, *pos;
  void *rows;
  uint32_t *counts;              // [n_groups][n_experts]; with sums: of the groups before, and [n_groups]: of all
  int64_t n_slots, x_stride, rows_stride, width, spans;
  int32_t k, n_experts, n_groups, group, parts, bits, batches;   // group: slots of one, whole tokens
};

// The place in its group of this lane's slot of batch b: a wave's batches follow
// each other, as many for each wave as a group needs (P.batches).
__device__ __forceinline__ int place_of(const DispatchParams &P, int wave, int lane, int b) {
  return (wave * P.batches + b) * kWave + lane;
}

// The ids of this lane's slots of group g; -1 without an expert, past the end and
// in batches that are not used.
__device__ __forceinline__ void load_ids(const DispatchParams &P, int g, int wave, int lane, int (&id)[kBatches]) {
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    const int i = place_of(P, wave, lane, b);
    const int64_t s = (int64_t)g * P.group + i;
    const int e = b < P.batches && i < P.group && s < P.n_slots ? P.experts[s] : -1;
    id[b] = (uint32_t)e < (uint32_t)P.n_experts ? e : -1;
  }
}

// Counts the wave's ids in LDS (-1: none).  The first lane's id, which under a
// skewed routing many share, is counted by one access for all of them: atomics
// on one word run one lane after the other (4000 slots, most of them of two
// experts, counted by every workgroup: 12.1 us without this, 8.7 with it).
__device__ __forceinline__ void count_ids(uint32_t *counts, int id, int lane) {
  const int first = __builtin_amdgcn_readfirstlane(id);
  const uint64_t same = __ballot(id == first);
  const bool one = lane == __builtin_ctzll(same);
  if (id >= 0 && (id != first || one)) atomicAdd(&counts[id], one ? (uint32_t)__popcll(same) : 1u);
}

// Counts of each wave's slots by expert, then for each wave the slots of the
// waves before it; total[e] the group's.  hist: [kWaves][n_experts], zeroed
// here.  Without a table of counts (up to kAlone slots) the other groups' slots
// are counted too: before[e] of the groups before this one, after[e] behind it,
// total[e] of all; others: after[n_experts + 1], then before[n_experts].
__device__ __forceinline__ void count_waves(const DispatchParams &P, const int (&id)[kBatches], int g, int wave, int lane,
                                            uint32_t *hist, uint32_t *total, uint32_t *others) {
  typedef int32_t ids __attribute__((ext_vector_type(4), aligned(4)));
  constexpr int kRounds = kAlone / (4 * kThreads);
  const int E = P.n_experts, slots = (int)P.n_slots, first = g * P.group;
  const bool alone = P.n_groups > 1 && !P.counts;
  ids other[kRounds];
  if (alone) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (r * kThreads * 4 >= slots) break;
      const int s = (r * kThreads + (int)threadIdx.x) * 4;
      if (s + 4 <= slots) {
        other[r] = *reinterpret_cast<const ids *>(P.experts + s);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) other[r][i] = s + i < slots ? P.experts[s + i] : -1;
      }
    }
    for (int i = (int)threadIdx.x; i < 2 * E + 1; i += kThreads) others[i] = 0;
  }
  for (int i = (int)threadIdx.x; i < kWaves * E; i += kThreads) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBatches; ++b)
    count_ids(hist + wave * E, id[b], lane);
  if (alone) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (r * kThreads * 4 >= slots) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = (r * kThreads + (int)threadIdx.x) * 4 + i;
        const bool counts = (uint32_t)other[r][i] < (uint32_t)E && (uint32_t)(s - first) >= (uint32_t)P.group;
        count_ids(others, counts ? other[r][i] + (s < first ? E + 1 : 0) : -1, lane);
      }
    }
  }
  __syncthreads();
  for (int e = (int)threadIdx.x; e < E; e += kThreads) {
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = hist[w * E + e];
      hist[w * E + e] = run;
      run += c;
    }
    total[e] = alone ? run + others[e] + others[E + 1 + e] : run;
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
      const uint32_t sum = wave_scan(c);
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
      wave_sync();
      if (rank == 0)
        __hip_atomic_store(h, before + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    wave_sync();
  }
}

// Slots by expert of the groups before g, and of all groups.  Several threads
// (`share`) share an expert's groups where that leaves no thread without one.  Of
// a table of some length the first counts of a thread are on their way while it
// counts its own slots (rows of 64 bf16, 8000 tokens to eight experts of 64, 4032
// counts: 11.8 -> 10.5 us; 2400 to four of 16, 160 counts: 8.0 and 8.3).
struct GroupSums {
  static constexpr int kAhead = 8, kAheadFrom = 1024;
  int share, my, e;              // this thread: expert e, groups my, my + share, ...
  bool table, early;
  uint32_t ahead[kAhead];

  __device__ __forceinline__ void load(const DispatchParams &P) {
    // There are kAlone / kGroupSlots + 1 groups at least, so that a table which is
    // summed here has no more experts than a workgroup threads.
    static_assert(kSumEntries / (kAlone / kGroupSlots + 1) <= kThreads, "a thread for each expert");
    const int E = P.n_experts, t = (int)threadIdx.x;
    table = P.n_groups * (int64_t)E > kSumEntries;
    early = !table && P.n_groups * E >= kAheadFrom;
    if (table) return;
    share = kThreads / E;
    my = t / E;
    e = t - my * E;
    if (!early) return;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = my + u * share;
      ahead[u] = my < share && i < P.n_groups ? P.counts[i * E + e] : 0;
    }
  }

  __device__ __forceinline__ void sum(const DispatchParams &P, int g, uint32_t *before, uint32_t *total) const {
    const int E = P.n_experts;
    if (table) {
      for (int e = (int)threadIdx.x; e < E; e += kThreads) {
        before[e] = P.counts[(int64_t)g * E + e];
        total[e] = P.counts[(int64_t)P.n_groups * E + e];
      }
    } else {
      if (my == 0) before[e] = total[e] = 0;
      __syncthreads();
      if (my < share) {
        uint32_t all = 0, mine = 0;
        int i = my;
        if (early) {
#pragma unroll
          for (int u = 0; u < kAhead; ++u, i += share) {
            all += ahead[u];
            mine += i < g ? ahead[u] : 0;
          }
        }
#pragma unroll 8
        for (; i < P.n_groups; i += share) {
          const uint32_t c = P.counts[i * E + e];
          all += c;
          mine += i < g ? c : 0;
        }
        atomicAdd(&total[e], all);
        atomicAdd(&before[e], mine);
      }
    }
    __syncthreads();
  }
};

// Token t's row to the rows of its slots, lane j's `slot` the row of slot j;
// this lane takes chunks `at`, at + step, ...
template <typename T, bool kStream>
__device__ __forceinline__ void copy_row(const DispatchParams &P, int64_t t, int64_t at, int64_t step, int slot) {
  constexpr int E = Chunk<T>::kElems;
  const T *x = static_cast<const T *>(P.x) + t * P.x_stride;
  T *out = static_cast<T *>(P.rows);
  const int64_t chunks = P.width / E;
  const uint64_t set = __ballot(slot >= 0);
  each_chunk<2>(at, chunks, step, [&](auto us, int64_t c) {
    constexpr int U = decltype(us)::value;
    typename Chunk<T>::vec v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load<false>(x + (c + u * step) * E);
    for (uint64_t left = set; left; left &= left - 1) {
      T *row = out + __builtin_amdgcn_readlane(slot, __builtin_ctzll(left)) * P.rows_stride;
#pragma unroll
      for (int u = 0; u < U; ++u) store<kStream>(row + (c + u * step) * E, v[u]);
    }
  });
  const int64_t i = chunks * E + at;               // the elements behind the last whole chunk
  if (at < E && i < P.width) {
    const T v = x[i];
    for (uint64_t left = set; left; left &= left - 1)
      out[__builtin_amdgcn_readlane(slot, __builtin_ctzll(left)) * P.rows_stride + i] = v;
  }
}

// The same for rows of a line or more that follow each other without a gap and
// begin anywhere in a line.  A row's lines are those that begin in it: the last
// one ends with the next row's first elements, which are read from that row's
// token.  So every line is written whole and once, where two waves on different
// XCDs would write a part each.
template <typename T>
__device__ __forceinline__ void copy_row_lines(const DispatchParams &P, int64_t t, int64_t at, int64_t step, int slot) {
  constexpr int E = Chunk<T>::kElems, kLineElems = kLine / (int)sizeof(T);
  const T *x = static_cast<const T *>(P.x) + t * P.x_stride;
  int next = -1;                                   // lane j: the token of the row behind slot j's
  if (slot >= 0 && slot + 1 < P.off[P.n_experts]) next = P.perm[slot + 1];
  for (uint64_t left = __ballot(slot >= 0); left; left &= left - 1) {
    const int j = __builtin_ctzll(left), r = __builtin_amdgcn_readlane(slot, j), behind = __builtin_amdgcn_readlane(next, j);
    T *row = static_cast<T *>(P.rows) + r * P.width;
    const int64_t head = head_of(row, P.width), lines = (P.width - head) / kLineElems;
    const int64_t i = head + lines * kLineElems + at, chunks = lines * (kLineElems / E);
    const bool ends = at < kLineElems && i < P.width, starts = at < kLineElems && i >= P.width && behind >= 0;
    T last = zero_of<T>();                         // this lane's element of the row's last line
    if (ends) last = x[i];
    if (starts) last = static_cast<const T *>(P.x)[behind * P.x_stride + (i - P.width)];
    each_chunk<4>(at, chunks, step, [&](auto us, int64_t c) {
      constexpr int U = decltype(us)::value;
      typename Chunk<T>::vec v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = load<false>(x + head + (c + u * step) * E);
#pragma unroll
      for (int u = 0; u < U; ++u) store<true>(row + head + (c + u * step) * E, v[u]);
    });
    if (ends || (starts && i - at < P.width)) __builtin_nontemporal_store(last, row + i);
    if (r == 0 && at < head) row[at] = x[at];      // before the first line
  }
}

template <typename T, bool kStream>
__global__ void __launch_bounds__(kThreads) dispatch_kernel(DispatchParams P) {
  extern __shared__ uint32_t lds[];
  const int E = P.n_experts;
  uint32_t *hist = lds, *total = hist + kWaves * E, *start = total + E, *before = start + E + 1;
  int32_t *rows = reinterpret_cast<int32_t *>(before + E);
  const int wave = wave_index(), lane = lane_index();
  const int g = (int)blockIdx.x / P.parts, part = (int)blockIdx.x - g * P.parts;
  const int64_t first = (int64_t)g * P.group;
  int id[kBatches], row[kBatches];
  GroupSums sums;
  load_ids(P, g, wave, lane, id);
  if (P.counts) sums.load(P);
  count_waves(P, id, g, wave, lane, hist, total, start);
  if (P.counts) sums.sum(P, g, before, total);
  expert_starts(E, total, start, wave, lane);
  if (P.n_groups > 1) {
    for (int e = (int)threadIdx.x; e < E; e += kThreads) before[e] += start[e];
    __syncthreads();
  }
  rank_slots(P, id, wave, lane, hist, P.n_groups > 1 ? before : start, row);
  if (blockIdx.x == 0)
    for (int e = (int)threadIdx.x; e <= E; e += kThreads) P.off[e] = (int32_t)start[e];
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    if (b >= P.batches) break;
    const int i = place_of(P, wave, lane, b);
    rows[i] = row[b];
    if (part == 0 && i < P.group && first + i < P.n_slots) {
      P.pos[first + i] = row[b];
      if (row[b] >= 0) P.perm[row[b]] = (int32_t)((first + i) / P.k);
    }
  }
  if (!P.x) return;
  __syncthreads();
  // the group's tokens, `spans` waves each, over the waves of its workgroups
  const int64_t left = P.n_slots - first;
  const int tokens = (int)(left < P.group ? left : P.group) / P.k, spans = (int)P.spans, waves = P.parts * kWaves;
  for (int u = part * kWaves + wave; u < tokens * spans; u += waves) {
    const int t = u / spans;
    copy_row<T, kStream>(P, first / P.k + t, (u - t * spans) * kWave + lane, P.spans * kWave,
                         lane < P.k ? rows[t * P.k + lane] : -1);
  }
}

// A wave takes a token, or one of `spans` parts of its row.
template <typename T, bool kStream, bool kLines>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(DispatchParams P) {
  const int64_t u = (int64_t)blockIdx.x * kCopyWaves + wave_index(), t = u / P.spans;
  if (t >= P.n_slots / P.k) return;
  const int lane = lane_index();
  const int64_t at = (u - t * P.spans) * kWave + lane, step = P.spans * kWave;
  const int slot = lane < P.k ? P.pos[t * P.k + lane] : -1;
  if (kLines) copy_row_lines<T>(P, t, at, step, slot);
  else copy_row<T, kStream>(P, t, at, step, slot);
}

// Narrow rows: G lanes take a token, a chunk each.
template <typename T, int G>
__global__ void __launch_bounds__(kCopyThreads) copy_narrow_kernel(DispatchParams P) {
  const int64_t t = ((int64_t)blockIdx.x * kCopyThreads + threadIdx.x) / G;
  const int c = (int)threadIdx.x % G;
  if (t >= P.n_slots / P.k || c * Chunk<T>::kElems >= P.width) return;
  const auto v = load_chunk(static_cast<const T *>(P.x) + t * P.x_stride, c, P.width);
  for (int j = 0; j < P.k; j += 4) {
    int row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = j + i < P.k ? P.pos[t * P.k + j + i] : -1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row[i] >= 0) store_chunk(static_cast<T *>(P.rows) + row[i] * P.rows_stride, c, P.width, v);
  }
}

__global__ void __launch_bounds__(kThreads) count_kernel(DispatchParams P) {
  extern __shared__ uint32_t lds[];
  const int wave = wave_index(), lane = lane_index();
  int id[kBatches];
  load_ids(P, (int)blockIdx.x, wave, lane, id);
  for (int e = (int)threadIdx.x; e < P.n_experts; e += kThreads) lds[e] = 0;
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBatches; ++b)
    count_ids(lds, id[b], lane);
  __syncthreads();
  for (int e = (int)threadIdx.x; e < P.n_experts; e += kThreads) P.counts[(int64_t)blockIdx.x * P.n_experts + e] = lds[e];
}

// counts[g][e] to the sum over the groups before g, in place, and
// counts[n_groups][e] the sum of all; a wave per expert, a lane per group.
__global__ void __launch_bounds__(kThreads) sum_kernel(DispatchParams P) {
  const int e = (int)blockIdx.x * kWaves + wave_index(), lane = lane_index();
  if (e >= P.n_experts) return;
  uint32_t before = 0;
  for (int g0 = 0; g0 < P.n_groups; g0 += kWave) {
    const int g = g0 + lane;
    uint32_t *at = P.counts + (int64_t)g * P.n_experts + e;
    const uint32_t c = g < P.n_groups ? *at : 0;
    const uint32_t sum = wave_scan(c);
    if (g < P.n_groups) *at = before + sum - c;
    before += (uint32_t)__builtin_amdgcn_readlane((int)sum, kWave - 1);
  }
  if (lane == 0) P.counts[(int64_t)P.n_groups * P.n_experts + e] = before;
}

int32_t group_of(int32_t k) { return kGroupSlots / k * k; }
int64_t groups_of(int64_t slots, int32_t k) { return (slots + group_of(k) - 1) / group_of(k); }
int64_t counts_of(int64_t slots, int32_t k, int32_t n_experts) {
  const int64_t groups = groups_of(slots, k);
  return slots <= kAlone ? 0 : (groups + 1) * n_experts * (int64_t)sizeof(uint32_t);
}

bfs_status check_sizes(const char *what, int64_t n_tokens, int32_t k, int32_t n_experts) {
  if (n_tokens < 0 || k < 1 || n_experts < 1) return fail(BFS_E_INVALID, std::string(what) + ": a negative or zero size");
  if (n_experts > kMaxExperts || k > kMaxK || n_tokens > kMaxTokens)
    return fail(BFS_E_RESOURCE, std::string(what) + ": at most 1024 experts, 64 per token and 2^24 - 1 tokens");
  return BFS_OK;
}

}  // namespace

extern "C" {

bfs_status bfs_moe_dispatch_workspace(int64_t n_tokens, int32_t k, int32_t n_experts, int64_t *bytes) {
  return entry([&]() -> bfs_status {
    bfs_status st = check_sizes("moe_dispatch_workspace", n_tokens, k, n_experts);
    if (st != BFS_OK) return st;
    if (!bytes) return fail(BFS_E_INVALID, "moe_dispatch_workspace: null result");
    *bytes = counts_of(n_tokens * k, k, n_experts);
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
    const int64_t slots = n_tokens * k, groups = groups_of(slots, k), need = counts_of(slots, k, n_experts);
    if (!expert_off || (slots > 0 && (!experts || !perm || !pos))) return fail(BFS_E_INVALID, "moe_dispatch: null buffer");
    if ((x == nullptr) != (rows == nullptr) && slots > 0)
      return fail(BFS_E_INVALID, "moe_dispatch: x and rows are given together");
    if (x && (width < 0 || x_stride < 0 || rows_stride < width))
      return fail(BFS_E_INVALID, "moe_dispatch: negative stride or width, or rows that overlap");
    if (x && width > kMaxWidth) return fail(BFS_E_RESOURCE, "moe_dispatch: at most 2^28 columns");
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
    P.counts = need > 0 ? static_cast<uint32_t *>(workspace) : nullptr;
    P.n_slots = slots;
    P.x_stride = x_stride;
    P.rows_stride = rows_stride;
    P.width = width;
    P.k = k;
    P.n_experts = n_experts;
    P.n_groups = (int32_t)groups;
    P.group = group_of(k);
    P.parts = 1;
    const int64_t in_first = slots < P.group ? slots : P.group;
    P.batches = in_first > 0 ? (int32_t)((in_first + kThreads - 1) / kThreads) : 1;
    while ((1 << P.bits) < n_experts) ++P.bits;
    auto copy = [&](auto t) -> bfs_status {
      using T = decltype(t);
      bfs_status s = BFS_OK;
      if (need > 0) s = launch("moe_dispatch", count_kernel, groups, kThreads, n_experts * sizeof(uint32_t), stream, P);
      if (s == BFS_OK && need > 0 && groups * n_experts > kSumEntries)
        s = launch("moe_dispatch", sum_kernel, (n_experts + kWaves - 1) / kWaves, kThreads, 0, stream, P);
      if (s != BFS_OK) return s;
      const size_t lds = ((kWaves + 3) * (size_t)n_experts + 1 + kGroupSlots) * sizeof(uint32_t);
      const int64_t all = groups > 0 ? groups : 1;
      if (!P.x) return launch("moe_dispatch", dispatch_kernel<T, false>, all, kThreads, lds, stream, P);
      // two waves for a row of four steps and more, one step for each wave where the
      // tokens are fewer than 512
      const int64_t steps = (width + kWave * Chunk<T>::kElems - 1) / (kWave * Chunk<T>::kElems);
      const int64_t wanted = (511 + n_tokens) / n_tokens, least = steps >= 4 ? 2 : 1;
      P.spans = wanted < least ? least : wanted < steps ? wanted : steps;
      const bool stream_rows = (k + 1) * n_tokens * width * (int64_t)sizeof(T) >= kStreamFrom;
      const int64_t in_group = (n_tokens < P.group / k ? n_tokens : P.group / k) * P.spans;
      P.parts = (int32_t)((in_group + kWaves - 1) / kWaves);
      const int64_t row_chunks = (width + Chunk<T>::kElems - 1) / Chunk<T>::kElems;
      const bool narrow = narrow_rows(row_chunks, n_tokens, k);
      // In the caches a launch less is worth more than a wave for each part of a
      // row, while five workgroups and more copy a group's rows (8000 tokens of
      // 2048 bf16 to two: 26.3 us, so 24.6; of 512: 12.7 and 11.9; 32768 of 264 to
      // four, with four workgroups: 28.4 and 32.2).
      if (!stream_rows && !narrow && all * 5 <= kBlocks && all * P.parts > kBlocks) P.parts = (int32_t)(kBlocks / all);
      if (all * P.parts <= kBlocks)
        return launch("moe_dispatch", stream_rows ? dispatch_kernel<T, true> : dispatch_kernel<T, false>, all * P.parts, kThreads,
                      lds, stream, P);
      P.parts = 1;
      P.x = nullptr;
      s = launch("moe_dispatch", dispatch_kernel<T, false>, all, kThreads, lds, stream, P);
      P.x = x;
      if (s != BFS_OK) return s;
      if (narrow)
        return with_group(row_chunks, [&](auto g) {
          constexpr int G = decltype(g)::value;
          return launch("moe_dispatch", copy_narrow_kernel<T, G>, (n_tokens + kCopyThreads / G - 1) / (kCopyThreads / G),
                        kCopyThreads, 0, stream, P);
        });
      // What passes the caches: rows in whole lines where those are shared
      // (32768 tokens of 1409 bf16 to eight: 235 -> 197 us, 5003 to two: 240 ->
      // 198), up to four waves for each; else a wave for each step of a row
      // (4096 to one: 109 -> 100 us, 8192 to two 326 -> 315, 4096 to four 273 and
      // 284), as far as the launch's size goes.
      const int64_t bytes = width * (int64_t)sizeof(T);
      const bool lines = stream_rows && rows_stride == width && bytes >= kLine && ((uintptr_t)rows % kLine || bytes % kLine);
      if (stream_rows && steps >= 4) {
        const int64_t most = (((int64_t)1 << 26) - kCopyWaves) / n_tokens, each = lines ? steps >= 8 ? 4 : 2 : steps;
        P.spans = each < most ? each : most;
      }
      return launch("moe_dispatch", !stream_rows ? copy_kernel<T, false, false> : lines ? copy_kernel<T, true, true>
                                                                                       : copy_kernel<T, true, false>,
                    (n_tokens * P.spans + kCopyWaves - 1) / kCopyWaves, kCopyThreads, 0, stream, P);
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
