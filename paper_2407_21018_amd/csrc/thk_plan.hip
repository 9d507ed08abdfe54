// The plan of a serving step: which sequence, position and rows each new token has (token map), which pages each sequence has
// (reserve), and the copies of pages that stop being shared.  Latency bounds the first two: a few trips to memory each.
#include "thk_step.h"

#include <algorithm>

namespace thk {
namespace {

// Sum of x over the lanes in front (of a wave), and of all lanes.
struct WaveSum { int64_t before, all; };
__device__ __forceinline__ WaveSum wave_sum(int64_t x) {
  const int lane = threadIdx.x & 63;
  int64_t s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  return {s - x, __shfl(s, 63)};
}

// ---- token map ----------------------------------------------------------------------------
constexpr int kMapThreads = 256;

// starts[b]: tokens in front of sequence b, at most n, and starts[B].  By one block.
template <int THREADS, class Put>
__device__ __forceinline__ void running_sums(const TokenMapArgs &a, int64_t *wave_total, Put put) {
  const int tid = threadIdx.x, wave = tid >> 6;
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += THREADS) {
    const int b = b0 + tid;
    const int64_t x = b >= a.B ? 0 : a.n_new == nullptr ? 1 : max(a.n_new[b], 0);
    const WaveSum w = wave_sum(x);
    if ((tid & 63) == 63) wave_total[wave] = w.all;
    __syncthreads();
    int64_t before = base + w.before;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
      if (i < wave) before += wave_total[i];
      base += wave_total[i];
    }
    if (b < a.B) put(b, (int)min(before, a.n));
    __syncthreads();
  }
  if (tid == 0) put(a.B, (int)min(base, a.n));
}

__device__ __forceinline__ void put_token(const TokenMapArgs &a, const int *starts, int64_t t) {
  i32x4 r = {-1, 0, -1, -1};
  if (t < starts[a.B]) {
    int lo = 0, hi = a.B;   // starts[lo] <= t < starts[hi]; of sequences without a token the last one goes on
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int64_t i = t - starts[lo], all = a.n_new == nullptr ? 1 : a.n_new[lo];
    const int64_t row = (a.row0 != nullptr ? a.row0[lo] : 0) + i, q_row = i - (all - a.q_rows);
    r[0] = lo;
    r[1] = (int)((uint32_t)a.pos0[lo] + (uint32_t)i);
    r[2] = row >= 0 && row < a.cap ? (int)row : -1;
    r[3] = q_row >= 0 ? (int)q_row : -1;
  }
  *(i32x4 *)(a.map + t * 4) = r;
}

// Every block makes the running sums of all sequences for itself: a trip to memory and some barriers, less than a second launch.
__global__ __launch_bounds__(kMapThreads) void k_token_map(TokenMapArgs a) {
  __shared__ int starts[kMapSequences + 1];
  __shared__ int64_t wave_total[kMapThreads / 64];
  running_sums<kMapThreads>(a, wave_total, [&](int b, int s) { starts[b] = s; });
  __syncthreads();
  if (blockIdx.x == 0 && a.starts != nullptr)
    for (int b = threadIdx.x; b <= a.B; b += kMapThreads) a.starts[b] = starts[b];
  const int64_t t = (int64_t)blockIdx.x * kMapThreads + threadIdx.x;
  if (t < a.n) put_token(a, starts, t);
}

// More sequences than that: the sums first, in memory.
__global__ __launch_bounds__(1024) void k_starts(TokenMapArgs a) {
  __shared__ int64_t wave_total[16];
  running_sums<1024>(a, wave_total, [&](int b, int s) { a.starts[b] = s; });
}
__global__ __launch_bounds__(kMapThreads) void k_token_map_of(TokenMapArgs a) {
  const int64_t t = (int64_t)blockIdx.x * kMapThreads + threadIdx.x;
  if (t < a.n) put_token(a, a.starts, t);
}

// ---- pages --------------------------------------------------------------------------------
// refs is written by atomic operations, which the L2 carries out, and read past the L1, so that one block's phases see each
// other's writes: a phase ends when its own have come back.
__device__ __forceinline__ int refs_at(const int32_t *refs, int64_t p) { return __hip_atomic_load(refs + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ int refs_add(int32_t *refs, int64_t p, int x) { return __hip_atomic_fetch_add(refs + p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refs_set(int32_t *refs, int64_t p, int x) { __hip_atomic_store(refs + p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void phase_end() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// A sequence's wishes.  `plan` in memory: what the phases tell each other.
struct SequencePlan {
  int have, need;   // pages kept, pages wanted
  int from;         // page that is to be replaced, -1: none
  int start;        // wishes of the sequences in front
};
constexpr int kOwner = -(1 << 30);   // + b: marks a page whose users all grow with the first of them

__device__ __forceinline__ SequencePlan wishes(const ReserveArgs &a, int b, int &held, bool &grows) {
  SequencePlan s;
  const int64_t rows = max(a.rows[b], 0);
  held = min(max(a.held[b], 0), a.max_pages);
  s.need = (int)min((rows + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift, (int64_t)a.max_pages);
  s.have = min(held, s.need);
  s.from = -1;
  s.start = 0;
  grows = false;
  if (a.now != nullptr) {
    const int now = a.now[b];
    const int64_t e = now >> a.page_shift;
    grows = now > 0 && rows > now && (now & ((1 << a.page_shift) - 1)) != 0 && e < s.have;
    if (grows) {
      s.from = a.table[(int64_t)b * a.max_pages + e];
      grows = s.from >= 0 && s.from < a.n_pages;
      if (!grows) s.from = -1;
    }
  }
  return s;
}

constexpr int kPlanThreads = 1024;

// Everything by one block.
__global__ __launch_bounds__(kPlanThreads) void k_reserve(ReserveArgs a) {
  constexpr int WAVES = kPlanThreads / 64, EACH = 8;   // EACH: pages a thread looks at in a step
  __shared__ int64_t wave_total[WAVES];
  __shared__ int counts[EACH * WAVES];
  __shared__ int n_ending, ending[kPlanThreads];
  SequencePlan *const plan = (SequencePlan *)a.ws;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // what sequences give back: by a wave for each that gives something
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    if (tid == 0) n_ending = 0;
    __syncthreads();
    const int b = b0 + tid;
    if (b < a.B) {
      int held;
      bool grows;
      const SequencePlan s = wishes(a, b, held, grows);
      plan[b] = s;
      if (held > s.need) ending[atomicAdd(&n_ending, 1)] = b;
      if (grows) {}
    }
    phase_end();
    for (int i = wave; i < n_ending; i += WAVES) {
      const int g = ending[i], held = min(max(a.held[g], 0), a.max_pages);
      int32_t *const row = a.table + (int64_t)g * a.max_pages;
      for (int e = plan[g].need + lane; e < held; e += 64) {
        const int p = row[e];
        row[e] = -1;
        if (p >= 0 && p < a.n_pages) refs_add(a.refs, p, -1);
      }
    }
    phase_end();
  }
  // pages that several use and at least one of them is to write
  if (a.now != nullptr) {
    for (int b = tid; b < a.B; b += kPlanThreads)
      if (plan[b].from >= 0) refs_add(a.refs, plan[b].from, -1);
    phase_end();
    for (int b = tid; b < a.B; b += kPlanThreads)
      if (plan[b].from >= 0 && refs_at(a.refs, plan[b].from) <= 0) __hip_atomic_fetch_min(a.refs + plan[b].from, kOwner + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    phase_end();
    // (the owner's page gets its number back when all have looked)
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
      const int b = b0 + tid;
      const bool owner = b < a.B && plan[b].from >= 0 && refs_at(a.refs, plan[b].from) == kOwner + b;
      if (owner) plan[b].from = -2 - plan[b].from;
    }
    phase_end();
    for (int b = tid; b < a.B; b += kPlanThreads)
      if (plan[b].from < -1) {
        refs_set(a.refs, -2 - plan[b].from, 1);
        plan[b].from = -1;
      }
    phase_end();
  }
  // wishes in order
  int64_t wanted = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    SequencePlan s{};
    int want = 0;
    if (b < a.B) {
      s = plan[b];
      want = (s.from >= 0) + s.need - s.have;
    }
    const WaveSum w = wave_sum(want);
    if (lane == 63) wave_total[wave] = w.all;
    __syncthreads();
    int64_t before = wanted + w.before;
    for (int i = 0; i < WAVES; ++i) {
      if (i < wave) before += wave_total[i];
      wanted += wave_total[i];
    }
    if (b < a.B) plan[b].start = (int)min(before, (int64_t)INT32_MAX);
    __syncthreads();
  }
  phase_end();
  // free pages in order: the one of rank k fulfils wish k
  int64_t found = 0;
  for (int64_t p0 = 0; p0 < a.n_pages && found < wanted; p0 += EACH * kPlanThreads) {
    bool free[EACH];
    int before[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t p = p0 + i * kPlanThreads + tid;
      free[i] = p < a.n_pages && refs_at(a.refs, p) <= 0;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint64_t m = __ballot(free[i]);
      before[i] = __popcll(m & ((1ull << lane) - 1));
      if (lane == 0) counts[i * WAVES + wave] = __popcll(m);
    }
    __syncthreads();
    int sum = 0, mine[EACH];
    for (int i = 0; i < EACH * WAVES; ++i) {
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (i == j * WAVES + wave) mine[j] = sum;
      sum += counts[i];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t k = found + mine[i] + before[i];
      if (!free[i] || k >= wanted) continue;
      const int p = (int)(p0 + i * kPlanThreads + tid);
      int lo = 0, hi = a.B;   // the last sequence that starts at or before wish k
      while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (plan[mid].start <= k) lo = mid;
        else hi = mid;
      }
      const SequencePlan s = plan[lo];
      const int nth = (int)(k - s.start) - (s.from >= 0);
      const int e = nth < 0 ? a.now[lo] >> a.page_shift : s.have + nth;
      a.table[(int64_t)lo * a.max_pages + e] = p;
      refs_set(a.refs, p, 1);
      if (nth < 0) {
        const int rows = a.now[lo] & ((1 << a.page_shift) - 1);
        *(i32x4 *)(a.moves + (int64_t)lo * 4) = i32x4{s.from, p, (rows + kTile - 1) / kTile, 0};
      }
    }
    found += sum;
    __syncthreads();
  }
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const SequencePlan s = plan[b];
    const int moved = s.from >= 0, want = moved + s.need - s.have;
    const int got = (int)min(max(found - s.start, (int64_t)0), (int64_t)want);
    const bool stuck = moved && got == 0;
    const int held = s.have + got - (moved && !stuck);
    a.held[b] = held;
    a.room[b] = stuck ? a.now[b] : held << a.page_shift;
    if (stuck) refs_add(a.refs, s.from, 1);
    if (a.moves != nullptr && (!moved || stuck)) *(i32x4 *)(a.moves + (int64_t)b * 4) = i32x4{-1, -1, 0, 0};
  }
}

// ---- copies -------------------------------------------------------------------------------
// `parts` blocks for a record, layer and KV head, whose tiles lie side by side.
__global__ __launch_bounds__(256) void k_paged_copy(PagedCopyArgs a, int parts) {
  const int64_t g = blockIdx.x / (unsigned)parts, i = g / a.units, unit = g - i * a.units;
  const i32x4 m = *(const i32x4 *)(a.moves + i * 4);
  if (m[0] < 0 || m[0] >= a.p.n_pages || m[1] < 0 || m[1] >= a.p.n_pages) return;
  const int64_t l = unit / a.p.N_kv, h = unit - l * a.p.N_kv, part = (int64_t)a.p.lay.tile_bytes << a.p.tpp_shift;
  char *const base = (char *)a.p.pool + (l * a.p.n_pages * a.p.N_kv + h) * part;
  const u32x4 *const src = (const u32x4 *)(base + m[0] * part * a.p.N_kv);
  u32x4 *const dst = (u32x4 *)(base + m[1] * part * a.p.N_kv);
  const int pieces = min(max(m[2], 0), 1 << a.p.tpp_shift) * (a.p.lay.tile_bytes / 16);
  for (int c = (int)(blockIdx.x - g * parts) * 256 + threadIdx.x; c < pieces; c += parts * 256) dst[c] = src[c];
}

template <class... A>
hipError_t launch(const void *k, int64_t blocks, int threads, hipStream_t st, A... a) {
  void *args[] = {&a...};
  return launch_main_kernel(k, dim3((unsigned)blocks), dim3(threads), args, 0, st);
}

}  // namespace

hipError_t launch_token_map(const TokenMapArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const int64_t blocks = std::max<int64_t>(1, (a.n + kMapThreads - 1) / kMapThreads);
  if (a.B <= kMapSequences) return launch((const void *)k_token_map, blocks, kMapThreads, st, a);
  const hipError_t e = launch((const void *)k_starts, 1, 1024, st, a);
  return e != hipSuccess || a.n == 0 ? e : launch((const void *)k_token_map_of, blocks, kMapThreads, st, a);
}

size_t reserve_ws_bytes(int64_t B) { return (size_t)B * sizeof(SequencePlan); }
hipError_t launch_reserve(const ReserveArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  return launch((const void *)k_reserve, 1, kPlanThreads, st, a);
}

hipError_t launch_paged_copy(const PagedCopyArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const int64_t groups = a.n * a.units;
  const int parts = (int)std::min<int64_t>(std::max<int64_t>(1, 8 * kCUs / groups), 8);
  return launch((const void *)k_paged_copy, groups * parts, 256, st, a, parts);
}

}  // namespace thk
