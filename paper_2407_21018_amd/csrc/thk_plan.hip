// The plan of a serving step: which sequence, position and rows each new token has (token map), which pages each sequence has
// (reserve), and the copies of pages that stop being shared.  Latency bounds the first two: a few trips to memory each.
#include "thk_step.h"

#include <algorithm>

namespace thk {
namespace {

typedef unsigned long long u64;

// Sum of x over the lanes in front (of a wave), and of all lanes.
template <class I> struct WaveSum { I before, all; };
template <class I>
__device__ __forceinline__ WaveSum<I> wave_sum(I x) {
  const int lane = threadIdx.x & 63;
  I s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const I y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  return {s - x, __shfl(s, 63)};
}

// ---- token map ----------------------------------------------------------------------------
constexpr int kMapThreads = 256;

// starts[b]: tokens in front of sequence b, at most n, and starts[B].  By one block, EACH sequences a thread at a time.
template <int THREADS, int EACH, class Put>
__device__ __forceinline__ void running_sums(const TokenMapArgs &a, int64_t (*wave_total)[THREADS / 64], Put put) {
  const int tid = threadIdx.x, wave = tid >> 6;
  int64_t base = 0;
  for (int b0 = 0, turn = 0; b0 < a.B; b0 += THREADS * EACH, turn ^= 1) {
    int64_t x[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int b = b0 + tid * EACH + i;
      x[i] = a.n_new == nullptr ? 1 : max(a.n_new[min(b, a.B - 1)], 0);
      if (b >= a.B) x[i] = 0;
      sum += x[i];
    }
    const WaveSum<int64_t> w = wave_sum(sum);
    if ((tid & 63) == 63) wave_total[turn][wave] = w.all;
    __syncthreads();
    int64_t before = base + w.before;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
      if (i < wave) before += wave_total[turn][i];
      base += wave_total[turn][i];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int b = b0 + tid * EACH + i;
      if (b < a.B) put(b, (int)min(before, a.n));
      before += x[i];
    }
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

// Every block makes the running sums of all sequences for itself: a trip to memory and some barriers, less than a second launch.  4 sequences and
// tokens 2.1 us, 1024 and 104275 3.9 us (1.7 MB written; a launch takes 2), 4096 and 12000 6.6, 4096 and 320000 11.6.
__global__ __launch_bounds__(kMapThreads) void k_token_map(TokenMapArgs a) {
  __shared__ int starts[kMapSequences + 1];
  __shared__ int64_t wave_total[2][kMapThreads / 64];
  auto put = [&](int b, int s) { starts[b] = s; };
  if (a.B <= kMapThreads) running_sums<kMapThreads, 1>(a, wave_total, put);
  else running_sums<kMapThreads, 4>(a, wave_total, put);
  __syncthreads();
  if (blockIdx.x == 0 && a.starts != nullptr)
    for (int b = threadIdx.x; b <= a.B; b += kMapThreads) a.starts[b] = starts[b];
  const int64_t t = (int64_t)blockIdx.x * kMapThreads + threadIdx.x;
  if (t < a.n) put_token(a, starts, t);
}

// More sequences than that: the sums first, in memory.  4097 sequences and 12000 tokens 5.5 + 4.9 us, 320000 tokens 5.5 + 6.0.
__global__ __launch_bounds__(1024) void k_starts(TokenMapArgs a) {
  __shared__ int64_t wave_total[2][16];
  running_sums<1024, 4>(a, wave_total, [&](int b, int s) { a.starts[b] = s; });
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

// A sequence's wishes.  In the workspace: what the phases tell each other.
struct SequencePlan {
  int have, need;   // pages kept, pages wanted
  int from;         // page that is to be replaced, -1: none
  int start;        // wishes of the sequences in front
};

__device__ __forceinline__ int held_of(const ReserveArgs &a, int b) { return min(max(a.held[b], 0), a.max_pages); }
__device__ __forceinline__ int needed(const ReserveArgs &a, int b) {
  const int64_t rows = max(a.rows[b], 0);
  return (int)min((rows + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift, (int64_t)a.max_pages);
}
// The page that holds some of the rows of a sequence that is to grow, -1: none.  have: pages that it keeps.
__device__ __forceinline__ int growing_page(const ReserveArgs &a, int b, int have) {
  const int now = a.now[b], e = now >> a.page_shift;
  if (now <= 0 || a.rows[b] <= now || (now & ((1 << a.page_shift) - 1)) == 0 || e >= have) return -1;
  const int p = a.table[(int64_t)b * a.max_pages + e];
  return p >= 0 && p < a.n_pages ? p : -1;
}
// Rows that a growing sequence has in that page, fewer than 2^16.  Of users that all grow the one with the most of them keeps the page, of several the
// first: it writes behind them, so that those for whom no page is left, and who stay in it, keep their rows.
__device__ __forceinline__ int rows_inside(const ReserveArgs &a, int b) { return a.now[b] & ((1 << a.page_shift) - 1); }
// A wave gives back the entries [from, to) of sequence b.
__device__ __forceinline__ void give_back(const ReserveArgs &a, int b, int from, int to, int lane) {
  int32_t *const row = a.table + (int64_t)b * a.max_pages;
  for (int e0 = from; e0 < to; e0 += 256) {
    int p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = row[min(e0 + i * 64 + lane, to - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e0 + i * 64 + lane >= to) break;
      row[e0 + i * 64 + lane] = -1;
      if (p[i] >= 0 && p[i] < a.n_pages) refs_add(a.refs, p[i], -1);
    }
  }
}
// Wish k, of sequence b whose wishes begin at `start`, gets page p.
__device__ __forceinline__ void grant(const ReserveArgs &a, int b, int64_t k, int start, int have, int from, int p) {
  const int nth = (int)(k - start) - (from >= 0);
  const int e = nth < 0 ? a.now[b] >> a.page_shift : have + nth;
  a.table[(int64_t)b * a.max_pages + e] = p;
  refs_set(a.refs, p, 1);
  if (nth < 0) {
    *(i32x4 *)(a.moves + (int64_t)b * 4) = i32x4{from, p, (rows_inside(a, b) + kTile - 1) / kTile, 0};
    refs_add(a.refs, from, -1);
  }
}
// ... of `found` free pages: what the sequence has now.
__device__ __forceinline__ void settle(const ReserveArgs &a, int b, int64_t found, int start, int have, int from, int want) {
  const bool moved = from >= 0;
  const int got = (int)min(max(found - start, (int64_t)0), (int64_t)want);
  const bool stuck = moved && got == 0;
  const int held = have + got - (moved && !stuck);
  a.held[b] = held;
  a.room[b] = stuck ? a.now[b] : held << a.page_shift;
  if (a.moves != nullptr && (!moved || stuck)) *(i32x4 *)(a.moves + (int64_t)b * 4) = i32x4{-1, -1, 0, 0};
}

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
constexpr int kPlanEach = 4, kPlanSequences = kPlanEach * kPlanThreads;   // sequences of a thread, and of a block, in LDS, at most

// Which of the pages that several use have to be replaced for whom: the growing users of a page meet in a table in LDS.
template <int THREADS, int EACH>
struct Meeting {
  int page[2 * EACH * THREADS], count[2 * EACH * THREADS];   // as many slots are used as twice the sequences, up to a power of two
  uint32_t mask;
  __device__ __forceinline__ void clear(int B, int tid) {
    const uint32_t m = (2u << (32 - __builtin_clz(max(B - 1, 1)))) - 1;
    if (tid == 0) mask = m;
    for (uint32_t i = tid; i <= m; i += THREADS) {
      page[i] = -1;
      count[i] = 0;
    }
  }
  __device__ __forceinline__ int enter(int p) {
    uint32_t at = ((uint32_t)p * 2654435761u) >> 7;
    for (;; ++at) {   // (fewer pages than slots)
      const int was = atomicCAS(&page[at & mask], -1, p);
      if (was == -1 || was == p) break;
    }
    atomicAdd(&count[at & mask], 1);
    return at & mask;
  }
};
template <bool MOVES, int THREADS, int EACH> struct MeetingOf { Meeting<THREADS, EACH> m; };
template <int THREADS, int EACH> struct MeetingOf<false, THREADS, EACH> { };

constexpr int kPagesEach = 8;   // pages that a thread looks at in a step
template <int THREADS, int EACH>
struct PlanLds {
  int start[EACH * THREADS], have[EACH * THREADS], from[EACH * THREADS];
  int64_t wave_total[2][THREADS / 64];
  int total;
  union {
    struct { int ending[EACH * THREADS], held[EACH * THREADS]; };
    int pages[kPagesEach * THREADS];   // free ones, in order
  };
};

// The block's sequences: what they give back (ONE), whose growing page is to be replaced, and their wishes in order.  Returns all wishes.
template <bool ONE, bool MOVES, int THREADS, int EACH>
__device__ __forceinline__ int64_t plan_sequences(const ReserveArgs &a, PlanLds<THREADS, EACH> &s, MeetingOf<MOVES, THREADS, EACH> &meeting, int (&want)[EACH]) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int need[EACH], have[EACH], from[EACH], held[EACH];
  if (tid == 0) s.total = 0;
  if constexpr (MOVES) meeting.m.clear(a.B, tid);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int b = i * THREADS + tid;
    need[i] = have[i] = held[i] = 0;
    from[i] = -1;
    if (b >= a.B) continue;
    need[i] = needed(a, b);
    held[i] = held_of(a, b);
    have[i] = min(held[i], need[i]);
    if constexpr (MOVES) from[i] = growing_page(a, b, have[i]);
  }
  __syncthreads();
  if constexpr (ONE) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int b = i * THREADS + tid;
      if (held[i] > need[i]) s.ending[atomicAdd(&s.total, 1)] = b;
      if (b < a.B) {
        s.have[b] = have[i];
        s.held[b] = held[i];
      }
    }
    __syncthreads();
    for (int i = wave; i < s.total; i += (THREADS / 64)) give_back(a, s.ending[i], s.have[s.ending[i]], s.held[s.ending[i]], lane);
    if (s.total > 0) phase_end();
  }
  if constexpr (MOVES) {
    Meeting<THREADS, EACH> &m = meeting.m;
    int slot[EACH], users[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      slot[i] = from[i] >= 0 ? m.enter(from[i]) : -1;
      users[i] = from[i] >= 0 ? refs_at(a.refs, from[i]) : 0;
    }
    __syncthreads();
    bool all[EACH];   // all users of the page grow: one of them keeps it
#pragma unroll
    for (int i = 0; i < EACH; ++i) all[i] = slot[i] >= 0 && m.count[slot[i]] >= users[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (all[i]) m.count[slot[i]] = 0;
    __syncthreads();
    int rank[EACH];   // by its rows, then backwards by its number
    static_assert(EACH * THREADS <= 1 << 12 && kMostTilesOfPage * kTile <= 1 << 16);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      rank[i] = all[i] ? rows_inside(a, i * THREADS + tid) << 12 | ((1 << 12) - 1 - (i * THREADS + tid)) : 0;
      if (all[i]) atomicMax(&m.count[slot[i]], rank[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (all[i] && m.count[slot[i]] == rank[i]) from[i] = -1;
  }
  int64_t wanted = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    want[i] = (from[i] >= 0) + need[i] - have[i];
    if (i * THREADS >= a.B) continue;
    const int b = i * THREADS + tid;
    const WaveSum<uint32_t> w = wave_sum((uint32_t)want[i]);   // (fewer than 2^25 each)
    if (lane == 63) s.wave_total[i & 1][wave] = w.all;
    __syncthreads();
    int64_t before = wanted + w.before;
#pragma unroll
    for (int j = 0; j < (THREADS / 64); ++j) {
      const int64_t x = s.wave_total[i & 1][j];
      before += j < wave ? x : 0;
      wanted += x;
    }
    if (b < a.B) {
      s.start[b] = (int)min(before, (int64_t)INT32_MAX);
      s.have[b] = have[i];
      s.from[b] = from[i];
    }
  }
  __syncthreads();
  return wanted;
}

// The last sequence whose wishes start at or before wish k.
__device__ __forceinline__ int wisher(const int *start, int B, int64_t k) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (start[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Everything by one block: latency is all there is to it, of memory for few sequences and pages and of instructions otherwise, which sixteen
// waves of a compute unit share.  A block of four waves takes 3.0 us for 4 sequences and 96 pages, one of sixteen 4.1; 64 sequences and 8000
// pages 4.2 and 4.6, 64 and 16000 5.1 and 4.5, 200 and 4000 6.4 and 5.2.
constexpr int kFew = 64, kFewPages = 8192;
template <bool MOVES, int THREADS>
__global__ __launch_bounds__(THREADS) void k_reserve_one(ReserveArgs a) {
  constexpr int PAGES = kPagesEach, kStep = PAGES * THREADS;   // a wave's pages lie side by side
  __shared__ PlanLds<THREADS, 1> s;
  __shared__ MeetingOf<MOVES, THREADS, 1> meeting;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int want[1];
  const int64_t wanted = plan_sequences<true, MOVES, THREADS, 1>(a, s, meeting, want);
  // free pages in order: the one of rank k fulfils wish k
  int64_t found = 0;
  int users[PAGES];
  auto look = [&](int64_t p0) {
#pragma unroll
    for (int i = 0; i < PAGES; ++i) {
      const int64_t p = p0 + (wave * PAGES + i) * 64 + lane;
      users[i] = refs_at(a.refs, min(p, a.n_pages - 1));   // (all loads under way at once)
    }
  };
  if (wanted > 0) look(0);
  for (int64_t p0 = 0, step = 0; p0 < a.n_pages && found < wanted; p0 += kStep, ++step) {
    u64 free[PAGES];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) {
      free[i] = __ballot(users[i] <= 0 && p0 + (wave * PAGES + i) * 64 + lane < a.n_pages);
      mine += __popcll(free[i]);
    }
    if (lane == 0) s.wave_total[step & 1][wave] = mine;
    __syncthreads();
    int k = 0, here = 0;
#pragma unroll
    for (int j = 0; j < THREADS / 64; ++j) {
      const int x = (int)s.wave_total[step & 1][j];
      k += j < wave ? x : 0;
      here += x;
    }
    if (found + here < wanted) look(p0 + kStep);
    const int most = (int)min((int64_t)here, wanted - found);
#pragma unroll
    for (int i = 0; i < PAGES; ++i) {
      const int rank = k + __popcll(free[i] & ((1ull << lane) - 1));
      k += __popcll(free[i]);
      if ((free[i] >> lane & 1) != 0 && rank < most) s.pages[rank] = (int)(p0 + (wave * PAGES + i) * 64 + lane);
    }
    __syncthreads();
    for (int r = tid; r < most; r += THREADS) {
      const int b = wisher(s.start, a.B, found + r);
      grant(a, b, found + r, s.start[b], s.have[b], s.from[b], s.pages[r]);
    }
    found += here;
  }
  if (tid < a.B) settle(a, tid, found, s.start[tid], s.have[tid], s.from[tid], want[0]);
}

constexpr int64_t kOnePages = 49152;
// More sequences than that block has threads, or pages than this: three launches, which cost 9 us and for many sequences grow more slowly (16 sequences
// and 48000 pages 6.6 us by one block, 8.7 by three launches; 65536 pages 8.8 and 8.8; 1024 sequences and 16000 pages 9.3 and 10.2, 24000 pages 10.5 and
// 10.0; 2000 sequences, two a thread, and 16000 pages 16.3 and 12.3; 4096 and 16000 26 and 16.6).
// What is given back, by a wave for each sequence; the sequences' plan, by one block, and the free pages counted beside it; the pages given out.
constexpr int kChunk = 4096, kChunkThreads = 1024, kChunkWaves = kChunkThreads / 64, kChunkEach = kChunk / kChunkThreads;   // pages that a block looks at together: its part of the pool is as many of them as make
constexpr int kMostChunks = 1024;   // at most so many parts
struct ReserveWs {
  SequencePlan *plan;
  int64_t *wanted;
  int32_t *counts;
};
__host__ __device__ inline ReserveWs reserve_ws(void *ws, int64_t B) {
  char *const p = (char *)ws;
  return {(SequencePlan *)p, (int64_t *)(p + B * sizeof(SequencePlan)), (int32_t *)(p + B * sizeof(SequencePlan) + 16)};
}
__global__ __launch_bounds__(256) void k_give_back(ReserveArgs a) {
  const int64_t b = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (b >= a.B) return;
  const int need = needed(a, (int)b), held = held_of(a, (int)b);
  if (held > need) give_back(a, (int)b, need, held, threadIdx.x & 63);
}
// A thread's pages of a chunk, in order of waves, 64 pages at a time, lanes.
__device__ __forceinline__ void chunk_pages(const ReserveArgs &a, int64_t p0, u64 (&free)[kChunkEach]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int users[kChunkEach];
#pragma unroll
  for (int i = 0; i < kChunkEach; ++i) {
    const int64_t p = p0 + (wave * kChunkEach + i) * 64 + lane;
    users[i] = a.refs[min(p, a.n_pages - 1)];   // (all loads under way at once)
  }
#pragma unroll
  for (int i = 0; i < kChunkEach; ++i) free[i] = __ballot(users[i] <= 0 && p0 + (wave * kChunkEach + i) * 64 + lane < a.n_pages);
}
// Block 0 plans, block 1 + i counts part i: neither needs what the other writes.
static_assert(kPlanThreads == kChunkThreads);
template <bool MOVES>
__global__ __launch_bounds__(kPlanThreads) void k_plan_and_count(ReserveArgs a, int64_t part) {
  __shared__ PlanLds<kPlanThreads, kPlanEach> s;
  __shared__ MeetingOf<MOVES, kPlanThreads, kPlanEach> meeting;
  const ReserveWs w = reserve_ws(a.ws, a.B);
  if (blockIdx.x == 0) {
    int want[kPlanEach];
    const int64_t wanted = plan_sequences<false, MOVES, kPlanThreads, kPlanEach>(a, s, meeting, want);
    if (threadIdx.x == 0) *w.wanted = wanted;
#pragma unroll
    for (int i = 0; i < kPlanEach; ++i) {
      const int b = i * kPlanThreads + threadIdx.x;
      if (b < a.B) w.plan[b] = {s.have[b], s.have[b] + want[i] - (s.from[b] >= 0), s.from[b], s.start[b]};
    }
    return;
  }
  const int64_t i = blockIdx.x - 1;
  if (threadIdx.x == 0) s.total = 0;
  __syncthreads();
  int n = 0;
  for (int64_t p0 = i * part; p0 < min((i + 1) * part, a.n_pages); p0 += kChunk) {
    u64 free[kChunkEach];
    chunk_pages(a, p0, free);
#pragma unroll
    for (int j = 0; j < kChunkEach; ++j) n += __popcll(free[j]);
  }
  if ((threadIdx.x & 63) == 0) atomicAdd(&s.total, n);
  __syncthreads();
  if (threadIdx.x == 0) w.counts[i] = s.total;
}
__global__ __launch_bounds__(kChunkThreads) void k_give_out(ReserveArgs a, int64_t part) {
  __shared__ int start[kPlanSequences], have[kPlanSequences];   // have: its highest bit where a page is to be replaced
  __shared__ int64_t sums[kChunkWaves][2];
  __shared__ int wave_total[2][kChunkWaves], pages[kChunk];
  const ReserveWs w = reserve_ws(a.ws, a.B);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  u64 free[kChunkEach];
  chunk_pages(a, blockIdx.x * part, free);
  const int64_t wanted = *w.wanted;
  int64_t before = 0, all = 0;
  for (int i = tid; i < (int)gridDim.x; i += kChunkThreads) {
    const int x = w.counts[i];
    all += x;
    before += i < (int)blockIdx.x ? x : 0;
  }
  before = wave_sum(before).all;
  all = wave_sum(all).all;
  if (lane == 0) {
    sums[wave][0] = before;
    sums[wave][1] = all;
  }
  for (int b = tid; b < a.B; b += kChunkThreads) {
    const SequencePlan s = w.plan[b];
    start[b] = s.start;
    have[b] = s.have | (s.from >= 0 ? INT32_MIN : 0);
  }
  __syncthreads();
  int64_t ahead = 0, found = 0;   // free pages in front of what is looked at, and in all
#pragma unroll
  for (int j = 0; j < kChunkWaves; ++j) {
    ahead += sums[j][0];
    found += sums[j][1];
  }
  for (int64_t b = (int64_t)blockIdx.x * kChunkThreads + tid; b < a.B; b += (int64_t)gridDim.x * kChunkThreads) {
    const SequencePlan s = w.plan[b];
    settle(a, (int)b, found, s.start, s.have, s.from, (s.from >= 0) + s.need - s.have);
  }
  const int64_t end = min((blockIdx.x + 1) * part, a.n_pages);
  int step = 0;
  for (int64_t p0 = blockIdx.x * part; p0 < end && ahead < wanted; p0 += kChunk, step ^= 1) {
    if (p0 != blockIdx.x * part) chunk_pages(a, p0, free);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kChunkEach; ++i) mine += __popcll(free[i]);
    if (lane == 0) wave_total[step][wave] = mine;
    __syncthreads();
    int k = 0, here = 0;
#pragma unroll
    for (int j = 0; j < kChunkWaves; ++j) {
      k += j < wave ? wave_total[step][j] : 0;
      here += wave_total[step][j];
    }
    const int most = (int)min((int64_t)here, wanted - ahead);
#pragma unroll
    for (int i = 0; i < kChunkEach; ++i) {
      const int rank = k + __popcll(free[i] & ((1ull << lane) - 1));
      k += __popcll(free[i]);
      if ((free[i] >> lane & 1) != 0 && rank < most) pages[rank] = (int)(p0 + (wave * kChunkEach + i) * 64 + lane);
    }
    __syncthreads();
    for (int r = tid; r < most; r += kChunkThreads) {
      const int b = wisher(start, a.B, ahead + r), h = have[b];
      grant(a, b, ahead + r, start[b], h & INT32_MAX, h < 0 ? w.plan[b].from : -1, pages[r]);
    }
    ahead += here;
  }
}

// More sequences than a block's LDS holds the plan of, which is what keeps the three launches to 4096: by one block, their plan in memory, every phase
// a trip, which a thread takes for each of its sequences, a search in memory for every page given out.  It is there so that calls of any size are
// answered, not for speed: 4097 sequences and 20550 pages 69 us, 603744 pages 359 us, where 4096 sequences take 19 and 21.
__global__ __launch_bounds__(kPlanThreads) void k_reserve_many(ReserveArgs a) {
  constexpr int EACH = 8;
  __shared__ int64_t wave_total[kPlanWaves];
  __shared__ int n_ending, ending[kPlanThreads];
  SequencePlan *const plan = (SequencePlan *)a.ws;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    if (tid == 0) n_ending = 0;
    __syncthreads();
    const int b = b0 + tid;
    if (b < a.B) {
      const int need = needed(a, b), held = held_of(a, b), have = min(held, need);
      plan[b] = {have, need, a.now != nullptr ? growing_page(a, b, have) : -1, 0};
      if (held > need) ending[atomicAdd(&n_ending, 1)] = b;
    }
    phase_end();
    for (int i = wave; i < n_ending; i += kPlanWaves) give_back(a, ending[i], plan[ending[i]].need, held_of(a, ending[i]), lane);
    phase_end();
  }
  // Pages that several use and at least one of them is to write: the growing users take themselves off the page's count, and where
  // nobody is left they mark it, by the most rows first and then by the first sequence that has so many.  The marks lie below
  // one another, and below all counts.  (start: the sequence is still in question.)
  if (a.now != nullptr) {
    constexpr int kMostRows = -(1 << 29), kFirst = INT32_MIN;   // less the rows; plus the sequence's number, which is below 2^30
    auto mark = [&](int p, int x) { __hip_atomic_fetch_min(a.refs + p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    auto each = [&](auto f) {
      for (int b = tid; b < a.B; b += kPlanThreads)
        if (plan[b].from >= 0) f(b, plan[b]);
      phase_end();
    };
    each([&](int, SequencePlan &s) { refs_add(a.refs, s.from, -1); });
    each([&](int b, SequencePlan &s) { if (refs_at(a.refs, s.from) <= 0) mark(s.from, kMostRows - rows_inside(a, b)); });
    each([&](int b, SequencePlan &s) { s.start = refs_at(a.refs, s.from) == kMostRows - rows_inside(a, b); });
    each([&](int b, SequencePlan &s) { if (s.start != 0) mark(s.from, kFirst + b); });
    each([&](int b, SequencePlan &s) { s.start = refs_at(a.refs, s.from) == kFirst + b; });
    each([&](int, SequencePlan &s) { if (s.start != 0) refs_set(a.refs, s.from, 0); });
    each([&](int, SequencePlan &s) {   // the counts as they were
      refs_add(a.refs, s.from, 1);
      if (s.start != 0) s.from = -1;
    });
  }
  int64_t wanted = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    SequencePlan s{};
    s.from = -1;
    if (b < a.B) s = plan[b];
    const WaveSum<uint32_t> w = wave_sum((uint32_t)((s.from >= 0) + s.need - s.have));   // (fewer than 2^25 each)
    if (lane == 63) wave_total[wave] = w.all;
    __syncthreads();
    int64_t before = wanted + w.before;
    for (int i = 0; i < kPlanWaves; ++i) {
      if (i < wave) before += wave_total[i];
      wanted += wave_total[i];
    }
    if (b < a.B) plan[b].start = (int)min(before, (int64_t)INT32_MAX);
    __syncthreads();
  }
  phase_end();
  int64_t found = 0;
  for (int64_t p0 = 0; p0 < a.n_pages && found < wanted; p0 += EACH * kPlanThreads) {
    u64 free[EACH];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t p = p0 + (wave * EACH + i) * 64 + lane;
      free[i] = __ballot(refs_at(a.refs, min(p, a.n_pages - 1)) <= 0 && p < a.n_pages);
      mine += __popcll(free[i]);
    }
    if (lane == 0) wave_total[wave] = mine;
    __syncthreads();
    int64_t k = found;
    for (int j = 0; j < kPlanWaves; ++j) {
      if (j < wave) k += wave_total[j];
      found += wave_total[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t rank = k + __popcll(free[i] & ((1ull << lane) - 1));
      k += __popcll(free[i]);
      if ((free[i] >> lane & 1) == 0 || rank >= wanted) continue;
      int lo = 0, hi = a.B;
      while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (plan[mid].start <= rank) lo = mid;
        else hi = mid;
      }
      grant(a, lo, rank, plan[lo].start, plan[lo].have, plan[lo].from, (int)(p0 + (wave * EACH + i) * 64 + lane));
    }
  }
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const SequencePlan s = plan[b];
    settle(a, b, found, s.start, s.have, s.from, (s.from >= 0) + s.need - s.have);
  }
}

// ---- copies -------------------------------------------------------------------------------
// `parts` blocks for a record, layer and KV head, whose tiles lie side by side: up to eight, so that small calls fill the card too.  Memory bounds it: 64
// pages of 8 layers and 8 heads, 60 MB read and written, 10 us, part of it in the last-level cache.
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

template <int THREADS>
hipError_t launch_reserve_one(const ReserveArgs &a, hipStream_t st) {
  return launch(a.now != nullptr ? (const void *)k_reserve_one<true, THREADS> : (const void *)k_reserve_one<false, THREADS>, 1, THREADS, st, a);
}

size_t reserve_ws_bytes(int64_t B) { return (size_t)B * sizeof(SequencePlan) + 16 + kMostChunks * sizeof(int32_t); }
hipError_t launch_reserve(const ReserveArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  if (a.B > kPlanSequences) return launch((const void *)k_reserve_many, 1, kPlanThreads, st, a);
  if (a.B <= kFew && a.n_pages <= kFewPages) return launch_reserve_one<256>(a, st);
  if (a.B <= kPlanThreads && a.n_pages <= kOnePages) return launch_reserve_one<kPlanThreads>(a, st);
  const int64_t chunks = (a.n_pages + kChunk - 1) / kChunk, part = (chunks + kMostChunks - 1) / kMostChunks * kChunk, parts = (a.n_pages + part - 1) / part;
  hipError_t e = launch((const void *)k_give_back, (a.B + 3) / 4, 256, st, a);
  if (e == hipSuccess) e = launch(a.now != nullptr ? (const void *)k_plan_and_count<true> : (const void *)k_plan_and_count<false>, 1 + parts, kPlanThreads, st, a, part);
  return e == hipSuccess ? launch((const void *)k_give_out, parts, kChunkThreads, st, a, part) : e;
}

hipError_t launch_paged_copy(const PagedCopyArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const int64_t groups = a.n * a.units;
  const int parts = (int)std::min<int64_t>(std::max<int64_t>(1, 8 * kCUs / groups), 8);
  return launch((const void *)k_paged_copy, groups * parts, 256, st, a, parts);
}

}  // namespace thk
