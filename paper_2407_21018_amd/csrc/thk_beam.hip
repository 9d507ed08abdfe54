// Beam search: the best continuations of every prompt's beams, and caches that follow their beams.
#include "thk_step.h"

#include <math.h>

#include <algorithm>

namespace thk {
namespace {

typedef unsigned long long u64;

// ---- selection ----------------------------------------------------------------------------
// A row of logits is cut into pieces, a block each.  A block's waves each go over a part of theirs once, with a running maximum and
// sum of exp(x - max) per lane and the part's best K elements as a sorted list, one a lane; a second launch joins the pieces of a
// prompt's rows.  An element is a key: its value in the order of unsigned numbers, above the complement of its index, so that of
// equal values the first is the larger key; 0 is no element.
constexpr int kWaves = 4;
constexpr int kLoads = 4;   // 16-byte loads of a lane for a tile

template <int DT> constexpr int kTileElems = 64 * kLoads * Elem<DT>::VEC;

struct PieceStats { float top; uint32_t bad; double sum; };

__device__ __forceinline__ u64 key_of(float x, uint32_t at) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 is 0
  return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | ~at;
}
__device__ __forceinline__ float value_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ u64 exchange(u64 key, int j, bool larger) {
  const u64 other = __shfl_xor(key, j);
  return (key > other) == larger ? key : other;
}
// 64 keys, one a lane, in descending order
__device__ __forceinline__ u64 sorted(u64 key, int lane) {
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) key = exchange(key, j, ((lane & k) == 0) == ((lane & j) == 0));
  return key;
}
// the largest 64 of two such lists
__device__ __forceinline__ u64 joined(u64 list, u64 more, int lane) {
  const u64 reversed = __shfl_xor(more, 63);
  list = list > reversed ? list : reversed;
#pragma unroll
  for (int j = 32; j > 0; j >>= 1) list = exchange(list, j, (lane & j) == 0);
  return list;
}

__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Joins (top, sum) of all lanes, in an order that does not depend on the values.
__device__ __forceinline__ void join_sums(float &top, double &sum) {
  float t = top;
#pragma unroll
  for (int j = 1; j < 64; j <<= 1) t = fmaxf(t, __shfl_xor(t, j));
  sum = top > -INFINITY ? sum * exp((double)top - (double)t) : 0.0;
#pragma unroll
  for (int j = 1; j < 64; j <<= 1) sum += __shfl_xor(sum, j);
  top = t;
}

template <int DT>
__global__ __launch_bounds__(kWaves * 64) void k_beam_pieces(BeamArgs a, int pieces, int tiles_each) {
  using E = Elem<DT>;
  constexpr int VEC = E::VEC, ELEMS = kLoads * VEC;
  __shared__ u64 pending[kWaves][128];
  __shared__ u64 lists[kWaves][64];
  __shared__ PieceStats stats[kWaves];
  const int64_t row = blockIdx.x / (unsigned)pieces;
  const int piece = (int)(blockIdx.x - row * pieces), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if ((a.done != nullptr && a.done[row] != 0) || !(fabsf(a.scores[row]) < INFINITY)) return;
  const char *const x_row = (const char *)a.logits + row * a.ld * E::EB;
  u64 *const buffer = pending[wave];

  float top = -INFINITY;
  double sum = 0;
  bool bad = false;
  u64 list = 0, least = 0;       // least: the list's last of K, or what is known to be below it
  float least_value = -INFINITY;
  int n = 0;
  auto flush = [&](int count) {
    wave_lds();
    const u64 more = lane < count ? buffer[lane] : 0, rest = buffer[64 + lane];
    wave_lds();
    if (lane < n - count) buffer[lane] = rest;
    n -= count;
    list = joined(list, sorted(more, lane), lane);
    const u64 last = __shfl(list, a.K - 1);
    if (last > least) {
      least = last;
      least_value = value_of(last);
    }
  };

  const int64_t first = ((int64_t)piece * kWaves + wave) * tiles_each;
  for (int64_t tile = first; tile < first + tiles_each; ++tile) {
    const int64_t e0 = tile * kTileElems<DT> + lane * VEC;
    if (tile * kTileElems<DT> >= a.V) break;
    float x[ELEMS];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t e = e0 + i * 64 * VEC;
      float f[VEC];
      if (e + VEC <= a.V) {
        u32x4 r;
        __builtin_memcpy(&r, x_row + e * E::EB, 16);   // (rows start anywhere)
        E::unpack(r, f);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = e + j < a.V ? E::load1(x_row, e + j) : -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i * VEC + j] = f[j];
    }
    float most = x[0];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < ELEMS; ++i) {
      most = fmaxf(most, x[i]);
      nan |= x[i] != x[i];
    }
    bad |= nan || most == INFINITY;
    // the sum
    if (most > top) {
      sum *= exp((double)top - (double)most);   // (0 where there was nothing)
      top = most;
    }
#pragma unroll
    for (int i = 0; i < ELEMS; i += 8) {
      float part = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // 2^y, y = d log2 e with what its rounding leaves
        constexpr float kLog2e = 0x1.715476p0f, kRest = 0x1.4ae0cp-26f;
        const float d = fmaxf(x[i + j] - top, -200.f);   // (-inf, and -inf - -inf)
        const float y = d * kLog2e, left = fmaf(d, kRest, fmaf(d, kLog2e, -y)), p = __builtin_amdgcn_exp2f(y);
        part += fmaf(p, left * 0x1.62e43p-1f, p);
      }
      sum += part;
    }
    // the list
    if (tile == first) {   // a start for `least`: at least K elements are not below the K-th best of the lanes' best
      int at = 0;
#pragma unroll
      for (int i = ELEMS - 1; i >= 0; --i) at = x[i] == most ? i : at;
      const u64 best = most > -INFINITY ? key_of(most, (uint32_t)(e0 + at / VEC * 64 * VEC + at % VEC)) : 0;
      const u64 kth = __shfl(sorted(best, lane), a.K - 1);
      if (kth != 0) {
        least = kth - 1;
        least_value = value_of(kth);
      }
    }
    if (__ballot(most >= least_value && most > -INFINITY) == 0) continue;
#pragma unroll
    for (int i = 0; i < ELEMS; ++i) {
      if (__ballot(x[i] >= least_value && x[i] > -INFINITY) == 0) continue;
      const u64 key = key_of(x[i], (uint32_t)(e0 + i / VEC * 64 * VEC + i % VEC));
      const bool take = x[i] > -INFINITY && key > least;
      const u64 m = __ballot(take);
      if (take) buffer[n + __popcll(m & ((1ull << lane) - 1))] = key;
      n += __popcll(m);
      if (n >= 64) flush(64);
    }
  }
  if (n > 0) flush(n);
  lists[wave][lane] = list;
  join_sums(top, sum);
  bad = __ballot(bad) != 0;
  if (lane == 0) stats[wave] = {top, bad, sum};
  __syncthreads();
  if (wave != 0) return;
  for (int w = 1; w < kWaves; ++w) list = joined(list, lists[w][lane], lane);
  PieceStats s = lane < kWaves ? stats[lane] : PieceStats{-INFINITY, 0, 0.0};
  join_sums(s.top, s.sum);
  s.bad = __ballot(s.bad != 0) != 0;
  if (lane == 0) ((PieceStats *)a.ws)[blockIdx.x] = s;
  u64 *const out = (u64 *)((PieceStats *)a.ws + (int64_t)a.B * a.W * pieces) + (int64_t)blockIdx.x * a.K;
  if (lane < a.K) out[lane] = list;
}

constexpr int kJoinWaves = 8;

// A block joins a prompt: a wave for each row joins its pieces' lists and sums, then the rows' candidates are ranked by counting.
__global__ __launch_bounds__(kJoinWaves * 64) void k_beam_join(BeamArgs a, int pieces) {
  __shared__ double score[kMostBeams * kMostContinuations];
  __shared__ int at[kMostBeams * kMostContinuations];      // beam * 2^24 + token
  __shared__ double live_score[kMostBeams * kMostContinuations];
  __shared__ int live_at[kMostBeams * kMostContinuations];
  __shared__ double kth[kMostBeams];
  __shared__ int ended[kMostBeams];
  __shared__ int n_live;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const PieceStats *const stats = (const PieceStats *)a.ws;
  const u64 *const lists = (const u64 *)(stats + (int64_t)a.B * a.W * pieces);
  if (tid == 0) n_live = 0;
  for (int w = wave; w < a.W; w += kJoinWaves) {
    const int64_t row = b * a.W + w;
    const float before = a.scores[row];
    const bool end = a.done != nullptr && a.done[row] != 0;
    double s = -INFINITY;
    int token = 0;
    if (!(fabsf(before) < INFINITY)) {
    } else if (end) {
      if (lane == 0) s = before;
      token = a.eos;
    } else {
      float top = -INFINITY;
      double sum = 0;
      bool bad = false;
      for (int p = lane; p < pieces; p += 64) {
        const PieceStats x = stats[row * pieces + p];
        bad |= x.bad != 0;
        if (x.top > top) {
          sum = sum * exp((double)top - (double)x.top) + x.sum;
          top = x.top;
        } else if (x.top > -INFINITY) {
          sum += x.sum * exp((double)x.top - (double)top);
        }
      }
      join_sums(top, sum);
      u64 list = lane < a.K ? lists[row * pieces * a.K + lane] : 0;
      for (int p = 1; p < pieces; ++p) {
        const u64 more = lane < a.K ? lists[(row * pieces + p) * a.K + lane] : 0;
        if (__ballot(more > __shfl(list, a.K - 1)) != 0) list = joined(list, more, lane);
      }
      if (__ballot(bad) == 0 && list != 0 && lane < a.K) {
        s = (double)before + (((double)value_of(list) - (double)top) - log(sum));
        token = (int)~(uint32_t)list;
        if (!(fabs(s) < INFINITY)) s = -INFINITY;
      }
    }
    if (lane < a.K) {
      score[w * a.K + lane] = s;
      at[w * a.K + lane] = w << 24 | token;
      if (lane == a.K - 1) kth[w] = s;
    }
    if (lane == 0) ended[w] = end;
  }
  __syncthreads();
  // what is below the K-th of one row is not among the K best of all
  double floor = -INFINITY;
  for (int w = 0; w < a.W; ++w) floor = fmax(floor, kth[w]);
  for (int i = tid; i < a.W * a.K; i += kJoinWaves * 64)
    if (score[i] > -INFINITY && score[i] >= floor) {
      const int to = atomicAdd(&n_live, 1);
      live_score[to] = score[i];
      live_at[to] = at[i];
    }
  __syncthreads();
  const int n = n_live;
  for (int i = tid; i < n; i += kJoinWaves * 64) {
    const double s = live_score[i];
    const int mine = live_at[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += live_score[j] > s || (live_score[j] == s && live_at[j] < mine);
    if (rank >= a.K) continue;
    const int64_t out = b * a.K + rank;
    const int w = mine >> 24, token = mine & 0xffffff;
    a.parent[out] = w;
    a.token[out] = token;
    a.score_out[out] = (float)s;
    if (a.done_out != nullptr) a.done_out[out] = token == a.eos || ended[w] != 0;
  }
  for (int k = n + tid; k < a.K; k += kJoinWaves * 64) {
    const int64_t out = b * a.K + k;
    a.parent[out] = -1;
    a.token[out] = -1;
    a.score_out[out] = -INFINITY;
    if (a.done_out != nullptr) a.done_out[out] = 0;
  }
}

// ---- caches that follow -------------------------------------------------------------------
// A thread has one place of 16 bytes in the tails of all beams of a prompt: it reads the parents' before it writes any, so that
// beams may go on from each other in place.
template <int DT, int W>
__global__ __launch_bounds__(256) void k_reorder_tails(ReorderArgs a, int blocks) {
  constexpr int CPR = kD * Elem<DT>::EB / 16;
  __shared__ int from[kMostBeams], rows[kMostBeams];
  const int64_t g = blockIdx.x / (unsigned)blocks;    // (layer, prompt, head)
  const int64_t lp = g / a.N_kv, h = g - lp * a.N_kv, p = lp % a.prompts;
  const int tid = threadIdx.x;
  if (tid < a.W) {
    const int par = a.parent[p * a.ld_parent + tid];
    const bool other = par >= 0 && par < a.W && par != tid;
    from[tid] = other ? par : -1;
    rows[tid] = other ? min(a.s_tail[p * a.W + par], a.cap) : 0;
  }
  __syncthreads();
  const int64_t c = (blockIdx.x - g * blocks) * 256 + tid, row = c / CPR;
  if (row >= a.cap) return;
  const int64_t stride = (int64_t)a.N_kv * a.cap * CPR, base = (lp * a.W * a.N_kv + h) * a.cap * CPR + c;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    u32x4 *const x = (u32x4 *)(kv ? a.v_tail : a.k_tail) + base;
    u32x4 v[W];
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < a.W && row < rows[j]) v[j] = x[from[j] * stride];
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < a.W && row < rows[j]) x[j * stride] = v[j];
  }
}

// A prompt's table rows and counts, likewise: a thread has one entry of all beams.
__global__ __launch_bounds__(256) void k_reorder_pages(ReorderArgs a) {
  __shared__ int from[kMostBeams], held[kMostBeams], keep[kMostBeams], pages[kMostBeams], tail[kMostBeams];
  const int64_t p = blockIdx.x;
  const int tid = threadIdx.x;
  if (tid < a.W) {
    const int64_t b = p * a.W + tid;
    const int par = a.parent[p * a.ld_parent + tid];
    const bool other = par >= 0 && par < a.W && par != tid;
    from[tid] = other ? par : -1;
    held[tid] = a.max_pages > 0 ? min(max(a.held[b], 0), a.max_pages) : 0;
    pages[tid] = a.s_pages != nullptr ? a.s_pages[b] : 0;
    tail[tid] = a.s_tail != nullptr ? a.s_tail[b] : 0;
  }
  __syncthreads();
  if (tid < a.W) {
    const int64_t b = p * a.W + tid;
    const int f = from[tid];
    if (f >= 0) {
      keep[tid] = (int)min((int64_t)held[f], ((int64_t)max(pages[f], 0) + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift);
      if (a.max_pages > 0) a.held[b] = keep[tid];
      if (a.s_pages != nullptr) a.s_pages[b] = pages[f];
      if (a.s_tail != nullptr) a.s_tail[b] = tail[f];
    }
  }
  __syncthreads();
  int most = 0;
  for (int j = 0; j < a.W; ++j)
    if (from[j] >= 0) most = max(most, max(held[j], keep[j]));
  int32_t *const table = a.table + p * a.W * a.max_pages;
  for (int e = tid; e < most; e += 256) {
    int old[kMostBeams];
#pragma unroll
    for (int j = 0; j < kMostBeams; ++j)
      if (j < a.W) old[j] = table[(int64_t)j * a.max_pages + e];
#pragma unroll
    for (int j = 0; j < kMostBeams; ++j) {
      if (j >= a.W || from[j] < 0) continue;
      const int mine = e < held[j] ? old[j] : -1;
      int now = -1;
#pragma unroll
      for (int i = 0; i < kMostBeams; ++i)
        if (i == from[j] && e < keep[j]) now = old[i];
      if (now != mine) {
        if (mine >= 0 && mine < a.n_pages) atomicAdd(a.refs + mine, -1);
        if (now >= 0 && now < a.n_pages) atomicAdd(a.refs + now, 1);
      }
      table[(int64_t)j * a.max_pages + e] = now;
    }
  }
}

template <class... A>
hipError_t launch(const void *k, int64_t blocks, int threads, hipStream_t st, A... a) {
  void *args[] = {&a...};
  return launch_main_kernel(k, dim3((unsigned)blocks), dim3(threads), args, 0, st);
}

struct BeamPlan { int pieces, tiles_each; };
BeamPlan beam_plan(int dtype, const BeamArgs &a) {
  const int64_t elems = dtype == THK_F32 ? kTileElems<THK_F32> : kTileElems<THK_BF16>, tiles = (a.V + elems - 1) / elems;
  const int64_t each = std::min<int64_t>(std::max<int64_t>(1, (int64_t)a.B * a.W * tiles / (16 * kCUs * kWaves)), 16);
  return {(int)((tiles + each * kWaves - 1) / (each * kWaves)), (int)each};
}

template <int W>
const void *tails_kernel(int dtype) { return dtype == THK_F32 ? (const void *)k_reorder_tails<THK_F32, W> : (const void *)k_reorder_tails<THK_BF16, W>; }

}  // namespace

size_t beam_ws_bytes(int dtype, const BeamArgs &a) {
  const int64_t pieces = beam_plan(dtype, a).pieces, blocks = (int64_t)a.B * a.W * pieces;
  return blocks * kWaves * 64 > 0xffffffffll ? 0 : (size_t)blocks * (sizeof(PieceStats) + a.K * sizeof(u64));
}

hipError_t launch_beam_select(int dtype, const BeamArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const BeamPlan p = beam_plan(dtype, a);
  const hipError_t e = launch(dtype == THK_F32 ? (const void *)k_beam_pieces<THK_F32> : (const void *)k_beam_pieces<THK_BF16>, (int64_t)a.B * a.W * p.pieces,
                              kWaves * 64, st, a, p.pieces, p.tiles_each);
  return e != hipSuccess ? e : launch((const void *)k_beam_join, a.B, kJoinWaves * 64, st, a, p.pieces);
}

hipError_t launch_reorder(int dtype, const ReorderArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  if (a.cap > 0) {
    const int blocks = (int)((a.cap * (int64_t)(dtype == THK_F32 ? 32 : 16) + 255) / 256);
    const void *k = a.W <= 4 ? tails_kernel<4>(dtype) : a.W <= 8 ? tails_kernel<8>(dtype) : a.W <= 16 ? tails_kernel<16>(dtype) : tails_kernel<32>(dtype);
    const hipError_t e = launch(k, a.L * a.prompts * a.N_kv * blocks, 256, st, a, blocks);
    if (e != hipSuccess) return e;
  }
  return launch((const void *)k_reorder_pages, a.prompts, 256, st, a);
}

}  // namespace thk
